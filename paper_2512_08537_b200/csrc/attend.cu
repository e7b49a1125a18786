// ardiff_attend_pages: attention of every request's new tokens over its tokens in a paged cache; tokens that a group of requests shares are
// read once for the whole group.
//
//   out = sum_p w_p v_p / sum_p w_p,   w_p = exp(scale q.k_p),   lse = ln sum_p w_p   over the keys p that the query sees.
//
// A sum over keys can be cut anywhere: a piece of it is its largest scale q.k, and sum and weighted values relative to that. So the shared tokens
// and a request's own are different blocks of work, blocks are cut into tiles of keys, and the tiles of all blocks and heads are dealt out
// evenly, in one line, to as many workers as the GPU holds: one request of many keys keeps all SMs busy, and so do many requests of
// different lengths.
//   plan_kernel     checks the call, forms the blocks (whole numbers, one CTA)
//   wide_kernel     blocks of many query rows, on the tensor cores' own pace (attend_wide.cu)
//   narrow_kernel   up to 16 or 32 query rows a block: bound by memory, a worker is a warp
//   join_kernel     joins the pieces of cut blocks, and shared with own tokens
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/ardiff.h"
#include "attend.cuh"
#include "common.cuh"
#include "launch.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace {

using namespace ardiff;

constexpr int kMaxSms = 160;                     // whose workers have places for pieces
constexpr int kPlanThreads = 1024;
// Fewer shared tokens are read by every request itself: a block of its own and the pieces to join cost more than they take.
constexpr int kLeastShared = 64;

// ---- the plan -----------------------------------------------------------------------------------
// What is summed over segments, for narrow and wide ones.
struct Sums {
    long long blocks, rows, steps[2];            // blocks, rows: the narrow ones in the upper half
};
// Exclusive sums over the CTA's threads, and the totals; `s` holds one of a warp each.
__device__ __forceinline__ Sums cta_scan(Sums v, Sums* s, Sums* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto inclusive = [&](Sums x) {
        x.blocks = warp_inclusive(x.blocks); x.rows = warp_inclusive(x.rows); x.steps[0] = warp_inclusive(x.steps[0]); x.steps[1] = warp_inclusive(x.steps[1]);
        return x;
    };
    const Sums inc = inclusive(v);
    __syncthreads();
    if (lane == 31) s[warp] = inc;
    __syncthreads();
    Sums own{0, 0, {0, 0}};
    if (lane < (int)(blockDim.x >> 5)) own = s[lane];
    const Sums w = inclusive(own);
    auto from = [&](long long x, int l) { return __shfl_sync(0xffffffffu, x, l); };
    *total = Sums{from(w.blocks, 31), from(w.rows, 31), {from(w.steps[0], 31), from(w.steps[1], 31)}};
    return Sums{inc.blocks - v.blocks + from(w.blocks - own.blocks, warp), inc.rows - v.rows + from(w.rows - own.rows, warp),
                {inc.steps[0] - v.steps[0] + from(w.steps[0] - own.steps[0], warp), inc.steps[1] - v.steps[1] + from(w.steps[1] - own.steps[1], warp)}};
}
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
    return Sums{a.blocks + b.blocks, a.rows + b.rows, {a.steps[0] + b.steps[0], a.steps[1] + b.steps[1]}};
}

// A segment's blocks: `b` but for the rows' place and what follows from it. The keys that its rows see end at `length` for requests' own tokens.
struct Segment {
    Block b;
    long long rows;
    int length;
    bool wide;
    __device__ __forceinline__ int blocks() const { return rows <= 0 ? 0 : wide ? (int)((rows + kWideRows - 1) / kWideRows) : 1; }
    __device__ __forceinline__ Block block(int j, const Call& c) const {
        Block k = b;
        const int per = wide ? kWideRows : kNarrowRows, tile = wide ? kWideKeys : kNarrowKeys;
        k.row0 = j * per;
        k.rows = (int)min((long long)per, rows - k.row0);
        k.key0 = wide ? k.low / tile * tile : k.low;
        const int last = min(length, k.limit + k.step * c.x.by_G.quotient(k.row0 + k.rows - 1));
        k.keys = last > k.low ? last - k.key0 : 0;
        return k;
    }
    __device__ __forceinline__ int steps(const Block& k, const Call& c) const {
        const int tile = wide ? kWideKeys : kNarrowKeys;
        return (k.keys + tile - 1) / tile * (wide ? c.cache.heads : c.cache.heads / c.plan.team);
    }
    // what the segment adds
    __device__ __forceinline__ Sums sums(const Call& c) const {
        Sums v{0, 0, {0, 0}};
        const int n = blocks(), up = wide ? 0 : 32;
        v.blocks = (long long)n << up;
        v.rows = rows > 0 ? rows << up : 0;
        for (int j = 0; j < n; ++j) v.steps[wide] += steps(block(j, c), c);
        return v;
    }
    // writes its blocks behind those of `before`; whether one of them has no key
    __device__ __forceinline__ bool write(const Call& c, const Sums& before) const {
        const List& l = wide ? c.plan.wide : c.plan.narrow;
        const int at = wide ? (int)before.blocks : (int)(before.blocks >> 32), n = blocks();
        long long step = before.steps[wide], row = wide ? (long long)(int)before.rows : before.rows >> 32;
        bool empty = false;
        for (int j = 0; j < n; ++j) {
            Block k = block(j, c);
            k.first_step = step;
            k.first_row = row;
            l.block[at + j] = k;
            l.steps[at + j] = step;
            step += steps(k, c);
            row += k.rows;
            empty |= k.keys == 0;
        }
        return empty;
    }
};

// Requests whose numbers fit here are read once; of more than that, again from memory.
constexpr int kPlanKept = 1024;

template <bool kKept>
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const Call c) {
    __shared__ Sums s_scan[32];
    __shared__ int s_offset[kKept ? kPlanKept + 1 : 1], s_length[kKept ? kPlanKept : 1];
    __shared__ Share s_share[kKept ? kPlanKept : 1];
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x, R = c.requests, G = c.x.G;
    const long long limit = (long long)c.cache.width * c.cache.page;
    const int* offset = kKept ? s_offset : c.offset;
    const int* length = kKept ? s_length : c.length;
    Share* share = kKept ? s_share : c.plan.share;
    bool bad = false;
    for (int r = tid; r < R; r += threads) {
        const int a = c.offset[r], b = c.offset[r + 1], len = c.length[r];
        bad |= a < 0 || b < a || b > c.x.tokens || len < 0 || len > limit || (c.most > 0 && b - a > c.most);
        if (kKept) {
            s_offset[r] = a;
            if (r + 1 == R) s_offset[R] = b;
            s_length[r] = len;
        }
        share[r] = Share{-1, 0, 0, 0, 0, r, 0, 0};
    }
    for (int g = tid; g < c.groups; g += threads) {
        const int a = c.group[g], b = c.group[g + 1];
        bad |= a < 0 || b < a || b > R || c.shared[g] < 0;
    }
    bad = __syncthreads_or(bad);
    if (tid == 0) *c.status = bad ? ARDIFF_ERR_SHAPE : ARDIFF_OK;
    if (bad) {
        if (tid < 2) *(tid ? c.plan.wide : c.plan.narrow).head = PlanHead{0, 0, 0, 0, 0, 0};
        return;
    }
    Sums before{0, 0, {0, 0}};
    if (c.groups > 0) {
        // The tokens that all queries of a group see are found through its first row of the table, and read once for all, unless
        // one request has queries, or all have so many that each fills its blocks of rows: then the same work is done, and there are no pieces to join.
        for (int g = tid >> 5; g < c.groups; g += threads / 32) {
            const int r0 = c.group[g], r1 = c.group[g + 1];
            int least = r0 < r1 ? min(c.shared[g], length[r0]) : 0, active = 0, fewest = 0x7fffffff;    // (its row holds no more)
            for (int r = r0 + lane; r < r1; r += 32) {
                const int n = offset[r + 1] - offset[r];
                if (n == 0) continue;
                ++active;
                fewest = min(fewest, n);
                least = min(least, max(0, c.causal ? length[r] - n + 1 : length[r]));
            }
            least = __reduce_min_sync(0xffffffffu, least);
            fewest = __reduce_min_sync(0xffffffffu, fewest);
            active = __reduce_add_sync(0xffffffffu, active);
            const bool once = active > 1 && least >= kLeastShared && (long long)fewest * G < kWideRows;
            for (int r = r0 + lane; r < r1; r += 32) share[r] = Share{-1, 0, 0, once ? least : 0, least, r0, 0, 0};
        }
        __syncthreads();
        // shared tokens: the group's rows
        for (int g0 = 0; g0 < c.groups; g0 += threads) {
            const int g = g0 + tid;
            Segment x;
            x.rows = 0;
            x.wide = false;
            int r0 = 0;
            if (g < c.groups) {
                r0 = c.group[g];
                const int r1 = c.group[g + 1], keys = r1 > r0 ? share[r0].shared : 0;
                if (keys > 0) {
                    x.b = Block{offset[r0], 0, 0, r0, 0, keys, 0, keys, 0, 0, r0, 0, 0, 0};
                    x.rows = (long long)(offset[r1] - offset[r0]) * G;
                    x.length = keys;
                    x.wide = x.rows > c.plan.narrow_rows;
                }
            }
            Sums total;
            const Sums at = before + cta_scan(x.sums(c), s_scan, &total);
            if (x.rows > 0) {
                x.write(c, at);
                share[r0].prefix = x.wide ? (int)at.blocks : (int)(at.blocks >> 32);
                share[r0].wide = x.wide;
            }
            before = before + total;
        }
        __syncthreads();
        for (int g = tid >> 5; g < c.groups; g += threads / 32) {
            const int r0 = c.group[g], r1 = c.group[g + 1];
            if (r0 == r1) continue;
            const Share first = share[r0];
            const int token0 = offset[r0];
            __syncwarp();
            for (int r = r0 + lane; r < r1 && first.prefix >= 0; r += 32) {
                Share s = first;
                s.row0 = (offset[r] - token0) * G;
                share[r] = s;
            }
        }
        __syncthreads();
    }
    const int own[2] = {(int)(before.blocks >> 32), (int)before.blocks};
    bool all_rows[2] = {false, false};
    for (int first = 0; first < R; first += threads) {
        const int r = first + tid;
        Segment x;
        x.rows = 0;
        x.wide = false;
        bool joined = false;
        if (r < R) {
            const Share mine = share[r];
            const int token0 = offset[r], news = offset[r + 1] - token0, len = length[r];
            if (kKept) c.plan.share[r] = mine;
            x.b = Block{token0, 0, 0, r, 0, 0, mine.shared, c.causal ? len - news + 1 : len, c.causal, (int)c.cache.by_page.quotient(mine.split), mine.front, 0, 0, 0};
            x.rows = (long long)news * G;
            x.length = len;
            x.wide = x.rows > c.plan.narrow_rows;
            joined = mine.prefix >= 0;
        }
        Sums total;
        const Sums at = before + cta_scan(x.sums(c), s_scan, &total);
        if (x.rows > 0) {
            const bool every = x.write(c, at) || joined;
            all_rows[0] |= every && !x.wide;
            all_rows[1] |= every && x.wide;
        }
        before = before + total;
    }
    const int any[2] = {__syncthreads_or(all_rows[0]) != 0, __syncthreads_or(all_rows[1]) != 0};
    if (tid < 2) {
        const List& l = tid ? c.plan.wide : c.plan.narrow;
        const int blocks = tid ? (int)before.blocks : (int)(before.blocks >> 32);
        const long long steps = tid ? before.steps[1] : before.steps[0];
        l.steps[blocks] = steps;
        *l.head = PlanHead{steps, tid ? before.rows >> 32 : 0, blocks, tid ? own[1] : own[0], tid ? any[1] : any[0], 0};
    }
}

// ---- few query rows -----------------------------------------------------------------------------
constexpr int kWarps = 8;                        // of a CTA, one CTA an SM
constexpr int kThreads = kWarps * 32;

template <int D> constexpr int kPitch16 = 2 * D + 16;                     // bytes from row to row: an odd number of 16-byte places
template <int D> constexpr int kStageBytes = 2 * kNarrowKeys * kPitch16<D>;
template <int D> constexpr int kStages = 28400 / kStageBytes<D> < 6 ? 28400 / kStageBytes<D> : 6;
template <int D> constexpr int kNarrowShared = kWarps * (kStages<D> * kStageBytes<D> + kNarrowKeys * 16 + 4 * 32 * 4);

// Every warp goes its own way (teams: through the same keys as its neighbours): 16 keys of a kv head a step, as many steps under way as its part of shared memory holds (26 to 28 KB: with
// eight warps some 200 KB an SM, more than memory's latency asks for), no meeting with other warps. Lanes look up the places of the keys of the
// step after the next one that is sent for, and copy 16 bytes each. (128 requests of 4096 tokens of 8 heads of 128 values,
// 2.1 GB: 380 us, 5.6 TB/s; 96 short requests of 16 heads of 80, 360 MB: 84 us, 4.3 TB/s; bulk copies of
// single rows, which come at 15 clocks each, took 122; rows loaded straight into the products' registers 183, since a warp then waits for memory in every step.)
// Rows lie 2 D + 16 bytes apart, so that the eight rows of a matrix are in different banks. Query rows are the left operand, 16 rows an
// instruction, or twice that (kTiles == 2): with few rows it is mostly empty, but reading 512 bytes a key and head from memory takes longer than its products.
template <typename T, int D, int kTiles>
__global__ void __launch_bounds__(kThreads, 1) narrow_kernel(const Call c) {
    extern __shared__ __align__(128) char smem[];
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const List& list = c.plan.narrow;
    const long long steps = list.head->steps, each = steps_each<false>(steps, list.workers);
    const int team = D % 64 ? c.plan.team : 1;                                         // (known where rows are whole lines)
    const int worker = warp / team * gridDim.x + blockIdx.x;                    // (few workers: on as many SMs)
    const long long begin = each * worker;
    if (begin >= steps) return;
    const int n = (int)(min(steps, begin + each) - begin), own = list.head->own;
    const char* ring = smem + warp * kStages<D> * kStageBytes<D>;
    longlong2* place = reinterpret_cast<longlong2*>(smem + kWarps * kStages<D> * kStageBytes<D>) + warp * kNarrowKeys;
    // this lane's sums of weights but for the last 32 steps': four rows, a lane beside the other
    float* sums = reinterpret_cast<float*>(smem + kWarps * (kStages<D> * kStageBytes<D> + kNarrowKeys * 16)) + warp * 4 * 32 + lane;
    const uint32_t ring_at = ptx::smem_u32(ring);

    // where this warp is in the line of steps, and what it needs of the block: of products, and of copies some steps ahead
    struct Place {
        int b, h, tile, tiles, key0, keys;       // h: this warp's of the team's heads
        __device__ __forceinline__ void enter(const List& list) {
            key0 = list.block[b].key0;
            keys = list.block[b].keys;
            tiles = (keys + kNarrowKeys - 1) / kNarrowKeys;
            tile = 0;
        }
        // the next step; whether it is another block's (only called while there is one)
        __device__ __forceinline__ bool next(const List& list, int heads, int team) {
            if (++tile < tiles) return false;
            tile = 0;
            h += team;
            if (h < heads) return false;
            h &= team - 1;
            do {
                ++b;
                enter(list);
            } while (tiles == 0);
            return true;
        }
    };
    Place now;
    now.b = find_last(list.steps, list.head->blocks, begin);
    now.enter(list);
    {
        const int in = (int)(begin - list.block[now.b].first_step);
        const int group = in / now.tiles;
        now.tile = in - group * now.tiles;
        now.h = group * team + warp % team;
    }
    Place load = now;                            // the step whose places are looked up next
    const int32_t *table, *front_table;
    int split;
    auto tables = [&]() {
        const Block& b = list.block[load.b];
        table = c.cache.table + (long long)b.request * c.cache.width;
        front_table = c.cache.table + (long long)b.front * c.cache.width;
        split = b.split;
    };
    tables();
    // A lane's key of the step at `load`: its page, not looked at before it is copied a step later (it comes from memory), and where it is in there.
    struct Key {
        int id, row, h;                          // row -1: none
    };
    auto look_up = [&]() -> Key {
        Key k{0, -1, load.h};
        const int in = load.tile * kNarrowKeys + lane;
        if (lane < kNarrowKeys && in < load.keys) {
            const unsigned key = load.key0 + in, pg = c.cache.by_page.quotient(key);
            k.row = (int)(key - pg * c.cache.page);
            k.id = ((int)pg < split ? front_table : table)[pg];
        }
        return k;
    };
    // this lane's chunks of the 16 keys, and of their values
    constexpr int kChunks = D / 8, kCopies = kNarrowKeys * kChunks / 32;
    auto fetch = [&](int step, const Key& k) {
        const bool there = k.row >= 0 && k.id >= 0 && k.id < c.cache.pages;
        if (lane < kNarrowKeys) {
            place[lane] = there ? make_longlong2(offset_of(c.cache.k_page, c.cache.k_token, c.cache.k_head, k.id, k.row, k.h),
                                                 offset_of(c.cache.v_page, c.cache.v_token, c.cache.v_head, k.id, k.row, k.h))
                                : make_longlong2(-1, -1);
            if (k.row >= 0 && !there) *c.status = ARDIFF_ERR_SHAPE;
        }
        const bool missing = __any_sync(0xffffffffu, lane < kNarrowKeys && !there);
        __syncwarp();
        const uint32_t to = ring_at + (step % kStages<D>) * kStageBytes<D>;
        longlong2 p[kCopies];
#pragma unroll
        for (int j = 0; j < kCopies; ++j) p[j] = place[(lane + 32 * j) / kChunks];
        if (!missing) {
#pragma unroll
            for (int j = 0; j < kCopies; ++j) {
                const int row = (lane + 32 * j) / kChunks, ch = lane + 32 * j - row * kChunks;
                const uint32_t at = to + row * kPitch16<D> + ch * 16;
                cp_async16(at, c.cache.k + p[j].x + ch * 16, 16);
                cp_async16(at + kNarrowKeys * kPitch16<D>, c.cache.v + p[j].y + ch * 16, 16);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kCopies; ++j) {
                const int row = (lane + 32 * j) / kChunks, ch = lane + 32 * j - row * kChunks;
                const uint32_t at = to + row * kPitch16<D> + ch * 16, bytes = p[j].x < 0 ? 0 : 16;       // (none: zeros)
                cp_async16(at, c.cache.k + (bytes ? p[j].x + ch * 16 : 0), bytes);
                cp_async16(at + kNarrowKeys * kPitch16<D>, c.cache.v + (bytes ? p[j].y + ch * 16 : 0), bytes);
            }
        }
        cp_async_commit();
        __syncwarp();
    };
    Key first[kStages<D>];                       // (all sent for before one is looked at)
#pragma unroll
    for (int s = 0; s < kStages<D>; ++s) {
        if (s < n) first[s] = look_up();
        if (s + 1 < n && load.next(list, c.cache.heads, team)) tables();
    }
#pragma unroll
    for (int s = 0; s < kStages<D>; ++s) {
        if (s < n) fetch(s, first[s]);
        else cp_async_commit();
    }
    Key found = look_up();

    const int G = c.x.G, quad = lane & 3, row8 = lane >> 2;
    uint32_t q[kTiles][D / 16][4];
    float o[kTiles][D / 8][4], m[kTiles][2], l[kTiles][2];        // l: the last steps' sum of weights
    int lim[kTiles][2], least = 0;               // keys below `least` are seen by all rows of the block
    bool fresh = true, whole = now.tile == 0;
    uint32_t stage = 0;
    const float scale = fabsf(c.scale);
    const uint32_t signs = c.scale < 0.f ? 0x80008000u : 0u;

    for (int i = 0; i < n; ++i) {
        if (fresh) {
            const Block b = list.block[now.b];
            const int end = b.key0 + b.keys;
            least = min(end, b.limit + b.step * (b.row0 / G));
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int in = t * 16 + row8 + 8 * u, row = b.row0 + in;
                    const bool there = in < b.rows;
                    const int tok = c.x.by_G.quotient(row), head = now.h * G + row - tok * G;
                    lim[t][u] = there ? min(end, b.limit + b.step * tok) : end;
                    const T* from = static_cast<const T*>(c.x.q) + (b.token0 + (long long)tok) * c.x.q_token + head * c.x.q_head;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        q[t][ks][u] = (there ? *reinterpret_cast<const uint32_t*>(from + ks * 16 + quad * 2) : 0u) ^ signs;
                        q[t][ks][u + 2] = (there ? *reinterpret_cast<const uint32_t*>(from + ks * 16 + quad * 2 + 8) : 0u) ^ signs;
                    }
                    m[t][u] = -INFINITY;
                    l[t][u] = sums[(t * 2 + u) * 32] = 0.f;
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) o[t][j][2 * u] = o[t][j][2 * u + 1] = 0.f;
                }
            fresh = false;
        }
        cp_async_wait<kStages<D> - 1>();
        __syncwarp();
        const uint32_t k_tile = ring_at + stage * kStageBytes<D>, v_tile = k_tile + kNarrowKeys * kPitch16<D>;
        const int key0 = now.key0 + now.tile * kNarrowKeys;
        const bool zone = key0 + kNarrowKeys > least;

        float s[kTiles][2][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][0][e] = s[t][1][e] = 0.f;
        const uint32_t k_row = k_tile + ((lane & 7) + ((lane >> 4) << 3)) * kPitch16<D> + ((lane >> 3) & 1) * 16;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            uint32_t b[4];
            ldmatrix_x4(b, k_row + ks * 32);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                mma_16816(s[t][0], q[t][ks], b[0], b[1], T());
                mma_16816(s[t][1], q[t][ks], b[2], b[3], T());
            }
        }
        uint32_t p[kTiles][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            if (zone) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key0 + u * 8 + quad * 2 + (e & 1) >= lim[t][e >> 1]) s[t][u][e] = -INFINITY;
            }
            float top[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                top[u] = fmaxf(fmaxf(s[t][0][2 * u], s[t][0][2 * u + 1]), fmaxf(s[t][1][2 * u], s[t][1][2 * u + 1])) * scale;
            // m is the base of the weights so far. A maximum that would pass it by more than sums and weights hold, anywhere: all rows move to theirs
            if (__any_sync(0xffffffffu, top[0] > m[t][0] + Pair<T>::kSlack || top[1] > m[t][1] + Pair<T>::kSlack)) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 1));
                    top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 2));
                    const float higher = fmaxf(m[t][u], top[u] - Pair<T>::kLift), alpha = m[t][u] == higher ? 1.f : ex2(m[t][u] - higher);
                    m[t][u] = higher;
                    l[t][u] *= alpha;
                    sums[(t * 2 + u) * 32] *= alpha;
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) { o[t][j][2 * u] *= alpha; o[t][j][2 * u + 1] *= alpha; }
                }
            }
            const float base[2] = {m[t][0] == -INFINITY ? 0.f : m[t][0], m[t][1] == -INFINITY ? 0.f : m[t][1]};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][u][e] = ex2(fmaf(s[t][u][e], scale, -base[e >> 1]));
            // A lane's sum of weights of N keys one by one is off by N / 4 steps of 2^-24 where they are alike and behind a heavy one (2.4e-4 for 16384
            // keys); by four, steps and groups of 32 steps it is by 32 and N / 512 of them.
#pragma unroll
            for (int u = 0; u < 2; ++u) l[t][u] += (s[t][0][2 * u] + s[t][0][2 * u + 1]) + (s[t][1][2 * u] + s[t][1][2 * u + 1]);
            p[t][0] = Pair<T>::pack(s[t][0][0], s[t][0][1]);
            p[t][1] = Pair<T>::pack(s[t][0][2], s[t][0][3]);
            p[t][2] = Pair<T>::pack(s[t][1][0], s[t][1][1]);
            p[t][3] = Pair<T>::pack(s[t][1][2], s[t][1][3]);
        }
        // Where some rows do not see all 16 keys, a value that is not finite must not reach them as 0 times it: such keys (there are none,
        // as a rule) are added one by one.
        const uint32_t v_row = v_tile + (lane & 15) * kPitch16<D> + (lane >> 4) * 16;
        bool odd = false;
        if (zone) {
#pragma unroll
            for (int j = 0; j < D / 8; j += 2) {
                uint32_t b[4];
                ldmatrix_x4_trans(b, v_row + j * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= Pair<T>::not_finite(b[e]);
            }
            odd = __any_sync(0xffffffffu, odd);
        }
        if (odd) {
            for (int key = 0; key < kNarrowKeys; ++key) {
                const int from = (lane & 28) | ((key & 7) >> 1);
                const T* row = reinterpret_cast<const T*>(ring + (v_tile - ring_at) + key * kPitch16<D>) + quad * 2;
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float a = key & 8 ? (key & 1 ? s[t][1][2 * u + 1] : s[t][1][2 * u]) : (key & 1 ? s[t][0][2 * u + 1] : s[t][0][2 * u]);
                        const float w = Pair<T>::rounded(__shfl_sync(0xffffffffu, a, from));
                        if (key0 + key >= lim[t][u]) continue;
#pragma unroll
                        for (int j = 0; j < D / 8; ++j) {
                            o[t][j][2 * u] += w * to_float(row[j * 8]);
                            o[t][j][2 * u + 1] += w * to_float(row[j * 8 + 1]);
                        }
                    }
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < D / 8; j += 2) {
                uint32_t b[4];
                ldmatrix_x4_trans(b, v_row + j * 16);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    mma_16816(o[t][j], p[t], b[0], b[1], T());
                    mma_16816(o[t][j + 1], p[t], b[2], b[3], T());
                }
            }
        }
        __syncwarp();                            // the stage has been read
        if (i + kStages<D> < n) {
            fetch(i + kStages<D>, found);
            if (i + kStages<D> + 1 < n) {
                if (load.next(list, c.cache.heads, team)) tables();
                found = look_up();
            }
        } else {
            cp_async_commit();                   // (one a step, so that the wait counts)
        }
        if (++stage == kStages<D>) stage = 0;

        const bool ends = now.tile + 1 == now.tiles;
        if ((i & 31) == 31) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) { sums[(t * 2 + u) * 32] += l[t][u]; l[t][u] = 0.f; }
        }
        if (ends || i + 1 == n) {
            const Block b = list.block[now.b];
            const long long unit = b.first_step + (long long)(now.h / team) * now.tiles;       // its first step
            const bool direct = whole && ends && now.b >= own && c.plan.share[b.request].prefix < 0;
            const long long at = direct ? 0 : piece_row<false>(c, 0, b, now.h, worker, quotient_of(unit, each));
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float sum = l[t][u] + sums[(t * 2 + u) * 32];
                    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                    const int in = t * 16 + row8 + 8 * u;
                    if (in >= b.rows) continue;
                    if (direct) {
                        const int row = b.row0 + in, tok = c.x.by_G.quotient(row), head = now.h * G + row - tok * G;
                        const float f = sum > 0.f ? 1.f / sum : sum;
                        T* to = static_cast<T*>(c.x.out) + (b.token0 + (long long)tok) * c.x.out_token + head * c.x.out_head;
#pragma unroll
                        for (int j = 0; j < D / 8; ++j)
                            *reinterpret_cast<uint32_t*>(to + j * 8 + quad * 2) = Pair<T>::pack(o[t][j][2 * u] * f, o[t][j][2 * u + 1] * f);
                        if (quad == 0) c.x.lse[(b.token0 + (long long)tok) * c.x.lse_token + head] = (m[t][u] + log2f(sum)) * 0.6931471805599453f;
                    } else {
#pragma unroll
                        for (int j = 0; j < D / 8; ++j)
                            *reinterpret_cast<float2*>(piece_values(c, at, D, b.rows, in, j * 8 + quad * 2)) = make_float2(o[t][j][2 * u], o[t][j][2 * u + 1]);
                        if (quad == 0) c.pieces.ml[at + in] = make_float2(m[t][u], sum);
                    }
                }
            fresh = whole = true;
        }
        if (i + 1 < n) now.next(list, c.cache.heads, team);
    }
}

// ---- pieces -------------------------------------------------------------------------------------
// The pieces of one row: of workers first .. first + count - 1, at row `main` of the pieces and, from the second on, at `others` + worker * cap; `rows`
// of the block, the row's place `in` among them.
struct Cut {
    long long main, others;
    int first, count, cap, rows, in;
    __device__ __forceinline__ long long piece(int i) const { return i ? others + (long long)(first + i) * cap : main; }
};
template <bool kWide> __device__ __forceinline__ Cut cut_of(const Call& c, const PlanHead& head, const Block& k, int h, int in) {
    const int tiles = (k.keys + Sizes<kWide>::keys - 1) / Sizes<kWide>::keys;
    Cut u;
    const int team = kWide ? 1 : c.plan.team;
    u.rows = k.rows; u.in = in; u.cap = (kWide ? c.pieces.wide_cap : c.pieces.narrow_cap) * team;
    u.others = place_row<kWide>(c, h, 0);
    u.first = u.count = 0;
    if (tiles) {
        const long long each = steps_each<kWide>(head.steps, list_of<kWide>(c).workers), s0 = k.first_step + (long long)(h / team) * tiles;
        u.first = quotient_of(s0, each);
        u.count = quotient_of(s0 + tiles - 1, each) - u.first + 1;
    }
    u.main = first_row<kWide>(c, head.rows_before, k, h, u.first);
    return u;
}

// Eight rows of a unit and a kv head, by four warps, or eight where there are not too many such: a lane has a row and every fourth of its groups of four
// values; a warp every fourth (eighth) of the row's pieces, those among its request's own tokens and those among its group's shared ones, by the maximum
// so far (one pass: maxima come with the values). One request of 8000 tokens, 8 heads, in pieces of 64 keys: 15 us with 32 rows a head, 10 with 4; with
// half a CTA for all rows of a unit, and two passes, it was 71 and 19. Several pieces of a warp at once cost registers, and so CTAs an SM.
// Bound by the latency of what leads to a piece (units, blocks, pieces): 5 us where there are few, 25 for the 147 units of 256 rows that 148 CTAs cut.
constexpr int kJoinRows = 8, kJoinWarps = 8;

template <int D> struct Joined {
    float4 value[kJoinWarps][D / 4][kJoinRows];
    float2 ml[kJoinWarps][kJoinRows];
};

// By W warps; with four of them, `half` says which of the CTA's. A barrier's number belongs to one number of threads: halves of a CTA may be in different
// lists, one with W == 4 and the next with W == 8.
template <typename T, int D, bool kWide, int W>
__device__ __forceinline__ void join_rows(const Call& c, Joined<D>& s, int half, const PlanHead& narrow, const PlanHead& wide, const Block& k, const Share& share,
                                          Cut mine, int h, int first_row) {
    const int lane = threadIdx.x & 31, place = threadIdx.x >> 5, warp = place % W, place0 = place - warp, G = c.x.G;
    const int bar = W == kJoinWarps ? 3 : 1 + half;
    const int r = lane % kJoinRows, quarter = lane / kJoinRows, in = first_row + r;
    const bool there = in < k.rows;
    mine.in = in;
    Cut theirs = mine;
    theirs.count = 0;
    if (share.prefix >= 0 && there) {
        const int row = share.row0 + k.row0 + in;
        theirs = share.wide ? cut_of<true>(c, wide, c.plan.wide.block[share.prefix + row / kWideRows], h, row % kWideRows)
                            : cut_of<false>(c, narrow, c.plan.narrow.block[share.prefix], h, row);
    }
    const int all = there ? mine.count + theirs.count : 0;
    float top = -INFINITY, sum = 0.f;
    float4 acc[D / 16];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int i = warp; i < all; i += W) {
        const Cut& u = i < mine.count ? mine : theirs;
        const long long at = u.piece(i < mine.count ? i : i - mine.count);
        const float2 ml = c.pieces.ml[at + u.in];
        const float* from = piece_values(c, at, D, u.rows, u.in, 4 * quarter);
        const long long step = 16 * u.rows;
        float4 x[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) x[j] = *reinterpret_cast<const float4*>(from + j * step);
        const float higher = fmaxf(top, ml.x), base = higher == -INFINITY ? 0.f : higher;
        const float old = top == higher ? 1.f : ex2(top - base), w = ex2(ml.x - base);
        top = higher;
        sum = sum * old + w * ml.y;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            acc[j].x = acc[j].x * old + w * x[j].x; acc[j].y = acc[j].y * old + w * x[j].y;
            acc[j].z = acc[j].z * old + w * x[j].z; acc[j].w = acc[j].w * old + w * x[j].w;
        }
    }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) s.value[place][4 * j + quarter][r] = acc[j];
    if (quarter == 0) s.ml[place][r] = make_float2(top, sum);
    ptx::bar_sync(bar, 32 * W);
    float all_top = -INFINITY, w[W];
    float all_sum = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) all_top = fmaxf(all_top, s.ml[place0 + i][r].x);
    const float all_base = all_top == -INFINITY ? 0.f : all_top;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float2 ml = s.ml[place0 + i][r];
        w[i] = ml.x == -INFINITY ? 0.f : ex2(ml.x - all_base);
        all_sum += w[i] * ml.y;
    }
    const float f = all_sum > 0.f ? 1.f / all_sum : all_sum;                         // no key: 0, and lse -inf
    const int row = k.row0 + in, tok = c.x.by_G.quotient(row), qh = h * G + row - tok * G;
    T* to = static_cast<T*>(c.x.out) + (k.token0 + (long long)tok) * c.x.out_token + qh * c.x.out_head;
    for (int j = warp * 4 + quarter; there && j < D / 4; j += 4 * W) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float4 x = s.value[place0 + i][j][r];
            v.x += w[i] * x.x; v.y += w[i] * x.y; v.z += w[i] * x.z; v.w += w[i] * x.w;
        }
        *reinterpret_cast<uint2*>(to + 4 * j) = make_uint2(Pair<T>::pack(v.x * f, v.y * f), Pair<T>::pack(v.z * f, v.w * f));
    }
    if (there && warp == 0 && quarter == 0)
        c.x.lse[(k.token0 + (long long)tok) * c.x.lse_token + qh] = (all_base + log2f(all_sum)) * 0.6931471805599453f;
    ptx::bar_sync(bar, 32 * W);
}

// The rows of a list: all of the requests' own, or, where nothing else is to be joined, those of units that are cut: all units are looked at, or
// those that a worker's first step cuts, whatever is less. With W == 8 a CTA takes eight rows of a unit, else half a CTA a narrow unit or an eighth of a wide one.
template <typename T, int D, bool kWide, int W>
__device__ __forceinline__ void join_parts(const Call& c, Joined<D>& s, int half, const PlanHead& narrow, const PlanHead& wide, long long items, bool by_unit) {
    const List& list = list_of<kWide>(c);
    const PlanHead& head = kWide ? wide : narrow;
    constexpr int kParts = W == kJoinWarps ? Sizes<kWide>::rows / kJoinRows : kWide ? 8 : 1, kRows = Sizes<kWide>::rows / kParts;
    const int H = c.cache.heads, team = kWide ? 1 : c.plan.team;
    const long long each = steps_each<kWide>(head.steps, list.workers);
    for (long long i = W == kJoinWarps ? blockIdx.x : blockIdx.x * 2 + half; i < items * kParts; i += gridDim.x * (kJoinWarps / W)) {
        const int item = quotient_of(i, kParts), row0 = (int)(i - (long long)item * kParts) * kRows;
        int b, h = 0;
        if (by_unit) {
            b = item / H;
            h = item - b * H;
            b += head.own;
        } else {
            b = find_last(list.steps, head.blocks, each * (item / team + 1));
        }
        const Block k = list.block[b];
        if (row0 >= k.rows) continue;
        if (!by_unit) {
            const long long at = each * (item / team + 1);
            const int tiles = (k.keys + Sizes<kWide>::keys - 1) / Sizes<kWide>::keys;
            h = (int)(at - k.first_step) / tiles;
            const long long unit = k.first_step + (long long)h * tiles;
            h = h * team + item % team;
            // (a unit that several workers cut is the first one's; shared tokens' units are joined with their requests' own)
            if (b < head.own || unit >= at || unit < at - each) continue;
        }
        const Share share = c.plan.share[k.request];
        const Cut mine = cut_of<kWide>(c, head, k, h, 0);
        if (mine.count == 1 && share.prefix < 0) continue;                              // written already
        for (int row = row0; row < min(row0 + kRows, k.rows); row += kJoinRows)
            join_rows<T, D, kWide, W>(c, s, half, narrow, wide, k, share, mine, h, row);
    }
}
template <typename T, int D, bool kWide>
__device__ __forceinline__ void join_list(const Call& c, Joined<D>& s, int half, const PlanHead& narrow, const PlanHead& wide) {
    const List& list = list_of<kWide>(c);
    const PlanHead& head = kWide ? wide : narrow;
    if (head.blocks == head.own) return;
    const long long cuts = (head.steps - 1) / steps_each<kWide>(head.steps, list.workers) * (kWide ? 1 : c.plan.team);
    const long long units = (long long)(head.blocks - head.own) * c.cache.heads;
    const bool by_unit = head.all_rows || units <= cuts;
    const long long items = by_unit ? units : cuts;
    if (items * (Sizes<kWide>::rows / kJoinRows) <= gridDim.x) join_parts<T, D, kWide, kJoinWarps>(c, s, 0, narrow, wide, items, by_unit);
    else join_parts<T, D, kWide, kJoinWarps / 2>(c, s, half, narrow, wide, items, by_unit);
}

template <typename T, int D>
__global__ void __launch_bounds__(256, 2) join_kernel(const Call c) {
    __shared__ Joined<D> s;
    ardiff::begin_kernel();
    const int half = threadIdx.x >> 7;
    const PlanHead narrow = *c.plan.narrow.head, wide = *c.plan.wide.head;
    join_list<T, D, false>(c, s, half, narrow, wide);
    join_list<T, D, true>(c, s, half, narrow, wide);
}

// ---- the call -----------------------------------------------------------------------------------
struct Layout {
    long long narrow_blocks, wide_blocks, first_rows, narrow_cap, wide_cap, bytes, block_at[2], steps_at[2], share_at, ml_at, o_at;
    bool begun;
};
Layout layout(long long requests, long long groups, long long tokens, long long q_heads, long long heads, long long width) {
    Layout s;
    const long long rows = tokens * (q_heads / heads), parts = groups > 0 ? 2 : 1, ends = requests + (groups < requests ? groups : requests);
    // narrow: a segment each; wide: the full blocks, and one for the end of every segment of more than 16 rows
    s.narrow_blocks = (ends < parts * rows ? ends : parts * rows) + 1;
    s.wide_blocks = parts * (rows / kWideRows + (rows / 16 < requests ? rows / 16 : requests)) + 1;
    s.narrow_cap = rows < 1 ? 1 : rows < kNarrowRows ? rows : kNarrowRows;
    s.wide_cap = rows <= 16 ? 0 : rows < kWideRows ? rows : kWideRows;
    const long long places = kMaxSms * (kWarps * s.narrow_cap + s.wide_cap);
    s.begun = groups == 0 && places < tokens * q_heads;
    s.first_rows = s.begun ? places : tokens * q_heads * parts;
    auto up = [](long long v) { return (v + 255) / 256 * 256; };
    long long at = 256;
    for (int i = 0; i < 2; ++i) {
        const long long blocks = i ? s.wide_blocks : s.narrow_blocks;
        s.block_at[i] = at; at = up(at + blocks * (long long)sizeof(Block));
        s.steps_at[i] = at; at = up(at + (blocks + 1) * 8);
    }
    s.share_at = at; at = up(at + requests * (long long)sizeof(Share));
    const long long pieces = s.first_rows + places;
    s.ml_at = at; at = up(at + pieces * 8);
    s.o_at = at; at = up(at + pieces * width * 4);
    s.bytes = at;
    return s;
}

// Whether a block may be wide: `most` and the number of tokens say what they can.
bool may_be_wide(const Call& c, int most) {
    const long long news = most > 0 && most < c.x.tokens ? most : c.x.tokens;
    return (c.groups > 0 ? c.x.tokens : news) * c.x.G > c.plan.narrow_rows;
}

template <typename T, int D, int kTiles> bool launch_narrow(const Call& c, cudaStream_t st) {
    static std::atomic<uint64_t> ready{0};
    return shared_memory(narrow_kernel<T, D, kTiles>, kNarrowShared<D>, ready) &&
           launch_early(narrow_kernel<T, D, kTiles>, c.plan.wide.workers, kThreads, 1, kNarrowShared<D>, st, c);
}
template <typename T, int D> bool launch(const Call& c, int32_t dtype, int most, int sms, cudaStream_t st) {
    const bool wide = may_be_wide(c, most);
    ardiff::set_launch_count(wide ? 4 : 3);
    const unsigned threads = c.requests <= 64 ? 64 : c.requests <= 256 ? 256 : kPlanThreads;
    const bool planned = c.requests <= kPlanKept ? launch_early(plan_kernel<true>, 1, threads, 1, 0, st, c) : launch_early(plan_kernel<false>, 1, threads, 1, 0, st, c);
    return planned && (!wide || launch_wide(c, dtype, D, st)) &&
           (c.plan.narrow_rows > 16 ? launch_narrow<T, D, 2>(c, st) : launch_narrow<T, D, 1>(c, st)) &&
           launch_early(join_kernel<T, D>, 4 * sms, 256, 1, 0, st, c);
}
template <typename T> bool launch_width(const Call& c, int32_t dtype, int width, int most, int sms, cudaStream_t st) {
    switch (width) {
        case 64: return launch<T, 64>(c, dtype, most, sms, st);
        case 80: return launch<T, 80>(c, dtype, most, sms, st);
        case 96: return launch<T, 96>(c, dtype, most, sms, st);
        default: return launch<T, 128>(c, dtype, most, sms, st);
    }
}

bool shape(int64_t requests, int64_t groups, int64_t tokens, int64_t q_heads, int64_t heads) {
    return requests >= 0 && requests <= ARDIFF_PAGES_MAX_REQUESTS && groups >= 0 && groups <= ARDIFF_PAGES_MAX_REQUESTS && tokens >= 0 && tokens < (int64_t)1 << 31 && heads >= 1 &&
           q_heads >= heads && q_heads % heads == 0 && q_heads <= ARDIFF_ROTARY_MAX_HEADS && tokens * q_heads < (int64_t)1 << 31;
}

}  // namespace

int ardiff::device_sms() {
    static std::atomic<int> known[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < 64 && known[dev].load(std::memory_order_relaxed)) return known[dev].load(std::memory_order_relaxed);
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) return 0;
    if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

extern "C" int64_t ardiff_attend_workspace(int32_t requests, int32_t groups, int64_t tokens, int32_t q_heads, int32_t heads, int32_t head_width) {
    if (!shape(requests, groups, tokens, q_heads, heads) || head_width < 1 || head_width > ARDIFF_ROTARY_MAX_WIDTH) return ARDIFF_ERR_SHAPE;
    return layout(requests, groups, tokens, q_heads, heads, head_width).bytes;
}

extern "C" int ardiff_attend_pages(const ardiff_attend_pages_call* call, void* stream) {
    if (!call) return ARDIFF_ERR_NULL;
    const ardiff_attend_pages_call& c = *call;
    if (!ardiff::in_32_bits({c.q_heads, c.dtype, c.pages, c.page, c.heads, c.head_width, c.width, c.requests, c.groups, c.most, c.causal})) return ARDIFF_ERR_SHAPE;
    const int requests = (int)c.requests, groups = (int)c.groups, q_heads = (int)c.q_heads, heads = (int)c.heads, head_width = (int)c.head_width;
    const int page = (int)c.page, width = (int)c.width, most = (int)c.most, dtype = (int)c.dtype;
    const int64_t tokens = c.tokens;
    const float scale = (float)c.scale;
    if (!shape(requests, groups, tokens, q_heads, heads) || c.pages < 0 || page < 1 || width < 0 || (int64_t)page * width > ARDIFF_CACHE_MAX_PLACES ||
        (int64_t)page * width * heads >= (int64_t)1 << 34 || most < 0 || !isfinite(scale * 1.4426950408889634f))
        return ARDIFF_ERR_SHAPE;
    if ((dtype != ARDIFF_BF16 && dtype != ARDIFF_F16) || (head_width != 64 && head_width != 80 && head_width != 96 && head_width != 128))
        return ARDIFF_ERR_UNSUPPORTED;
    if (!c.status || !c.offset || !c.workspace) return ARDIFF_ERR_NULL;
    if (requests > 0 && (!c.length || (width > 0 && !c.table) || !c.k_cache || !c.v_cache)) return ARDIFF_ERR_NULL;
    if (tokens > 0 && (!c.q || !c.out || !c.lse)) return ARDIFF_ERR_NULL;
    if (groups > 0 && (!c.group || !c.shared)) return ARDIFF_ERR_NULL;
    auto low = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if (((low(c.q) | low(c.out) | low(c.k_cache) | low(c.v_cache)) & 15u) || (low(c.workspace) & 255u) ||
        ((c.q_token | c.q_head | c.out_token | c.out_head | c.k_page | c.k_token | c.k_head | c.v_page | c.v_token | c.v_head) & 7))
        return ARDIFF_ERR_ALIGN;
    const Layout s = layout(requests, groups, tokens, q_heads, heads, head_width);
    if (c.workspace_bytes < s.bytes) return ARDIFF_ERR_SHAPE;
    if (tokens > 0 && c.q == c.out) return ARDIFF_ERR_UNSUPPORTED;         // (blocks of other workers still read them)
    const int sms = device_sms();
    if (sms < 1) return ARDIFF_ERR_CUDA;
    Call a;
    memset(&a, 0, sizeof(a));
    a.cache.k = static_cast<const char*>(c.k_cache); a.cache.v = static_cast<const char*>(c.v_cache);
    a.cache.table = c.table; a.cache.width = width; a.cache.page = page; a.cache.pages = c.pages; a.cache.heads = heads; a.cache.by_page = divide_by(page);
    if (!strides_of(c.k_page, c.k_token, c.k_head, a.cache, a.cache.k_page, a.cache.k_token, a.cache.k_head) ||
        !strides_of(c.v_page, c.v_token, c.v_head, a.cache, a.cache.v_page, a.cache.v_token, a.cache.v_head))
        return ARDIFF_ERR_SHAPE;
    a.x.q = c.q; a.x.out = c.out; a.x.lse = c.lse; a.x.q_token = c.q_token; a.x.q_head = c.q_head; a.x.out_token = c.out_token; a.x.out_head = c.out_head;
    a.x.lse_token = c.lse_token; a.x.heads = q_heads; a.x.G = q_heads / heads; a.x.tokens = tokens;
    a.x.by_G = divide_by(q_heads / heads);
    char* w = static_cast<char*>(c.workspace);
    for (int i = 0; i < 2; ++i) {
        List& l = i ? a.plan.wide : a.plan.narrow;
        l.head = reinterpret_cast<PlanHead*>(w) + i;
        l.block = reinterpret_cast<Block*>(w + s.block_at[i]);
        l.steps = reinterpret_cast<long long*>(w + s.steps_at[i]);
    }
    a.plan.wide.workers = sms < kMaxSms ? sms : kMaxSms;
    // Memory is read in lines of 128 bytes. Where rows of neighbouring heads share them, warps of a CTA go through the same keys of
    // several heads, so that what one does not want is in L2 for the next (96 requests of 3500 tokens, 16 heads of 80 values side by side, 1.7 GB:
    // 313 us, 472 without).
    a.plan.team = 1;
    if (head_width % 64 && c.k_head < c.k_token && c.k_head % 64)
        while (a.plan.team < kWarps && heads % (2 * a.plan.team) == 0) a.plan.team *= 2;
    a.plan.narrow.workers = a.plan.wide.workers * kWarps / a.plan.team;
    // (a request's rows at most, or on average where that is not known: those of more go the wide way)
    const int64_t news = most > 0 ? most : requests > 0 ? (tokens + requests - 1) / requests : 0;
    a.plan.narrow_rows = news * a.x.G <= 16 ? 16 : 32;
    a.plan.share = reinterpret_cast<Share*>(w + s.share_at);
    a.pieces.ml = reinterpret_cast<float2*>(w + s.ml_at);
    a.pieces.o = reinterpret_cast<float*>(w + s.o_at);
    a.pieces.narrow_rows = s.first_rows;
    a.pieces.wide_rows = s.first_rows + kMaxSms * kWarps * s.narrow_cap;
    a.pieces.narrow_cap = (int)s.narrow_cap; a.pieces.wide_cap = (int)s.wide_cap; a.pieces.begun = s.begun;
    a.length = c.length; a.offset = c.offset; a.group = c.group; a.shared = c.shared; a.status = c.status;
    a.scale = scale * 1.4426950408889634f;
    if (fabsf(a.scale) < 1.2e-38f) a.scale = 1.2e-38f;       // (0 times the -inf of a key that is not seen would be NaN)
    a.requests = requests; a.groups = groups; a.causal = c.causal != 0; a.most = most;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool ok = dtype == ARDIFF_F16 ? launch_width<__half>(a, dtype, head_width, most, sms, st)
                                        : launch_width<__nv_bfloat16>(a, dtype, head_width, most, sms, st);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}
