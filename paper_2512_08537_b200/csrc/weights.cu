// ardiff_attend_weights: the attention weight that every token of a cache gets from the call's queries, added to what it had:
//
//   new_score[r][p] = decay score[r][p] + sum over the request's new tokens i and query heads h of exp(scale q_ih.k_p - lse_ih)
//
// lse comes from the attention itself, so no maximum and no second pass is needed, and every key's sum stands alone. Products are
// transposed: 128 keys are the rows of the left operand, so that a sum over queries is one thread's (a lane of tensor memory), and up to 128
// query rows of a head the columns, 16 at least. A CTA takes consecutive tiles of 128 keys of a request, up to 8 together, and goes through heads
// and rows for all of them, so that queries are fetched once for 8 tiles; up to 16 rows a head and 16 heads are fetched at once, and heads
// follow one another inside a tile, as they lie in memory. Keys stream through four stages. Where there are fewer tiles than
// SMs, the heads of a tile are split among CTAs, and the last of them adds the parts in their order. No atomics on sums: equal calls give equal bits.
//
// Bound by the keys' memory for few rows (512 bytes would be keys and values; here it is 256 a head of 128 values), by exponentials (16 a clock and SM)
// from some 90 rows a kv head on. 128 requests of one query, up to 4096 tokens, 8 heads of 128: 540 MB in 112 us, 4.8 TB/s (15 tiles for the fullest of 148
// CTAs where 14.2 are the mean, 82 % of the copy rate between its start and end); 8 requests of 32 queries, up to 16384 tokens: 46 us, of which the
// exponentials take 19 and the keys 21.
//
// Warps: 0-3 and 4-7 sums, every other product each; 8 issues products; 9 copies keys (by TMA where pages allow, else by 16 bytes), 10 queries, 11 what is
// known of their rows.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/ardiff.h"
#include "attend.cuh"
#include "common.cuh"
#include "launch.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace {

using namespace ardiff;

constexpr int kPlanThreads = 1024;
constexpr int kThreads = 12 * 32;
constexpr int kKeys = 128, kRows = 128;          // of a product
constexpr int kTogether = 8;                     // tiles of keys
constexpr int kFew = 16;                         // rows of a head, and heads, that are fetched at once
constexpr int kStages = 4, kScores = 4;          // keys in shared memory, products in tensor memory
constexpr int kMaxSplit = 256;                   // CTAs, where heads are split among them

struct Weights {
    Pages cache;
    Queries x;
    const int32_t* length;
    const int32_t* offset;
    const int32_t* first;
    const float* score;
    float* new_score;
    int32_t* status;
    long long* tiles;                            // [requests + 1]: tiles of the requests before
    int* arrived;                                // [kMaxSplit]: parts of a tile that are there
    float* part;                                 // [kMaxSplit][128]
    long long ld, new_ld, limit;
    float scale, decay;                          // scale: times log2 e
    int requests, causal;
};

struct KeyBoxes {
    CUtensorMap k, q, few;                       // few: boxes of 16 rows of queries
    int tokens;                                  // of a box of keys; 0: by 16 bytes
    bool queries;                                // by boxes
};

// The first key of a request's tiles: a multiple of 128, so that boxes of tokens do not cross pages.
__device__ __forceinline__ int first_of(const Weights& c, int r) { return c.first ? max(0, c.first[r]) : 0; }

__global__ void __launch_bounds__(kPlanThreads) tiles_kernel(const Weights c) {
    __shared__ long long s_scan[32];
    ardiff::begin_kernel();
    const int tid = threadIdx.x, R = c.requests;
    bool bad = false;
    long long tiles = 0;
    for (int r0 = 0; r0 < R; r0 += kPlanThreads) {
        const int r = r0 + tid;
        int n = 0;
        if (r < R) {
            const int a = c.offset[r], b = c.offset[r + 1], len = c.length[r];
            bad |= a < 0 || b < a || b > c.x.tokens || len < 0 || len > c.limit;
            const int first = first_of(c, r);
            n = len > first ? (len - first / kKeys * kKeys + kKeys - 1) / kKeys : 0;
        }
        long long total;
        const long long at = tiles + cta_scan(n, s_scan, &total);
        if (r < R) c.tiles[r] = at;
        tiles += total;
    }
    bad = __syncthreads_or(bad);
    if (tid < kMaxSplit) c.arrived[tid] = 0;
    if (tid == 0) {
        *c.status = bad ? ARDIFF_ERR_SHAPE : ARDIFF_OK;
        c.tiles[R] = bad ? 0 : tiles;
    }
}

// Consecutive tiles of one request that are worked on together.
struct Segment {
    int r, tiles, key0, keys;                    // keys: the end of the request's
    int first, token0, news, rows;
    // what is gone through for every tile: `units` of queries (chunks of up to 128 rows of a head), or one of all heads (few)
    int units, heads;                            // heads: of a unit
    bool few;
};
__device__ __forceinline__ Segment segment(const Weights& c, long long at, long long end, int heads) {
    Segment s;
    s.r = find_last(c.tiles, c.requests, at);
    s.first = first_of(c, s.r);
    s.key0 = s.first / kKeys * kKeys + (int)(at - c.tiles[s.r]) * kKeys;
    s.keys = c.length[s.r];
    s.tiles = (int)min(min(end, c.tiles[s.r + 1]) - at, (long long)kTogether);
    s.token0 = c.offset[s.r];
    s.news = c.offset[s.r + 1] - s.token0;
    s.rows = s.news * c.x.G;
    s.few = s.rows <= kFew && heads <= kFew;
    s.heads = s.few ? heads : 1;
    s.units = s.rows == 0 ? 0 : s.few ? 1 : (s.rows + kRows - 1) / kRows * heads;
    return s;
}

template <int D> constexpr int kSub = (D + 63) / 64;                       // blocks of 64 values of a row
template <int D> constexpr int kTile = kSub<D> * 128 * 128;                // bytes of 128 rows
template <int D> constexpr int kShared = 1024 + (kStages + 2) * kTile<D> + 2 * kTogether * kKeys * 4 + kTogether * kKeys * 8 + 2 * kRows * 8;

enum Bar { kKFull, kKEmpty = kKFull + kStages, kSFull = kKEmpty + kStages, kSEmpty = kSFull + kScores, kQFull = kSEmpty + kScores, kQEmpty = kQFull + 2,
           kColFull = kQEmpty + 2, kColEmpty = kColFull + 2, kDrained = kColEmpty + 2, kBars };

// The sum of a key's weights from `cols` scores in tensor memory; kSome: only rows that see the key.
template <bool kSome> __device__ __forceinline__ float sum_of(uint32_t scores, const float* column, const int* seen, int cols, float scale, int key) {
    const Two scale2 = two(scale, scale);
    Two sum[2] = {two(0.f, 0.f), two(0.f, 0.f)};
    const int groups = (cols + 15) / 16;
    uint32_t x[2][16];
    ptx::tmem_ld_32x32b_x16(scores, x[0]);
    for (int g = 0; g < groups; g += 2) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (g + e >= groups) break;
            ptx::tmem_ld_wait_for(x[e]);
            if (g + e + 1 < groups) ptx::tmem_ld_32x32b_x16(scores + (g + e + 1) * 16, x[e ^ 1]);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 c = *reinterpret_cast<const float4*>(column + (g + e) * 16 + j);
                const float2 a = apart(fma2(two(__uint_as_float(x[e][j]), __uint_as_float(x[e][j + 1])), scale2, two(c.x, c.y)));
                const float2 b = apart(fma2(two(__uint_as_float(x[e][j + 2]), __uint_as_float(x[e][j + 3])), scale2, two(c.z, c.w)));
                float2 p = make_float2(ex2(a.x), ex2(a.y)), q = make_float2(ex2(b.x), ex2(b.y));
                if (kSome) {
                    const int4 k = *reinterpret_cast<const int4*>(seen + (g + e) * 16 + j);
                    p.x = key < k.x ? p.x : 0.f; p.y = key < k.y ? p.y : 0.f; q.x = key < k.z ? q.x : 0.f; q.y = key < k.w ? q.y : 0.f;
                }
                sum[0] = sum[0] + two(p.x, p.y);
                sum[1] = sum[1] + two(q.x, q.y);
            }
        }
    }
    const float2 s = apart(sum[0] + sum[1]);
    return s.x + s.y;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) weights_kernel(const Weights c, const __grid_constant__ KeyBoxes boxes) {
    extern __shared__ char raw[];
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kQ = kStages * kTile<D>;
    float* sums = reinterpret_cast<float*>(smem + kQ + 2 * kTile<D>);                 // [2][tiles][128]: every other product's
    long long* place = reinterpret_cast<long long*>(sums + 2 * kTogether * kKeys);   // [tiles][128]: offsets of keys (odd: none), or of boxes
    // of the rows of both buffers of queries (few: 16 a head, in both): -lse log2 e, keys that the row sees
    float* column = reinterpret_cast<float*>(place + kTogether * kKeys);
    int* seen = reinterpret_cast<int*>(column + 2 * kRows);
    __shared__ __align__(8) uint64_t s_bar[kBars];
    __shared__ uint32_t s_tmem;
    __shared__ int s_stop, s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bars = ptx::smem_u32(s_bar), smem_at = ptx::smem_u32(smem);
    ardiff::begin_kernel();
    const int H = c.cache.heads, G = c.x.G, workers = gridDim.x;
    const long long tiles = c.tiles[c.requests];
    if (tiles == 0) return;
    // few tiles: `split` CTAs a tile, each some of its heads
    const int split = tiles * 2 > workers ? 1 : min(H, (int)(workers / tiles));
    const long long each = (tiles + workers - 1) / workers;
    const long long begin = split > 1 ? blockIdx.x / split : each * blockIdx.x, end = split > 1 ? begin + 1 : min(tiles, begin + each);
    if (begin >= tiles) return;
    const int part = split > 1 ? blockIdx.x % split : 0, h0 = part * H / split, h1 = (part + 1) * H / split;
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            int count = 1;
            if (i < kKEmpty) count = boxes.tokens ? 1 : 32;
            else if (i >= kSEmpty && i < kQFull) count = 128;
            else if (i >= kQFull && i < kQEmpty) count = boxes.queries ? 1 : 32;
            else if (i >= kColFull && i < kColEmpty) count = 32;
            else if (i >= kColEmpty && i < kDrained) count = 256;
            ptx::mbar_init(bars + i * 8, count);
        }
        s_stop = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 8) {
        ptx::tmem_alloc(ptx::smem_u32(&s_tmem), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = s_tmem;
    const Waits wait{bars, &s_stop, c.status};
    auto all = [](bool ok) { return __all_sync(0xffffffffu, ok) != 0; };     // a warp goes on or leaves as one
    bool good = true;

    if (warp == 9) {
        // ---- keys
        constexpr int kLanes = D / 8 <= 8 ? 8 : 16, kAtOnce = 32 / kLanes, kPeriod = 8 / kAtOnce;    // lanes a row, rows at once, before they repeat
        const int ch = lane % kLanes, row0 = lane / kLanes, tokens = boxes.tokens;
        const bool mine = ch < D / 8;
        uint32_t to[kPeriod];
#pragma unroll
        for (int u = 0; u < kPeriod; ++u) to[u] = smem_at + swizzled(row0 + u * kAtOnce, ch);
        uint32_t i = 0;
        for (long long at = begin; at < end && good;) {
            const Segment s = segment(c, at, end, h1 - h0);
            const int32_t* table = c.cache.table + (long long)s.r * c.cache.width;
            const int step = tokens ? tokens : 1;
            __syncwarp();
            for (int j = lane; j < s.tiles * kKeys / step; j += 32) {
                const int key = s.key0 + j * step;
                long long p = 1;
                if (key < s.keys) {
                    const unsigned pg = c.cache.by_page.quotient(key), in = key - pg * c.cache.page;
                    const int id = table[pg];
                    if (id >= 0 && id < c.cache.pages) p = tokens ? (long long)id << 32 | in << 1 : offset_of(c.cache.k_page, c.cache.k_token, 0, id, in, 0);
                    else if (key + step > s.first) *c.status = ARDIFF_ERR_SHAPE;     // (tokens in front of the first one may lie anywhere)
                }
                place[j] = p;
            }
            __syncwarp();
            for (int v = 0; v < s.units && good; ++v)
                for (int t = 0; t < s.tiles && good; ++t)
                    for (int w = 0; w < s.heads; ++w, ++i) {
                        const int stage = i % kStages, h = h0 + (s.few ? w : v % (h1 - h0));
                        good = all(wait(kKEmpty + stage, ((i / kStages) & 1) ^ 1));
                        if (!good) break;
                        const uint32_t bar = bars + (kKFull + stage) * 8;
                        if (tokens) {
                            const int of_tile = kKeys / tokens;
                            const long long p = lane < of_tile ? place[t * of_tile + lane] : 1;
                            const uint32_t there = __ballot_sync(0xffffffffu, !(p & 1));
                            if (lane == 0) ptx::mbar_arrive_expect_tx(bar, __popc(there) * tokens * 128 * kSub<D>);
                            __syncwarp();
                            if (!(p & 1)) {
#pragma unroll
                                for (int b = 0; b < kSub<D>; ++b)
                                    ptx::tma_load_4d(smem_at + stage * kTile<D> + b * 16384 + lane * tokens * 128, &boxes.k, bar, b * 64, (int)((uint32_t)p >> 1), h,
                                                     (int)(p >> 32));
                            }
                        } else {
                            const long long* p = place + t * kKeys + row0;
                            const char* from = c.cache.k + (long long)h * c.cache.k_head * 16 + ch * 16;
#pragma unroll 1
                            for (int j = 0; j < kKeys / kAtOnce; j += 16) {
                                long long o[16];
#pragma unroll
                                for (int u = 0; u < 16; ++u) o[u] = p[(j + u) * kAtOnce];
                                const uint32_t base = stage * kTile<D> + (j / kPeriod) * 1024;
#pragma unroll
                                for (int u = 0; u < 16; ++u)
                                    if (mine) cp_async16(to[u % kPeriod] + base + (u / kPeriod) * 1024, from + (o[u] & 1 ? 0 : o[u]), o[u] & 1 ? 0 : 16);
                            }
                            cp_async_arrive(bar);
                        }
                    }
            at += s.tiles;
        }
        cp_async_commit();
        cp_async_wait<0>();
        if (!good) wait_for_copies(bars, kKFull, i, kStages);
    } else if (warp == 10) {
        // ---- queries
        constexpr int kLanes = D / 8 <= 8 ? 8 : 16;
        const int ch = lane % kLanes;
        const bool mine = ch < D / 8;
        uint32_t u = 0;
        bool few = false;                        // the unit before
        for (long long at = begin; at < end && good;) {
            const Segment s = segment(c, at, end, h1 - h0);
            for (int v = 0; v < s.units; ++v, ++u) {
                const int buf = u & 1;
                // (few: both buffers, when all units before are done with)
                good = all(wait(kQEmpty + buf, ((u >> 1) & 1) ^ 1) && (!(s.few || few) || u == 0 || wait(kQEmpty + (buf ^ 1), ((u - 1) >> 1) & 1)));
                if (!good) break;
                few = s.few;
                if (boxes.queries) {
                    const uint32_t bar = bars + (kQFull + buf) * 8;
                    if (lane == 0) ptx::mbar_arrive_expect_tx(bar, s.few ? s.heads * kSub<D> * kFew * 128 : kTile<D>);
                    __syncwarp();
                    // (rows of other requests behind this one's are no rows of its columns)
                    for (int j = lane; j < s.heads * kSub<D>; j += 32) {
                        const int w = j / kSub<D>, x = j - w * kSub<D>, h = h0 + (s.few ? w : v % (h1 - h0));
                        if (s.few) ptx::tma_load_3d(smem_at + kQ + j * kFew * 128, &boxes.few, bar, x * 64, h * G, s.token0);
                        else ptx::tma_load_3d(smem_at + kQ + buf * kTile<D> + x * 16384, &boxes.q, bar, x * 64, h * G, s.token0 + v / (h1 - h0) * (kRows / G));
                    }
                    continue;
                }
                for (int w = 0; w < s.heads; ++w) {
                    const int h = h0 + (s.few ? w : v % (h1 - h0)), row0 = s.few ? 0 : v / (h1 - h0) * kRows, rows = min(kRows, s.rows - row0);
                    const uint32_t to = smem_at + kQ + (s.few ? w * kSub<D> * 2048 : buf * kTile<D>);
                    const T* base = static_cast<const T*>(c.x.q) + (long long)s.token0 * c.x.q_token + (long long)h * G * c.x.q_head + ch * 8;
#pragma unroll 8
                    for (int in = lane / kLanes; in < (rows + 15) / 16 * 16; in += 32 / kLanes) {
                        const unsigned row = row0 + in, tok = c.x.by_G.quotient(row);
                        const T* from = base + (in < rows ? tok * c.x.q_token + (row - tok * G) * c.x.q_head : 0);
                        const uint32_t place_in = s.few ? (ch >> 3) * 2048 + in * 128 + (((ch & 7) ^ (in & 7)) << 4) : swizzled(in, ch);
                        if (mine) cp_async16(to + place_in, from, in < rows ? 16 : 0);
                    }
                }
                cp_async_arrive(bars + (kQFull + buf) * 8);
            }
            at += s.tiles;
        }
        cp_async_commit();
        cp_async_wait<0>();
        if (!good) wait_for_copies(bars, kQFull, u, 2);
    } else if (warp == 11) {
        // ---- what is known of their rows
        uint32_t u = 0;
        bool few = false;
        for (long long at = begin; at < end && good;) {
            const Segment s = segment(c, at, end, h1 - h0);
            const int limit = c.causal ? s.keys - s.news + 1 : s.keys;
            for (int v = 0; v < s.units; ++v, ++u) {
                const int buf = u & 1;
                good = all(wait(kColEmpty + buf, ((u >> 1) & 1) ^ 1) && (!(s.few || few) || u == 0 || wait(kColEmpty + (buf ^ 1), ((u - 1) >> 1) & 1)));
                if (!good) break;
                few = s.few;
                for (int j = lane; j < (s.few ? s.heads * kFew : kRows); j += 32) {
                    const int in = s.few ? j % kFew : j, h = h0 + (s.few ? j / kFew : v % (h1 - h0)), row = in + (s.few ? 0 : v / (h1 - h0) * kRows);
                    float x = -INFINITY;                                               // no such row
                    int y = 0;
                    if (row < s.rows) {
                        const unsigned tok = c.x.by_G.quotient(row);
                        const float lse = c.x.lse[(s.token0 + (long long)tok) * c.x.lse_token + h * G + row - tok * G];
                        x = lse == -INFINITY ? -INFINITY : lse * -1.4426950408889634f;            // a row without keys
                        y = limit + (c.causal ? (int)tok : 0);
                    }
                    column[(s.few ? 0 : buf * kRows) + j] = x;
                    seen[(s.few ? 0 : buf * kRows) + j] = y;
                }
                ptx::mbar_arrive(bars + (kColFull + buf) * 8);
            }
            at += s.tiles;
        }
    } else if (warp == 8) {
        // ---- products
        const uint64_t q_desc = ptx::smem_desc_sw128(smem_at + kQ), k_desc = ptx::smem_desc_sw128(smem_at);
        uint32_t i = 0, u = 0;
        for (long long at = begin; at < end && good;) {
            const Segment s = segment(c, at, end, h1 - h0);
            for (int v = 0; v < s.units && good; ++v, ++u) {
                const int rows = s.few ? kFew : min(kRows, s.rows - v / (h1 - h0) * kRows);
                const uint32_t idesc = ptx::idesc_16(Pair<T>::kBf16, kKeys, (rows + 15) / 16 * 16, false, false);
                const uint32_t next = s.few ? 128 : 1024;                              // blocks of 64 values of the queries, in 16 bytes
                good = all(wait(kQFull + (u & 1), (u >> 1) & 1));
                for (int t = 0; t < s.tiles && good; ++t)
                    for (int w = 0; w < s.heads; ++w, ++i) {
                        const int stage = i % kStages, to = i % kScores;
                        good = all(wait(kKFull + stage, (i / kStages) & 1) && wait(kSEmpty + to, ((i / kScores) & 1) ^ 1));
                        if (!good) break;
                        ptx::fence_proxy_async_smem();
                        ptx::tc_fence_after();
                        const uint64_t a = k_desc + stage * (kTile<D> / 16), b = q_desc + (s.few ? w * kSub<D> * 128 : (u & 1) * (kTile<D> / 16));
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                ptx::mma_f16_ss(tmem + to * 128, a + (ks >> 2) * 1024 + (ks & 3) * 2, b + (ks >> 2) * next + (ks & 3) * 2, idesc, ks > 0);
                            ptx::mma_commit(bars + (kSFull + to) * 8);
                            ptx::mma_commit(bars + (kKEmpty + stage) * 8);
                            if (t + 1 == s.tiles && w + 1 == s.heads) ptx::mma_commit(bars + (kQEmpty + (u & 1)) * 8);
                        }
                        __syncwarp();
                    }
            }
            at += s.tiles;
        }
        if (!good) {
            // products in flight end before tensor memory is given back
            if (ptx::elect_one()) ptx::mma_commit(bars + kDrained * 8);
            __syncwarp();
            for (int j = 0; j < 1 << 20 && !ptx::mbar_try_wait(bars + kDrained * 8, 0); ++j) {}
        }
        __syncwarp();
    } else {
        // ---- sums: a thread a key
        const int side = warp >> 2, key = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
        uint32_t i = 0, u = 0;
        for (long long at = begin; at < end;) {
            const Segment s = segment(c, at, end, h1 - h0);
            float* mine = sums + side * kTogether * kKeys + key;
            for (int t = 0; t < s.tiles; ++t) mine[t * kKeys] = 0.f;
            const int least = c.causal ? s.keys - s.news + 1 : s.keys;              // keys below are seen by all rows
            for (int v = 0; v < s.units && good; ++v, ++u) {
                const int cols = s.few ? s.rows : min(kRows, s.rows - v / (h1 - h0) * kRows);
                good = all(wait(kColFull + (u & 1), (u >> 1) & 1));
                for (int t = 0; t < s.tiles && good; ++t)
                    for (int w = 0; w < s.heads; ++w, ++i) {
                        if ((int)(i & 1) != side) continue;
                        const int from = i % kScores, at_col = s.few ? w * kFew : (u & 1) * kRows;
                        good = all(wait(kSFull + from, (i / kScores) & 1));
                        if (!good) break;
                        ptx::tc_fence_after();
                        const uint32_t scores = lanes + from * 128;
                        // (a column that is no row of the request may hold anything)
                        mine[t * kKeys] += s.key0 + (t + 1) * kKeys > least || (cols & 15)
                                               ? sum_of<true>(scores, column + at_col, seen + at_col, cols, c.scale, s.key0 + t * kKeys + key)
                                               : sum_of<false>(scores, column + at_col, seen + at_col, cols, c.scale, 0);
                        ptx::tc_fence_before();
                        ptx::mbar_arrive(bars + (kSEmpty + from) * 8);
                    }
                ptx::mbar_arrive(bars + (kColEmpty + (u & 1)) * 8);
            }
            ptx::bar_sync(2, 256);               // (all eight warps come here for every segment, whether they gave up or not)
            if (split == 1) {
                for (int t = side; t < s.tiles; t += 2) {
                    const int p = s.key0 + t * kKeys + key;
                    if (p < s.first || p >= s.keys) continue;
                    const float got = sums[t * kKeys + key] + sums[(kTogether + t) * kKeys + key];
                    c.new_score[s.r * c.new_ld + p] = (p < s.keys - s.news ? c.decay * c.score[s.r * c.ld + p] : 0.f) + got;
                }
            } else {
                float* parts = c.part + (long long)begin * split * kKeys;
                if (side == 0) {
                    parts[part * kKeys + key] = sums[key] + sums[kTogether * kKeys + key];
                    __threadfence();
                }
                ptx::bar_sync(2, 256);
                if (tid == 0) {
                    s_last = atomicAdd(&c.arrived[begin], 1) == split - 1;
                    __threadfence();
                }
                ptx::bar_sync(2, 256);
                const int p = s.key0 + key;
                if (s_last && side == 0 && p >= s.first && p < s.keys) {
                    float got = 0.f;
                    for (int j = 0; j < split; ++j) got += __ldcg(parts + j * kKeys + key);
                    c.new_score[s.r * c.new_ld + p] = (p < s.keys - s.news ? c.decay * c.score[s.r * c.ld + p] : 0.f) + got;
                }
            }
            ptx::bar_sync(2, 256);               // the sums have been read
            at += s.tiles;
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 8) ptx::tmem_dealloc(tmem, 512);
}

template <typename T, int D> bool launch(const Weights& c, const KeyBoxes& boxes, int sms, cudaStream_t st) {
    static std::atomic<uint64_t> ready{0};
    return shared_memory(weights_kernel<T, D>, kShared<D>, ready) && launch_early(tiles_kernel, 1, kPlanThreads, 1, 0, st, c) &&
           launch_early(weights_kernel<T, D>, sms < kMaxSplit ? sms : kMaxSplit, kThreads, 1, kShared<D>, st, c, boxes);
}
template <typename T> bool launch_width(const Weights& c, int width, const KeyBoxes& boxes, int sms, cudaStream_t st) {
    switch (width) {
        case 64: return launch<T, 64>(c, boxes, sms, st);
        case 80: return launch<T, 80>(c, boxes, sms, st);
        case 96: return launch<T, 96>(c, boxes, sms, st);
        default: return launch<T, 128>(c, boxes, sms, st);
    }
}

// the numbers of tiles, the parts' counters, the parts
int64_t arrived_at(int64_t requests) { return (requests + 1) * 8; }
int64_t part_at(int64_t requests) { return (arrived_at(requests) + kMaxSplit * 4 + 255) / 256 * 256; }

}  // namespace

extern "C" int64_t ardiff_attend_weights_workspace(int32_t requests) {
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS) return ARDIFF_ERR_SHAPE;
    return part_at(requests) + (int64_t)kMaxSplit * kKeys * 4;
}

extern "C" int ardiff_attend_weights(const ardiff_attend_weights_call* call, void* stream) {
    if (!call) return ARDIFF_ERR_NULL;
    const ardiff_attend_weights_call& c = *call;
    if (!ardiff::in_32_bits({c.q_heads, c.dtype, c.pages, c.page, c.heads, c.head_width, c.width, c.requests, c.causal})) return ARDIFF_ERR_SHAPE;
    const int requests = (int)c.requests, q_heads = (int)c.q_heads, heads = (int)c.heads, head_width = (int)c.head_width, page = (int)c.page;
    const int width = (int)c.width, dtype = (int)c.dtype;
    const int64_t tokens = c.tokens;
    const float scale = (float)c.scale, decay = (float)c.decay;
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS || tokens < 0 || tokens >= (int64_t)1 << 31 || heads < 1 || q_heads < heads || q_heads % heads ||
        q_heads > ARDIFF_ROTARY_MAX_HEADS || tokens * q_heads >= (int64_t)1 << 31 || c.pages < 0 || page < 1 || width < 0 ||
        (int64_t)page * width > ARDIFF_CACHE_MAX_PLACES || c.ld < 0 || c.new_ld < 0 || !isfinite(scale * 1.4426950408889634f) || !isfinite(decay))
        return ARDIFF_ERR_SHAPE;
    if ((dtype != ARDIFF_BF16 && dtype != ARDIFF_F16) || (head_width != 64 && head_width != 80 && head_width != 96 && head_width != 128))
        return ARDIFF_ERR_UNSUPPORTED;
    if (!c.status || !c.offset || !c.workspace) return ARDIFF_ERR_NULL;
    if (requests > 0 && (!c.length || (width > 0 && !c.table) || !c.k_cache || !c.score || !c.new_score)) return ARDIFF_ERR_NULL;
    if (tokens > 0 && (!c.q || !c.lse)) return ARDIFF_ERR_NULL;
    auto low = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if (((low(c.q) | low(c.k_cache)) & 15u) || (low(c.workspace) & 15u) || ((c.q_token | c.q_head | c.k_page | c.k_token | c.k_head) & 7)) return ARDIFF_ERR_ALIGN;
    if (c.workspace_bytes < ardiff_attend_weights_workspace(requests)) return ARDIFF_ERR_SHAPE;
    if (c.score == c.new_score && requests > 1 && c.ld != c.new_ld) return ARDIFF_ERR_SHAPE;
    const int sms = device_sms();
    if (sms < 1) return ARDIFF_ERR_CUDA;
    Weights a;
    memset(&a, 0, sizeof(a));
    a.cache.k = static_cast<const char*>(c.k_cache);
    a.cache.table = c.table; a.cache.width = width; a.cache.page = page; a.cache.pages = c.pages; a.cache.heads = heads; a.cache.by_page = divide_by(page);
    if (!strides_of(c.k_page, c.k_token, c.k_head, a.cache, a.cache.k_page, a.cache.k_token, a.cache.k_head)) return ARDIFF_ERR_SHAPE;
    a.x.q = c.q; a.x.lse = const_cast<float*>(c.lse); a.x.q_token = c.q_token; a.x.q_head = c.q_head; a.x.lse_token = c.lse_token;
    a.x.heads = q_heads; a.x.G = q_heads / heads; a.x.tokens = tokens; a.x.by_G = divide_by(q_heads / heads);
    a.length = c.length; a.offset = c.offset; a.first = c.first; a.score = c.score; a.new_score = c.new_score; a.status = c.status;
    char* w = static_cast<char*>(c.workspace);
    a.tiles = reinterpret_cast<long long*>(w);
    a.arrived = reinterpret_cast<int*>(w + arrived_at(requests));
    a.part = reinterpret_cast<float*>(w + part_at(requests));
    a.ld = c.ld; a.new_ld = c.new_ld;
    const int64_t cap = (int64_t)page * width, rows = c.ld < c.new_ld ? c.ld : c.new_ld;
    a.limit = cap < rows ? cap : rows;
    a.scale = scale * 1.4426950408889634f; a.decay = decay;
    a.requests = requests; a.causal = c.causal != 0;
    const bool bf16 = dtype == ARDIFF_BF16;
    KeyBoxes boxes;
    memset(&boxes, 0, sizeof(boxes));
    const int box = box_tokens(page);
    if (box && describe(&boxes.k, a.cache.k, bf16, head_width, box, a.cache, a.cache.k_token, a.cache.k_head, a.cache.k_page)) boxes.tokens = box;
    boxes.queries = describe_queries(&boxes.q, a.x, bf16, head_width, kRows) && describe_queries(&boxes.few, a.x, bf16, head_width, kFew);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool ok = bf16 ? launch_width<__nv_bfloat16>(a, head_width, boxes, sms, st) : launch_width<__half>(a, head_width, boxes, sms, st);
    ardiff::set_launch_count(2);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}
