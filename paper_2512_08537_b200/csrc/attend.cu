// ardiff_attend_pages: attention of every request's new tokens over its tokens in a paged cache; tokens that a group of requests shares are
// read once for the whole group.
//
//   out = sum_p w_p v_p / sum_p w_p,   w_p = exp(scale q.k_p),   lse = ln sum_p w_p   over the keys p that the query sees.
//
// A sum over keys can be cut anywhere: a piece of it is its largest scale q.k, and sum and weighted values relative to that. So the shared tokens
// and a request's own are different blocks of work, blocks are cut into tiles of 64 keys, and the tiles of all blocks and heads are dealt out
// evenly, in one line, to as many CTAs as the GPU holds: one request of many keys keeps all SMs busy, and so do many requests of
// different lengths.
//   plan_kernel     checks the call, forms the blocks (whole numbers, one CTA)
//   narrow_kernel   up to 64 query rows a block
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

constexpr int kBlockRows = 64;
constexpr int kTileKeys = 64;
constexpr int kMaxCtas = 512;                    // CTAs that have a place for pieces
constexpr int kPlanThreads = 1024;
// Fewer shared tokens are read by every request itself: a block of its own and the pieces to join cost more than they take.
constexpr int kLeastShared = 64;

struct Call {
    Pages cache;
    Queries x;
    Plan plan;
    Pieces pieces;
    const int32_t* length;
    const int32_t* offset;
    const int32_t* group;
    const int32_t* shared;
    int32_t* status;
    float scale;                                 // times log2 e
    int requests, groups, causal;
};

// ---- the plan -----------------------------------------------------------------------------------
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const Call c) {
    __shared__ long long s_scan[32];
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, R = c.requests, G = c.x.G;
    const long long limit = (long long)c.cache.width * c.cache.page;
    bool bad = false;
    for (int r = tid; r < R; r += kPlanThreads) {
        const int a = c.offset[r], b = c.offset[r + 1], len = c.length[r];
        bad |= a < 0 || b < a || b > c.x.tokens || len < 0 || len > limit;
        c.plan.shared[r] = 0;
        c.plan.share[r] = Share{-1, 0};
    }
    for (int g = tid; g < c.groups; g += kPlanThreads) {
        const int a = c.group[g], b = c.group[g + 1];
        bad |= a < 0 || b < a || b > R || c.shared[g] < 0;
    }
    bad = __syncthreads_or(bad);
    if (tid == 0) *c.status = bad ? ARDIFF_ERR_SHAPE : ARDIFF_OK;
    if (bad) {
        if (tid == 0) { c.plan.head->steps = 0; c.plan.head->blocks = 0; c.plan.head->own = 0; }
        return;
    }
    // the tokens that all queries of a group see; nothing is gained where one request has queries
    for (int g = tid >> 5; g < c.groups; g += kPlanThreads / 32) {
        const int r0 = c.group[g], r1 = c.group[g + 1];
        int least = c.shared[g], active = 0;
        for (int r = r0 + lane; r < r1; r += 32) {
            const int n = c.offset[r + 1] - c.offset[r];
            if (n == 0) continue;
            ++active;
            least = min(least, max(0, c.causal ? c.length[r] - n + 1 : c.length[r]));
        }
        least = __reduce_min_sync(0xffffffffu, least);
        active = __reduce_add_sync(0xffffffffu, active);
        if (active < 2 || least < kLeastShared) least = 0;
        for (int r = r0 + lane; r < r1; r += 32) c.plan.shared[r] = least;
    }
    __syncthreads();

    long long blocks = 0;
    // shared tokens: blocks of the group's rows
    for (int g0 = 0; g0 < c.groups; g0 += kPlanThreads) {
        const int g = g0 + tid;
        int n = 0, r0 = 0, r1 = 0, keys = 0, token0 = 0;
        long long rows = 0;
        if (g < c.groups) {
            r0 = c.group[g]; r1 = c.group[g + 1];
            if (r1 > r0) {
                keys = c.plan.shared[r0];
                token0 = c.offset[r0];
                rows = keys > 0 ? (long long)(c.offset[r1] - token0) * G : 0;
            }
            n = (int)((rows + kBlockRows - 1) / kBlockRows);
        }
        long long total;
        const long long at = blocks + cta_scan(n, s_scan, &total);
        for (int j = 0; j < n; ++j) {
            Block b;
            b.token0 = token0; b.row0 = j * kBlockRows; b.rows = (int)min((long long)kBlockRows, rows - b.row0);
            b.request = r0; b.key0 = 0; b.keys = keys; b.limit = keys; b.step = 0;
            c.plan.block[at + j] = b;
        }
        if (n > 0) c.plan.share[r0].prefix = (int)at;
        blocks += total;
    }
    __syncthreads();
    for (int g = tid >> 5; g < c.groups; g += kPlanThreads / 32) {
        const int r0 = c.group[g], r1 = c.group[g + 1];
        if (r0 == r1) continue;
        const int prefix = c.plan.share[r0].prefix, token0 = c.offset[r0];
        __syncwarp();
        for (int r = r0 + lane; r < r1 && prefix >= 0; r += 32) c.plan.share[r] = Share{prefix, (c.offset[r] - token0) * G};
    }
    const long long own = blocks;
    for (int first = 0; first < R; first += kPlanThreads) {
        const int r = first + tid;
        int n = 0, token0 = 0, keys0 = 0, len = 0, news = 0;
        long long rows = 0;
        if (r < R) {
            token0 = c.offset[r];
            news = c.offset[r + 1] - token0;
            len = c.length[r];
            keys0 = c.plan.shared[r];
            rows = (long long)news * G;
            n = (int)((rows + kBlockRows - 1) / kBlockRows);
        }
        long long total;
        const long long at = blocks + cta_scan(n, s_scan, &total);
        for (int j = 0; j < n; ++j) {
            Block b;
            b.token0 = token0; b.row0 = j * kBlockRows; b.rows = (int)min((long long)kBlockRows, rows - b.row0);
            b.request = r; b.key0 = keys0;
            b.step = c.causal ? 1 : 0;
            b.limit = c.causal ? len - news + 1 : len;
            const int last = min(len, b.limit + b.step * ((b.row0 + b.rows - 1) / G));
            b.keys = max(0, last - keys0);
            c.plan.block[at + j] = b;
        }
        blocks += total;
    }
    __syncthreads();
    long long steps = 0, rows = 0;
    for (int first = 0; first < blocks; first += kPlanThreads) {
        const int b = first + tid;
        long long s = 0, w = 0;
        if (b < blocks) {
            s = (long long)((c.plan.block[b].keys + kTileKeys - 1) / kTileKeys) * c.cache.heads;
            w = c.plan.block[b].rows;
        }
        long long total;
        const long long at = steps + cta_scan(s, s_scan, &total);
        steps += total;
        const long long rows_at = rows + cta_scan(w, s_scan, &total);
        rows += total;
        if (b < blocks) { c.plan.steps[b] = at; c.plan.rows[b] = rows_at; }
    }
    if (tid == 0) {
        c.plan.steps[blocks] = steps;
        c.plan.rows[blocks] = rows;
        c.plan.head->steps = steps;
        c.plan.head->blocks = (int)blocks;
        c.plan.head->own = (int)own;
    }
}

// The steps of a CTA: the same number for all but the last ones.
__device__ __forceinline__ long long steps_each(long long steps, int ctas) { return max(1ll, (steps + ctas - 1) / ctas); }

// ---- up to 64 query rows ------------------------------------------------------------------------
constexpr int kThreads = 128;
constexpr int kStages = 3;

template <int D> constexpr int kTileBytes = kTileKeys * kPitch<D>;
template <int D> constexpr int kNarrowShared = kStages * 2 * kTileBytes<D> + 16 * D * 4 + kStages * kTileKeys * 16 + 4 * 16 * 8;

// Where a CTA is in the line of steps: block, head, tile of keys.
struct Cursor {
    int b, h, tile, tiles;
    Block at;
    __device__ __forceinline__ void enter(const Plan& p) {
        at = p.block[b];
        tiles = (at.keys + kTileKeys - 1) / kTileKeys;
    }
    // (only called while there is a next step)
    __device__ __forceinline__ void next(const Plan& p, int heads) {
        if (++tile < tiles) return;
        tile = 0;
        if (++h < heads) return;
        h = 0;
        do {
            ++b;
            enter(p);
        } while (tiles == 0);
    }
};

// Four warps. Those that share 16 query rows (all four where the block has up to 16 rows, two up to 32) take turns at groups of 16 keys, each
// with a running maximum, sum and weighted values of its own, joined in shared memory when the unit ends. Keys and values come by asynchronous copies,
// two tiles ahead, through offsets that are looked up in the table a step before that.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2) narrow_kernel(const Call c, int ctas) {
    extern __shared__ __align__(128) char smem[];
    char* tiles = smem;
    float* joined = reinterpret_cast<float*>(smem + kStages * 2 * kTileBytes<D>);
    longlong2* place = reinterpret_cast<longlong2*>(joined + 16 * D);                // [stages][keys]
    float2* part = reinterpret_cast<float2*>(place + kStages * kTileKeys);           // [warps][16]
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long steps = c.plan.head->steps, each = steps_each(steps, ctas);
    const long long begin = each * blockIdx.x;
    if (begin >= steps) return;
    const int n = (int)(min(steps, begin + each) - begin);
    const int blocks = c.plan.head->blocks;
    const uint32_t tiles_at = ptx::smem_u32(tiles);

    Cursor now;
    now.b = find_last(c.plan.steps, blocks, begin);
    now.enter(c.plan);
    {
        const long long in = begin - c.plan.steps[now.b];
        now.h = (int)(in / now.tiles);
        now.tile = (int)(in - (long long)now.h * now.tiles);
    }
    Cursor load = now;                           // the step whose places are looked up next

    // the offsets of key `j` of the step at `load`, -1 for none
    auto look_up = [&](int j) -> longlong2 {
        const int in = load.tile * kTileKeys + j;
        if (in >= load.at.keys) return make_longlong2(-1, -1);
        const unsigned key = load.at.key0 + in, pg = key / (unsigned)c.cache.page, row = key - pg * c.cache.page;
        const int id = c.cache.table[(long long)load.at.request * c.cache.width + pg];
        if (id < 0 || id >= c.cache.pages) {
            *c.status = ARDIFF_ERR_SHAPE;
            return make_longlong2(-1, -1);
        }
        return make_longlong2(id * c.cache.k_page + row * c.cache.k_token + load.h * c.cache.k_head,
                              id * c.cache.v_page + row * c.cache.v_token + load.h * c.cache.v_head);
    };
    auto fetch = [&](int step) {
        if (step < n) {
            const int stage = step % kStages;
            const uint32_t k_to = tiles_at + stage * 2 * kTileBytes<D>, v_to = k_to + kTileBytes<D>;
            constexpr int kChunks = D / 8;
            for (int i = tid; i < kTileKeys * kChunks; i += kThreads) {
                const int row = i / kChunks, ch = i - row * kChunks;
                const longlong2 p = place[stage * kTileKeys + row];
                cp_async16(k_to + chunk_at<D>(row, ch), c.cache.k + (p.x < 0 ? 0 : p.x + ch * 16), p.x < 0 ? 0 : 16);
                cp_async16(v_to + chunk_at<D>(row, ch), c.cache.v + (p.x < 0 ? 0 : p.y + ch * 16), p.x < 0 ? 0 : 16);
            }
        }
        cp_async_commit();
    };

    // places of the first three steps, copies of the first two
    for (int s = 0; s < kStages && s < n; ++s) {
        if (tid < kTileKeys) place[s * kTileKeys + tid] = look_up(tid);
        if (s + 1 < n) load.next(c.plan, c.cache.heads);
    }
    __syncthreads();
    for (int s = 0; s < kStages - 1; ++s) fetch(s);

    const int G = c.x.G, quad = lane & 3, row8 = lane >> 2;
    uint32_t q[D / 16][4];
    float o[D / 8][4];
    float m[2], l[2];
    int lim[2];
    int least = 0;                               // keys below this are seen by all rows of the block
    int groups_m = 1, wm = 0, wk = 0, groups_k = 4;
    bool fresh = true;
    bool whole = now.tile == 0;

    for (int i = 0; i < n; ++i) {
        if (fresh) {
            const Block& b = now.at;
            groups_m = b.rows <= 16 ? 1 : b.rows <= 32 ? 2 : 4;
            groups_k = 4 / groups_m;
            wm = warp % groups_m;
            wk = warp / groups_m;
            const int end = b.key0 + b.keys;
            least = min(end, b.limit + b.step * (b.row0 / G));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int row = b.row0 + wm * 16 + row8 + 8 * u;
                const bool there = row < b.row0 + b.rows;
                const int tok = row / G, head = now.h * G + row - tok * G;
                lim[u] = there ? min(end, b.limit + b.step * tok) : end;
                const T* from = static_cast<const T*>(c.x.q) + (b.token0 + (long long)tok) * c.x.q_token + head * c.x.q_head;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    q[ks][u] = there ? *reinterpret_cast<const uint32_t*>(from + ks * 16 + quad * 2) : 0u;
                    q[ks][u + 2] = there ? *reinterpret_cast<const uint32_t*>(from + ks * 16 + quad * 2 + 8) : 0u;
                }
                m[u] = -INFINITY;
                l[u] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < D / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
            fresh = false;
        }
        cp_async_wait<kStages - 2>();
        __syncthreads();
        fetch(i + kStages - 1);
        const int ahead = i + kStages;
        longlong2 found;
        if (ahead < n && tid < kTileKeys) found = look_up(tid);

        const uint32_t k_tile = tiles_at + (i % kStages) * 2 * kTileBytes<D>, v_tile = k_tile + kTileBytes<D>;
        const int left = now.at.keys - now.tile * kTileKeys;
        const int key0 = now.at.key0 + now.tile * kTileKeys;
        for (int g = wk; g < kTileKeys / 16 && g * 16 < left; g += groups_k) {
            float s[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[u][e] = 0.f;
            const int k_row = g * 16 + (lane & 7) + ((lane >> 4) << 3), k_ch = (lane >> 3) & 1;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                uint32_t b[4];
                ldmatrix_x4(b, k_tile + chunk_at<D>(k_row, ks * 2 + k_ch));
                mma_16816(s[0], q[ks], b[0], b[1], T());
                mma_16816(s[1], q[ks], b[2], b[3], T());
            }
            const int key = key0 + g * 16 + quad * 2;
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[u][e] = key + u * 8 + (e & 1) < lim[e >> 1] ? s[u][e] * c.scale : -INFINITY;
                    top[e >> 1] = fmaxf(top[e >> 1], s[u][e]);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 1));
                top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 2));
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
                float alpha[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float higher = fmaxf(m[u], top[u]);
                    alpha[u] = m[u] == higher ? 1.f : ex2(m[u] - higher);
                    m[u] = higher;
                    l[u] *= alpha[u];
                }
#pragma unroll
                for (int j = 0; j < D / 8; ++j) {
                    o[j][0] *= alpha[0]; o[j][1] *= alpha[0];
                    o[j][2] *= alpha[1]; o[j][3] *= alpha[1];
                }
            }
            const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[u][e] = ex2(s[u][e] - base[e >> 1]);
                    l[e >> 1] += s[u][e];
                }
            const uint32_t p[4] = {Pair<T>::pack(s[0][0], s[0][1]), Pair<T>::pack(s[0][2], s[0][3]), Pair<T>::pack(s[1][0], s[1][1]),
                                   Pair<T>::pack(s[1][2], s[1][3])};
            const int v_row = g * 16 + (lane & 15), v_ch = lane >> 4;
            // Where some rows do not see all 16 keys, a value that is not finite must not reach them as 0 times it: such keys (there are none,
            // as a rule) are added one by one.
            bool odd = false;
            if (key0 + g * 16 + 16 > least) {
#pragma unroll
                for (int j = 0; j < D / 8; j += 2) {
                    uint32_t b[4];
                    ldmatrix_x4_trans(b, v_tile + chunk_at<D>(v_row, j + v_ch));
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd |= Pair<T>::not_finite(b[e]);
                }
                odd = __any_sync(0xffffffffu, odd);
            }
            if (odd) {
                for (int n16 = 0; n16 < 16; ++n16) {
                    const int from = (lane & 28) | ((n16 & 7) >> 1);
                    const float a0 = n16 & 8 ? (n16 & 1 ? s[1][1] : s[1][0]) : (n16 & 1 ? s[0][1] : s[0][0]);
                    const float a1 = n16 & 8 ? (n16 & 1 ? s[1][3] : s[1][2]) : (n16 & 1 ? s[0][3] : s[0][2]);
                    const float w[2] = {Pair<T>::rounded(__shfl_sync(0xffffffffu, a0, from)), Pair<T>::rounded(__shfl_sync(0xffffffffu, a1, from))};
                    const char* row = smem + (v_tile - tiles_at);
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) {
                        const T* v = reinterpret_cast<const T*>(row + chunk_at<D>(g * 16 + n16, j)) + quad * 2;
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            if (key0 + g * 16 + n16 < lim[u]) {
                                o[j][2 * u] += w[u] * to_float(v[0]);
                                o[j][2 * u + 1] += w[u] * to_float(v[1]);
                            }
                    }
                }
                continue;
            }
#pragma unroll
            for (int j = 0; j < D / 8; j += 2) {
                uint32_t b[4];
                ldmatrix_x4_trans(b, v_tile + chunk_at<D>(v_row, j + v_ch));
                mma_16816(o[j], p, b[0], b[1], T());
                mma_16816(o[j + 1], p, b[2], b[3], T());
            }
        }
        if (ahead < n && tid < kTileKeys) place[(ahead % kStages) * kTileKeys + tid] = found;
        if (ahead + 1 < n) load.next(c.plan, c.cache.heads);

        const bool ends = now.tile + 1 == now.tiles;
        if (ends || i + 1 == n) {
            // the unit's end, or this CTA's: join the warps that share rows, write
            const Block& b = now.at;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                l[u] += __shfl_xor_sync(0xffffffffu, l[u], 1);
                l[u] += __shfl_xor_sync(0xffffffffu, l[u], 2);
            }
            float all_m[2] = {m[0], m[1]}, all_l[2] = {l[0], l[1]};
            if (groups_k > 1) {
                if (quad == 0) {
                    part[warp * 16 + row8] = make_float2(m[0], l[0]);
                    part[warp * 16 + row8 + 8] = make_float2(m[1], l[1]);
                }
                __syncthreads();
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float top = -INFINITY, sum = 0.f;
                    for (int w = wm; w < 4; w += groups_m) top = fmaxf(top, part[w * 16 + row8 + 8 * u].x);
                    for (int w = wm; w < 4; w += groups_m) {
                        const float2 p = part[w * 16 + row8 + 8 * u];
                        if (p.x > -INFINITY) sum += p.y * ex2(p.x - top);
                    }
                    all_m[u] = top;
                    all_l[u] = sum;
                    const float f = m[u] > -INFINITY ? ex2(m[u] - top) : 0.f;
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) { o[j][2 * u] *= f; o[j][2 * u + 1] *= f; }
                }
                // two row groups: one half of the values at a time, so that both fit
                const int halves = groups_m;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (half >= halves) break;
                    for (int w = 0; w < groups_k; ++w) {
                        if (wk == w) {
#pragma unroll
                            for (int j = 0; j < D / 8; ++j) {
                                if (halves == 2 && (j >= D / 16) != (half == 1)) continue;
                                const int col = (halves == 2 ? j % (D / 16) : j) * 8 + quad * 2, pitch = halves == 2 ? D / 2 : D;
#pragma unroll
                                for (int u = 0; u < 2; ++u) {
                                    float2* at = reinterpret_cast<float2*>(joined + (wm * 16 + row8 + 8 * u) * pitch + col);
                                    float2 v = make_float2(o[j][2 * u], o[j][2 * u + 1]);
                                    if (w > 0) { const float2 old = *at; v.x += old.x; v.y += old.y; }
                                    if (w + 1 < groups_k) *at = v;
                                    else { o[j][2 * u] = v.x; o[j][2 * u + 1] = v.y; }
                                }
                            }
                        }
                        __syncthreads();
                    }
                }
            }
            if (wk == groups_k - 1) {
                const long long unit_begin = c.plan.steps[now.b] + (long long)now.h * now.tiles;   // among all steps
                const bool direct = whole && ends && now.b >= c.plan.head->own && c.plan.share[b.request].prefix < 0;
                const int first_cta = (int)(unit_begin / each);
                const long long at = direct ? 0 : piece_row(c.pieces, c.plan.rows[now.b], c.cache.heads, b.rows, now.h, blockIdx.x, first_cta, kBlockRows);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int in = wm * 16 + row8 + 8 * u;
                    if (in >= b.rows) continue;
                    if (direct) {
                        const int row = b.row0 + in, tok = row / G, head = now.h * G + row - tok * G;
                        const float f = all_l[u] > 0.f ? 1.f / all_l[u] : all_l[u];
                        T* to = static_cast<T*>(c.x.out) + (b.token0 + (long long)tok) * c.x.out_token + head * c.x.out_head;
#pragma unroll
                        for (int j = 0; j < D / 8; ++j)
                            *reinterpret_cast<uint32_t*>(to + j * 8 + quad * 2) = Pair<T>::pack(o[j][2 * u] * f, o[j][2 * u + 1] * f);
                        if (quad == 0)
                            c.x.lse[(b.token0 + (long long)tok) * c.x.lse_token + head] = (all_m[u] + log2f(all_l[u])) * 0.6931471805599453f;
                    } else {
                        float* to = c.pieces.o + (at + in) * D;
#pragma unroll
                        for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(to + j * 8 + quad * 2) = make_float2(o[j][2 * u], o[j][2 * u + 1]);
                        if (quad == 0) c.pieces.ml[at + in] = make_float2(all_m[u], all_l[u]);
                    }
                }
            }
            fresh = true;
            whole = true;
        }
        if (i + 1 < n) now.next(c.plan, c.cache.heads);
    }
    cp_async_wait<0>();
}

// ---- pieces -------------------------------------------------------------------------------------
// A CTA a unit of the requests' own tokens, a warp a row: the pieces of the unit and those of the same row among its group's shared tokens.
template <typename T, int D>
__global__ void __launch_bounds__(256) join_kernel(const Call c, int ctas) {
    ardiff::begin_kernel();
    const int lane = threadIdx.x & 31, H = c.cache.heads, G = c.x.G;
    const PlanHead head = *c.plan.head;
    const long long each = steps_each(head.steps, ctas), units = (long long)(head.blocks - head.own) * H;
    for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int b = head.own + (int)(unit / H), h = (int)(unit % H);
        const Block k = c.plan.block[b];
        const Share share = c.plan.share[k.request];
        const int tiles = (k.keys + kTileKeys - 1) / kTileKeys;
        const long long s0 = c.plan.steps[b] + (long long)h * tiles;
        const int c0 = (int)(s0 / each), mine = tiles ? (int)((s0 + tiles - 1) / each) - c0 + 1 : 0;
        if (mine == 1 && share.prefix < 0) continue;                                // written already
        for (int in = threadIdx.x >> 5; in < k.rows; in += 8) {
            int theirs = 0, t0 = 0, t_in = 0, t_rows = 0;
            long long t_before = 0;
            if (share.prefix >= 0) {
                const int row = share.row0 + k.row0 + in, pb = share.prefix + row / kBlockRows;
                const Block p = c.plan.block[pb];
                const int p_tiles = (p.keys + kTileKeys - 1) / kTileKeys;
                const long long p0 = c.plan.steps[pb] + (long long)h * p_tiles;
                t0 = (int)(p0 / each);
                theirs = (int)((p0 + p_tiles - 1) / each) - t0 + 1;
                t_in = row % kBlockRows;
                t_rows = p.rows;
                t_before = c.plan.rows[pb];
            }
            auto row_of = [&](int i) -> long long {
                return i < mine ? piece_row(c.pieces, c.plan.rows[b], H, k.rows, h, c0 + i, c0, kBlockRows) + in
                                : piece_row(c.pieces, t_before, H, t_rows, h, t0 + i - mine, t0, kBlockRows) + t_in;
            };
            const int all = mine + theirs;
            float top = -INFINITY;
            for (int i = lane; i < all; i += 32) top = fmaxf(top, c.pieces.ml[row_of(i)].x);
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float base = top == -INFINITY ? 0.f : top;
            constexpr int kValues = (D + 31) / 32;
            float acc[kValues], sum = 0.f;
#pragma unroll
            for (int j = 0; j < kValues; ++j) acc[j] = 0.f;
            for (int i0 = 0; i0 < all; i0 += 32) {
                float w = 0.f;
                long long at = 0;
                if (i0 + lane < all) {
                    at = row_of(i0 + lane);
                    const float2 ml = c.pieces.ml[at];
                    w = ex2(ml.x - base);
                    sum += w * ml.y;
                }
                for (int i = 0; i < min(32, all - i0); ++i) {
                    const float f = __shfl_sync(0xffffffffu, w, i);
                    const float* from = c.pieces.o + __shfl_sync(0xffffffffu, at, i) * D;
#pragma unroll
                    for (int j = 0; j < kValues; ++j)
                        if (lane + 32 * j < D) acc[j] += f * from[lane + 32 * j];
                }
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float f = sum > 0.f ? 1.f / sum : sum;                             // no key: 0, and lse -inf
            const int row = k.row0 + in, tok = row / G, qh = h * G + row - tok * G;
            T* to = static_cast<T*>(c.x.out) + (k.token0 + (long long)tok) * c.x.out_token + qh * c.x.out_head;
#pragma unroll
            for (int j = 0; j < kValues; ++j)
                if (lane + 32 * j < D) to[lane + 32 * j] = from_float<T>(acc[j] * f);
            if (lane == 0) c.x.lse[(k.token0 + (long long)tok) * c.x.lse_token + qh] = (base + log2f(sum)) * 0.6931471805599453f;
        }
    }
}

// ---- the call -----------------------------------------------------------------------------------
struct Sizes {
    long long blocks, main_rows, bytes, block_at, steps_at, rows_at, share_at, shared_at, ml_at, o_at;
};
Sizes sizes(long long requests, long long groups, long long tokens, long long q_heads, long long heads, long long width) {
    Sizes s;
    const long long G = q_heads / heads;
    // blocks of requests or groups: one each for their ends, and the full ones
    s.blocks = requests + tokens * G / kBlockRows + (groups > 0 ? (groups < requests ? groups : requests) + tokens * G / kBlockRows : 0) + 1;
    s.main_rows = tokens * q_heads * (groups > 0 ? 2 : 1);
    auto up = [](long long v) { return (v + 255) / 256 * 256; };
    long long at = 256;
    s.block_at = at; at = up(at + s.blocks * (long long)sizeof(Block));
    s.steps_at = at; at = up(at + (s.blocks + 1) * 8);
    s.rows_at = at; at = up(at + (s.blocks + 1) * 8);
    s.share_at = at; at = up(at + requests * (long long)sizeof(Share));
    s.shared_at = at; at = up(at + requests * 4);
    const long long rows = s.main_rows + (long long)kMaxCtas * kBlockRows;
    s.ml_at = at; at = up(at + rows * 8);
    s.o_at = at; at = up(at + rows * width * 4);
    s.bytes = at;
    return s;
}

template <typename T, int D> bool launch(const Call& c, int sms, cudaStream_t st) {
    const int ctas = 2 * sms < kMaxCtas ? 2 * sms : kMaxCtas;
    if (cudaFuncSetAttribute(narrow_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kNarrowShared<D>) != cudaSuccess) return false;
    return launch_early(plan_kernel, 1, kPlanThreads, 1, 0, st, c) && launch_early(narrow_kernel<T, D>, ctas, kThreads, 1, kNarrowShared<D>, st, c, ctas) &&
           launch_early(join_kernel<T, D>, 8 * sms, 256, 1, 0, st, c, ctas);
}
template <typename T> bool launch_width(const Call& c, int width, int sms, cudaStream_t st) {
    switch (width) {
        case 64: return launch<T, 64>(c, sms, st);
        case 80: return launch<T, 80>(c, sms, st);
        case 96: return launch<T, 96>(c, sms, st);
        default: return launch<T, 128>(c, sms, st);
    }
}

bool shape(int64_t requests, int64_t groups, int64_t tokens, int64_t q_heads, int64_t heads) {
    return requests >= 0 && requests <= ARDIFF_PAGES_MAX_REQUESTS && groups >= 0 && groups <= ARDIFF_PAGES_MAX_REQUESTS && tokens >= 0 && heads >= 1 &&
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
    return sizes(requests, groups, tokens, q_heads, heads, head_width).bytes;
}

extern "C" int ardiff_attend_pages(const void* q, int64_t q_token, int64_t q_head, int32_t q_heads, int64_t tokens, int32_t dtype, const void* k_cache,
                                   int64_t k_page, int64_t k_token, int64_t k_head, const void* v_cache, int64_t v_page, int64_t v_token,
                                   int64_t v_head, int32_t pages, int32_t page, int32_t heads, int32_t head_width, const int32_t* table,
                                   int32_t width, int32_t requests, const int32_t* length, const int32_t* offset, int32_t groups,
                                   const int32_t* group, const int32_t* shared, int32_t most, float scale, int32_t causal, void* out,
                                   int64_t out_token, int64_t out_head, float* lse, int64_t lse_token, int32_t* status, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
    if (!shape(requests, groups, tokens, q_heads, heads) || pages < 0 || page < 1 || width < 0 || (int64_t)page * width >= (int64_t)1 << 31 || most < 0 ||
        !isfinite(scale))
        return ARDIFF_ERR_SHAPE;
    if ((dtype != ARDIFF_BF16 && dtype != ARDIFF_F16) || (head_width != 64 && head_width != 80 && head_width != 96 && head_width != 128))
        return ARDIFF_ERR_UNSUPPORTED;
    if (!status || !offset || !workspace) return ARDIFF_ERR_NULL;
    if (requests > 0 && (!length || (width > 0 && !table) || !k_cache || !v_cache)) return ARDIFF_ERR_NULL;
    if (tokens > 0 && (!q || !out || !lse)) return ARDIFF_ERR_NULL;
    if (groups > 0 && (!group || !shared)) return ARDIFF_ERR_NULL;
    auto low = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if (((low(q) | low(out) | low(k_cache) | low(v_cache)) & 15u) || (low(workspace) & 255u) ||
        ((q_token | q_head | out_token | out_head | k_page | k_token | k_head | v_page | v_token | v_head) & 7))
        return ARDIFF_ERR_ALIGN;
    const Sizes s = sizes(requests, groups, tokens, q_heads, heads, head_width);
    if (workspace_bytes < s.bytes) return ARDIFF_ERR_SHAPE;
    const int sms = device_sms();
    if (sms < 1) return ARDIFF_ERR_CUDA;
    Call c;
    memset(&c, 0, sizeof(c));
    c.cache = Pages{static_cast<const char*>(k_cache), static_cast<const char*>(v_cache), k_page * 2, k_token * 2, k_head * 2, v_page * 2,
                    v_token * 2, v_head * 2, table, width, page, pages, heads};
    c.x.q = q; c.x.out = out; c.x.lse = lse; c.x.q_token = q_token; c.x.q_head = q_head; c.x.out_token = out_token; c.x.out_head = out_head;
    c.x.lse_token = lse_token; c.x.heads = q_heads; c.x.G = q_heads / heads; c.x.tokens = tokens;
    char* w = static_cast<char*>(workspace);
    c.plan.head = reinterpret_cast<PlanHead*>(w);
    c.plan.block = reinterpret_cast<Block*>(w + s.block_at);
    c.plan.steps = reinterpret_cast<long long*>(w + s.steps_at);
    c.plan.rows = reinterpret_cast<long long*>(w + s.rows_at);
    c.plan.share = reinterpret_cast<Share*>(w + s.share_at);
    c.plan.shared = reinterpret_cast<int*>(w + s.shared_at);
    c.pieces.ml = reinterpret_cast<float2*>(w + s.ml_at);
    c.pieces.o = reinterpret_cast<float*>(w + s.o_at);
    c.pieces.main_rows = s.main_rows;
    c.length = length; c.offset = offset; c.group = group; c.shared = shared; c.status = status;
    c.scale = scale * 1.4426950408889634f;
    c.requests = requests; c.groups = groups; c.causal = causal != 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool ok = dtype == ARDIFF_F16 ? launch_width<__half>(c, head_width, sms, st) : launch_width<__nv_bfloat16>(c, head_width, sms, st);
    ardiff::set_launch_count(3);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}
