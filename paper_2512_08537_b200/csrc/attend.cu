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

constexpr int kMaxCtas = 512, kMaxWideCtas = 256;    // CTAs that have a place for pieces
constexpr int kPlanThreads = 1024;
// Fewer shared tokens are read by every request itself: a block of its own and the pieces to join cost more than they take.
constexpr int kLeastShared = 64;

// ---- the plan -----------------------------------------------------------------------------------
// Blocks of a segment: of which list, how many.
__device__ __forceinline__ bool is_wide(long long rows) { return rows > kNarrowRows; }
__device__ __forceinline__ int blocks_of(long long rows) {
    return (int)(is_wide(rows) ? (rows + kWideRows - 1) / kWideRows : (rows + kNarrowRows - 1) / kNarrowRows);
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const Call c) {
    __shared__ long long s_scan[32];
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, R = c.requests, G = c.x.G;
    const long long limit = (long long)c.cache.width * c.cache.page;
    bool bad = false;
    for (int r = tid; r < R; r += kPlanThreads) {
        const int a = c.offset[r], b = c.offset[r + 1], len = c.length[r];
        bad |= a < 0 || b < a || b > c.x.tokens || len < 0 || len > limit;
        c.plan.share[r] = Share{-1, 0, 0, 0, 0, r, 0, 0};
    }
    for (int g = tid; g < c.groups; g += kPlanThreads) {
        const int a = c.group[g], b = c.group[g + 1];
        bad |= a < 0 || b < a || b > R || c.shared[g] < 0;
    }
    bad = __syncthreads_or(bad);
    if (tid == 0) *c.status = bad ? ARDIFF_ERR_SHAPE : ARDIFF_OK;
    if (bad) {
        if (tid < 2) *(tid ? c.plan.wide : c.plan.narrow).head = PlanHead{0, 0, 0, 0};
        return;
    }
    // The tokens that all queries of a group see are found through its first row of the table, and read once for all, unless
    // one request has queries, or all have so many that each fills its blocks of rows: then the same work is done, and there are no pieces to join.
    for (int g = tid >> 5; g < c.groups; g += kPlanThreads / 32) {
        const int r0 = c.group[g], r1 = c.group[g + 1];
        int least = c.shared[g], active = 0, fewest = 0x7fffffff;
        for (int r = r0 + lane; r < r1; r += 32) {
            const int n = c.offset[r + 1] - c.offset[r];
            if (n == 0) continue;
            ++active;
            fewest = min(fewest, n);
            least = min(least, max(0, c.causal ? c.length[r] - n + 1 : c.length[r]));
        }
        least = __reduce_min_sync(0xffffffffu, least);
        fewest = __reduce_min_sync(0xffffffffu, fewest);
        active = __reduce_add_sync(0xffffffffu, active);
        const bool once = active > 1 && least >= kLeastShared && (long long)fewest * G < kWideRows;
        for (int r = r0 + lane; r < r1; r += 32) c.plan.share[r] = Share{-1, 0, 0, once ? least : 0, least, r0, 0, 0};
    }
    __syncthreads();

    long long blocks[2] = {0, 0};                // narrow, wide
    // shared tokens: blocks of the group's rows
    for (int g0 = 0; g0 < c.groups; g0 += kPlanThreads) {
        const int g = g0 + tid;
        int n = 0, r0 = 0, keys = 0, token0 = 0;
        long long rows = 0;
        if (g < c.groups) {
            r0 = c.group[g];
            const int r1 = c.group[g + 1];
            if (r1 > r0) {
                keys = c.plan.share[r0].shared;
                token0 = c.offset[r0];
                rows = keys > 0 ? (long long)(c.offset[r1] - token0) * G : 0;
            }
            n = blocks_of(rows);
        }
        const bool wide = is_wide(rows);
        long long total;
        const long long packed = cta_scan((long long)(wide ? 0 : n) << 32 | (wide ? n : 0), s_scan, &total);
        const long long at = wide ? blocks[1] + (int)packed : blocks[0] + (packed >> 32);
        const int per = wide ? kWideRows : kNarrowRows;
        for (int j = 0; j < n; ++j) {
            Block b;
            b.token0 = token0; b.row0 = j * per; b.rows = (int)min((long long)per, rows - b.row0);
            b.request = r0; b.key0 = b.low = 0; b.keys = keys; b.limit = keys; b.step = 0; b.split = 0; b.front = r0; b.pad = 0;
            (wide ? c.plan.wide : c.plan.narrow).block[at + j] = b;
        }
        if (n > 0) { c.plan.share[r0].prefix = (int)at; c.plan.share[r0].wide = wide; }
        blocks[0] += total >> 32;
        blocks[1] += (int)total;
    }
    const int own[2] = {(int)blocks[0], (int)blocks[1]};
    __syncthreads();
    for (int g = tid >> 5; g < c.groups; g += kPlanThreads / 32) {
        const int r0 = c.group[g], r1 = c.group[g + 1];
        if (r0 == r1) continue;
        const Share first = c.plan.share[r0];
        const int token0 = c.offset[r0];
        __syncwarp();
        for (int r = r0 + lane; r < r1 && first.prefix >= 0; r += 32) {
            Share s = first;
            s.row0 = (c.offset[r] - token0) * G;
            c.plan.share[r] = s;
        }
    }
    __syncthreads();
    for (int first = 0; first < R; first += kPlanThreads) {
        const int r = first + tid;
        int n = 0, token0 = 0, len = 0, news = 0;
        long long rows = 0;
        Share share{-1, 0, 0, 0, 0, 0, 0, 0};
        if (r < R) {
            token0 = c.offset[r];
            news = c.offset[r + 1] - token0;
            len = c.length[r];
            share = c.plan.share[r];
            rows = (long long)news * G;
            n = blocks_of(rows);
        }
        const bool wide = is_wide(rows);
        long long total;
        const long long packed = cta_scan((long long)(wide ? 0 : n) << 32 | (wide ? n : 0), s_scan, &total);
        const long long at = wide ? blocks[1] + (int)packed : blocks[0] + (packed >> 32);
        const int per = wide ? kWideRows : kNarrowRows;
        for (int j = 0; j < n; ++j) {
            Block b;
            b.token0 = token0; b.row0 = j * per; b.rows = (int)min((long long)per, rows - b.row0);
            b.request = r; b.low = share.shared; b.split = share.split; b.front = share.front; b.pad = 0;
            b.key0 = wide ? b.low / kWideKeys * kWideKeys : b.low;
            b.step = c.causal ? 1 : 0;
            b.limit = c.causal ? len - news + 1 : len;
            const int last = min(len, b.limit + b.step * ((b.row0 + b.rows - 1) / G));
            b.keys = last > b.low ? last - b.key0 : 0;
            (wide ? c.plan.wide : c.plan.narrow).block[at + j] = b;
        }
        blocks[0] += total >> 32;
        blocks[1] += (int)total;
    }
    __syncthreads();
    long long before = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const List& l = i ? c.plan.wide : c.plan.narrow;
        const int keys = i ? kWideKeys : kNarrowKeys;
        long long steps = 0, rows = 0;
        for (int first = 0; first < blocks[i]; first += kPlanThreads) {
            const int b = first + tid;
            long long s = 0, w = 0;
            if (b < blocks[i]) {
                s = (long long)((l.block[b].keys + keys - 1) / keys) * c.cache.heads;
                w = l.block[b].rows;
            }
            long long total;
            const long long at = steps + cta_scan(s, s_scan, &total);
            steps += total;
            const long long rows_at = rows + cta_scan(w, s_scan, &total);
            rows += total;
            if (b < blocks[i]) { l.steps[b] = at; l.rows[b] = rows_at; }
        }
        if (tid == 0) {
            l.steps[blocks[i]] = steps;
            l.rows[blocks[i]] = rows;
            *l.head = PlanHead{steps, before, (int)blocks[i], own[i]};
        }
        before = rows;
    }
}

// ---- up to 64 query rows ------------------------------------------------------------------------
constexpr int kThreads = 128;
constexpr int kStages = 3;

template <int D> constexpr int kTileBytes = kNarrowKeys * kPitch<D>;
template <int D> constexpr int kNarrowShared = kStages * 2 * kTileBytes<D> + 16 * D * 4 + kStages * kNarrowKeys * 16 + 4 * 16 * 8;

// Four warps. Those that share 16 query rows (all four where the block has up to 16 rows, two up to 32) take turns at groups of 16 keys, each
// with a running maximum, sum and weighted values of its own, joined in shared memory when the unit ends. Keys and values come by asynchronous copies,
// two tiles ahead, through offsets that are looked up in the table a step before that.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2) narrow_kernel(const Call c) {
    extern __shared__ __align__(128) char smem[];
    char* tiles = smem;
    float* joined = reinterpret_cast<float*>(smem + kStages * 2 * kTileBytes<D>);
    longlong2* place = reinterpret_cast<longlong2*>(joined + 16 * D);                // [stages][keys]
    float2* part = reinterpret_cast<float2*>(place + kStages * kNarrowKeys);           // [warps][16]
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const List& list = c.plan.narrow;
    const long long steps = list.head->steps, each = steps_each(steps, list.ctas);
    const long long begin = each * blockIdx.x;
    if (begin >= steps) return;
    const int n = (int)(min(steps, begin + each) - begin), own = list.head->own;
    const uint32_t tiles_at = ptx::smem_u32(tiles);

    Cursor<false> now;
    now.start(c, find_last(list.steps, list.head->blocks, begin), begin);
    Cursor<false> load = now;                    // the step whose places are looked up next

    auto fetch = [&](int step) {
        if (step < n) {
            const int stage = step % kStages;
            const uint32_t k_to = tiles_at + stage * 2 * kTileBytes<D>, v_to = k_to + kTileBytes<D>;
            constexpr int kChunks = D / 8;
            for (int i = tid; i < kNarrowKeys * kChunks; i += kThreads) {
                const int row = i / kChunks, ch = i - row * kChunks;
                const longlong2 p = place[stage * kNarrowKeys + row];
                cp_async16(k_to + chunk_at<D>(row, ch), c.cache.k + (p.x < 0 ? 0 : p.x + ch * 16), p.x < 0 ? 0 : 16);
                cp_async16(v_to + chunk_at<D>(row, ch), c.cache.v + (p.x < 0 ? 0 : p.y + ch * 16), p.x < 0 ? 0 : 16);
            }
        }
        cp_async_commit();
    };

    // places of the first three steps, copies of the first two
    for (int s = 0; s < kStages && s < n; ++s) {
        if (tid < kNarrowKeys) place[s * kNarrowKeys + tid] = place_of<false>(c, load, tid);
        if (s + 1 < n) load.next(c);
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
        if (ahead < n && tid < kNarrowKeys) found = place_of<false>(c, load, tid);

        const uint32_t k_tile = tiles_at + (i % kStages) * 2 * kTileBytes<D>, v_tile = k_tile + kTileBytes<D>;
        const int left = now.at.keys - now.tile * kNarrowKeys;
        const int key0 = now.at.key0 + now.tile * kNarrowKeys;
        for (int g = wk; g < kNarrowKeys / 16 && g * 16 < left; g += groups_k) {
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
        if (ahead < n && tid < kNarrowKeys) place[(ahead % kStages) * kNarrowKeys + tid] = found;
        if (ahead + 1 < n) load.next(c);

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
                const long long unit = list.steps[now.b] + (long long)now.h * now.tiles;       // its first step
                const bool direct = whole && ends && now.b >= own && c.plan.share[b.request].prefix < 0;
                const long long at = direct ? 0 : piece_row<false>(c, now.b, b, now.h, blockIdx.x, (int)(unit / each));
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
        if (i + 1 < n) now.next(c);
    }
    cp_async_wait<0>();
}

// ---- pieces -------------------------------------------------------------------------------------
// The pieces of a unit: of CTAs first .. first + count - 1.
struct Cut {
    int first, count;
};
template <bool kWide> __device__ __forceinline__ Cut cut_of(const Call& c, int b, const Block& k, int h) {
    const List& l = list_of<kWide>(c);
    const int tiles = (k.keys + Sizes<kWide>::keys - 1) / Sizes<kWide>::keys;
    if (tiles == 0) return Cut{0, 0};
    const long long each = steps_each(l.head->steps, l.ctas), s0 = l.steps[b] + (long long)h * tiles;
    const int first = (int)(s0 / each);
    return Cut{first, (int)((s0 + tiles - 1) / each) - first + 1};
}

// A CTA a unit of the requests' own tokens, a warp a row: the pieces of the unit and those of the same row among its group's shared tokens.
template <typename T, int D, bool kWide>
__device__ __forceinline__ void join_unit(const Call& c, int b, int h) {
    const int lane = threadIdx.x & 31, G = c.x.G;
    const Block k = list_of<kWide>(c).block[b];
    const Share share = c.plan.share[k.request];
    const Cut mine = cut_of<kWide>(c, b, k, h);
    if (mine.count == 1 && share.prefix < 0) return;                                // written already
    for (int in = threadIdx.x >> 5; in < k.rows; in += 8) {
        Cut theirs{0, 0};
        Block p = k;
        int pb = 0, p_in = 0;
        if (share.prefix >= 0) {
            const int row = share.row0 + k.row0 + in, per = share.wide ? kWideRows : kNarrowRows;
            pb = share.prefix + row / per;
            p_in = row % per;
            p = (share.wide ? c.plan.wide : c.plan.narrow).block[pb];
            theirs = share.wide ? cut_of<true>(c, pb, p, h) : cut_of<false>(c, pb, p, h);
        }
        auto row_of = [&](int i) -> long long {
            if (i < mine.count) return piece_row<kWide>(c, b, k, h, mine.first + i, mine.first) + in;
            const int cta = theirs.first + i - mine.count;
            return (share.wide ? piece_row<true>(c, pb, p, h, cta, theirs.first) : piece_row<false>(c, pb, p, h, cta, theirs.first)) + p_in;
        };
        const int all = mine.count + theirs.count;
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

template <typename T, int D>
__global__ void __launch_bounds__(256) join_kernel(const Call c) {
    ardiff::begin_kernel();
    const int H = c.cache.heads;
    const PlanHead narrow = *c.plan.narrow.head, wide = *c.plan.wide.head;
    const long long narrow_units = (long long)(narrow.blocks - narrow.own) * H, units = narrow_units + (long long)(wide.blocks - wide.own) * H;
    for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        if (unit < narrow_units) join_unit<T, D, false>(c, narrow.own + (int)(unit / H), (int)(unit % H));
        else join_unit<T, D, true>(c, wide.own + (int)((unit - narrow_units) / H), (int)((unit - narrow_units) % H));
    }
}

// ---- the call -----------------------------------------------------------------------------------
struct Layout {
    long long narrow_blocks, wide_blocks, main_rows, bytes, block_at[2], steps_at[2], rows_at[2], share_at, ml_at, o_at;
};
Layout layout(long long requests, long long groups, long long tokens, long long q_heads, long long heads, long long width) {
    Layout s;
    const long long rows = tokens * (q_heads / heads), parts = groups > 0 ? 2 : 1, ends = requests + (groups < requests ? groups : requests);
    // narrow: a segment of 1 to 64 rows each; wide: the full blocks, and one for the end of every segment of more than 64 rows
    s.narrow_blocks = (ends < parts * rows ? ends : parts * rows) + 1;
    s.wide_blocks = parts * (rows / kWideRows + (rows / kNarrowRows < requests ? rows / kNarrowRows : requests)) + 1;
    s.main_rows = tokens * q_heads * parts;
    auto up = [](long long v) { return (v + 255) / 256 * 256; };
    long long at = 256;
    for (int i = 0; i < 2; ++i) {
        const long long blocks = i ? s.wide_blocks : s.narrow_blocks;
        s.block_at[i] = at; at = up(at + blocks * (long long)sizeof(Block));
        s.steps_at[i] = at; at = up(at + (blocks + 1) * 8);
        s.rows_at[i] = at; at = up(at + (blocks + 1) * 8);
    }
    s.share_at = at; at = up(at + requests * (long long)sizeof(Share));
    const long long pieces = s.main_rows + (long long)kMaxCtas * kNarrowRows + (long long)kMaxWideCtas * kWideRows;
    s.ml_at = at; at = up(at + pieces * 8);
    s.o_at = at; at = up(at + pieces * width * 4);
    s.bytes = at;
    return s;
}

// Whether a block may have more than 64 rows: `most` and the number of tokens say what they can.
bool may_be_wide(const Call& c, int most) {
    const long long news = most > 0 && most < c.x.tokens ? most : c.x.tokens;
    return (c.groups > 0 ? c.x.tokens : news) * c.x.G > kNarrowRows;
}

template <typename T, int D> bool launch(const Call& c, int32_t dtype, int most, int sms, cudaStream_t st) {
    if (cudaFuncSetAttribute(narrow_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kNarrowShared<D>) != cudaSuccess) return false;
    const bool wide = may_be_wide(c, most);
    ardiff::set_launch_count(wide ? 4 : 3);
    return launch_early(plan_kernel, 1, kPlanThreads, 1, 0, st, c) && (!wide || launch_wide(c, dtype, D, st)) &&
           launch_early(narrow_kernel<T, D>, c.plan.narrow.ctas, kThreads, 1, kNarrowShared<D>, st, c) &&
           launch_early(join_kernel<T, D>, 8 * sms, 256, 1, 0, st, c);
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
    return layout(requests, groups, tokens, q_heads, heads, head_width).bytes;
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
    const Layout s = layout(requests, groups, tokens, q_heads, heads, head_width);
    if (workspace_bytes < s.bytes) return ARDIFF_ERR_SHAPE;
    const int sms = device_sms();
    if (sms < 1) return ARDIFF_ERR_CUDA;
    Call c;
    memset(&c, 0, sizeof(c));
    c.cache = Pages{static_cast<const char*>(k_cache), static_cast<const char*>(v_cache), k_page * 2, k_token * 2, k_head * 2, v_page * 2,
                    v_token * 2, v_head * 2, table, width, page, pages, heads};
    c.x.q = q; c.x.out = out; c.x.lse = lse; c.x.q_token = q_token; c.x.q_head = q_head; c.x.out_token = out_token; c.x.out_head = out_head;
    c.x.lse_token = lse_token; c.x.heads = q_heads; c.x.G = q_heads / heads; c.x.tokens = tokens;
    c.x.by_G = divide_by(q_heads / heads);
    char* w = static_cast<char*>(workspace);
    for (int i = 0; i < 2; ++i) {
        List& l = i ? c.plan.wide : c.plan.narrow;
        l.head = reinterpret_cast<PlanHead*>(w) + i;
        l.block = reinterpret_cast<Block*>(w + s.block_at[i]);
        l.steps = reinterpret_cast<long long*>(w + s.steps_at[i]);
        l.rows = reinterpret_cast<long long*>(w + s.rows_at[i]);
    }
    c.plan.narrow.ctas = 2 * sms < kMaxCtas ? 2 * sms : kMaxCtas;
    c.plan.wide.ctas = sms < kMaxWideCtas ? sms : kMaxWideCtas;
    c.plan.share = reinterpret_cast<Share*>(w + s.share_at);
    c.pieces.ml = reinterpret_cast<float2*>(w + s.ml_at);
    c.pieces.o = reinterpret_cast<float*>(w + s.o_at);
    c.pieces.narrow_rows = s.main_rows;
    c.pieces.wide_rows = s.main_rows + (long long)kMaxCtas * kNarrowRows;
    c.length = length; c.offset = offset; c.group = group; c.shared = shared; c.status = status;
    c.scale = scale * 1.4426950408889634f;
    c.requests = requests; c.groups = groups; c.causal = causal != 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool ok = dtype == ARDIFF_F16 ? launch_width<__half>(c, dtype, head_width, most, sms, st)
                                        : launch_width<__nv_bfloat16>(c, dtype, head_width, most, sms, st);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}
