// Attention over pages for blocks of more than 64 query rows, on the tensor cores: a CTA takes 256 rows (two tiles of 128) through the
// tiles of 128 keys that are its share of the line of steps.
//
//   S_t = Q_t K^T          tcgen05, 128 x 128 in tensor memory, tile t = 0, 1
//   P_t = 2^(S_t scale - m_t), m_t a running maximum of every row
//   O_t = O_t + P_t V      tcgen05, P_t from tensor memory (16-bit, over S_t's first columns), V as it lies in the cache (keys are rows: N-major)
//
// While one tile's rows go through the exponentials the tensor cores work on the other's products, so both pipes stay busy: per step 4 x 128 x 128
// x width multiply-adds (2048 cycles at 128) and 2 x 128 x 128 exponentials (2048 cycles of 16 a clock).
// The maximum only moves when it would grow by more than 8 (a factor 256 that P and the sums hold easily): then O is rescaled in
// tensor memory, which is rare; the product that last wrote O is done by then, since its successor S_t is issued after it.
//
// Warps: 0-3 and 4-7 the rows of tile 0 and 1 (a thread a row), 8 issues products, 9-11 copy. Queries, keys and values come by asynchronous 16-byte
// copies through places looked up in the table, into the 128-byte-swizzled layout that the products read; pages may have any size and strides.
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

constexpr int kThreads = 12 * 32;               // three warps a quarter of the SM: 168 registers each
constexpr int kLoaders = 96;                    // threads that copy
constexpr int kRows = 128;                       // of a tile
constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemColumns = 512;
constexpr float kSlack = 8.f;
constexpr unsigned long long kWaitLimit = 4000000000ull;   // ns

template <int D> constexpr int kSub = (D + 63) / 64;                       // blocks of 64 values of a row
template <int D> constexpr int kTile = kSub<D> * 128 * 128;                // bytes of 128 rows
template <int D> constexpr int kShared = 1024 + 6 * kTile<D> + 2 * 128 * 16;

enum Bar { kQFull, kQEmpty, kKFull, kKEmpty = kKFull + 2, kVFull = kKEmpty + 2, kVEmpty = kVFull + 2, kSFull = kVEmpty + 2, kPFull = kSFull + 2,
           kOFull = kPFull + 2, kDrained = kOFull + 2, kBars };

// Waits give up after kWaitLimit, tell the status and make all others give up.
struct Waits {
    uint32_t bars;
    volatile int* stop;
    int32_t* status;
    __device__ __forceinline__ bool operator()(int bar, uint32_t parity) const {
        if (ptx::mbar_try_wait(bars + bar * 8, parity)) return true;
        return slow(bar, parity);
    }
    __device__ __noinline__ bool slow(int bar, uint32_t parity) const {
        const unsigned long long t0 = ptx::globaltimer_ns();
        while (!*stop) {
            for (int i = 0; i < 64; ++i)
                if (ptx::mbar_try_wait(bars + bar * 8, parity)) return true;
            if (ptx::globaltimer_ns() - t0 > kWaitLimit) {
                *stop = 1;
                *status = ARDIFF_ERR_TIMEOUT;
            }
        }
        return false;
    }
};

__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// byte of 16-byte chunk c of a row of D values, in tiles of blocks of 64 values
__device__ __forceinline__ uint32_t swizzled(int row, int c) {
    return (uint32_t)((c >> 3) * 16384 + row * 128 + (((c & 7) ^ (row & 7)) << 4));
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) wide_kernel(const Call c) {
    extern __shared__ char raw[];
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kQ = 0, kK = 2 * kTile<D>, kV = 4 * kTile<D>;
    longlong2* place = reinterpret_cast<longlong2*>(smem + 6 * kTile<D>);            // [2][128]
    __shared__ __align__(8) uint64_t s_bar[kBars];
    __shared__ uint32_t s_tmem;
    __shared__ int s_stop;
    __shared__ int s_odd[2];                     // values of the stage that are not finite, where some row does not see them
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bars = ptx::smem_u32(s_bar), at = ptx::smem_u32(smem);
    ardiff::begin_kernel();
    const List& list = c.plan.wide;
    const long long steps = list.head->steps, each = steps_each(steps, list.ctas), begin = each * blockIdx.x;
    if (begin >= steps) return;
    const int n = (int)(min(steps, begin + each) - begin), own = list.head->own, G = c.x.G;
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            const bool loaders = i == kQFull || i == kKFull || i == kKFull + 1 || i == kVFull || i == kVFull + 1;
            ptx::mbar_init(bars + i * 8, loaders ? kLoaders : i == kPFull || i == kPFull + 1 ? 128 : 1);
        }
        s_stop = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 8) {
        ptx::tmem_alloc(ptx::smem_u32(&s_tmem), kTmemColumns);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = s_tmem;
    const Waits wait{bars, &s_stop, c.status};
    Cursor<true> now;
    now.start(c, find_last(list.steps, list.head->blocks, begin), begin);

    if (warp >= 9) {
        // ---- copies
        const int t = tid - 9 * 32;
        constexpr int kChunks = D / 8;
        longlong2 found[2];                      // of keys t and t + 96 of the step that is copied next
        auto look_up = [&](const Cursor<true>& x) {
            found[0] = place_of<true>(c, x, t);
            if (t + kLoaders < kWideKeys) found[1] = place_of<true>(c, x, t + kLoaders);
        };
        look_up(now);
        Cursor<true> load = now;                 // of the places looked up last
        uint32_t unit = 0;
        bool fresh = true;
        auto signal_v = [&](int i, const Cursor<true>& x) {
            // the keys that some row of the block does not see must not reach it as 0 times a value that is not finite
            const int least = min(x.at.key0 + x.at.keys, x.at.limit + x.at.step * (x.at.row0 / G));
            const int stage = i & 1;
            if (x.at.key0 + (x.tile + 1) * kWideKeys > least) {
                bool odd = false;
                for (int j = t; j < kWideKeys * kChunks; j += kLoaders) {
                    const uint4 v = *reinterpret_cast<const uint4*>(smem + kV + stage * kTile<D> + swizzled(j / kChunks, j % kChunks));
                    odd |= Pair<T>::not_finite(v.x) || Pair<T>::not_finite(v.y) || Pair<T>::not_finite(v.z) || Pair<T>::not_finite(v.w);
                }
                if (odd) s_odd[stage] = 1;
            }
            ptx::fence_proxy_async_smem();
            ptx::mbar_arrive(bars + (kVFull + stage) * 8);
        };
        Cursor<true> last = now;                 // of step i - 1
        auto copy = [&](int i) -> bool {
            const int stage = i & 1;
            const uint32_t parity = (((uint32_t)i >> 1) & 1) ^ 1;
            if (fresh) {
                if (!wait(kQEmpty, (unit & 1) ^ 1)) return false;
                for (int j = t; j < 2 * kRows * kChunks; j += kLoaders) {
                    const int in = j / kChunks, ch = j - in * kChunks;
                    const bool there = in < now.at.rows;
                    const int row = now.at.row0 + in, tok = row / G;
                    const T* from = static_cast<const T*>(c.x.q);
                    if (there) from += (now.at.token0 + (long long)tok) * c.x.q_token + (now.h * G + row - tok * G) * c.x.q_head + ch * 8;
                    cp_async16(at + kQ + (in >> 7) * kTile<D> + swizzled(in & 127, ch), from, there ? 16 : 0);
                }
            }
            if (!wait(kKEmpty + stage, parity)) return false;
            for (int j = t; j < kWideKeys * kChunks; j += kLoaders) {
                const int row = j / kChunks, ch = j - row * kChunks;
                const long long p = place[stage * 128 + row].x;
                cp_async16(at + kK + stage * kTile<D> + swizzled(row, ch), c.cache.k + (p < 0 ? 0 : p + ch * 16), p < 0 ? 0 : 16);
            }
            cp_async_commit();
            if (i > 0) {
                cp_async_wait<1>();
                signal_v(i - 1, last);
            }
            if (!wait(kVEmpty + stage, parity)) return false;
            if (t == 0) s_odd[stage] = 0;
            for (int j = t; j < kWideKeys * kChunks; j += kLoaders) {
                const int row = j / kChunks, ch = j - row * kChunks;
                const longlong2 p = place[stage * 128 + row];
                cp_async16(at + kV + stage * kTile<D> + swizzled(row, ch), c.cache.v + (p.x < 0 ? 0 : p.y + ch * 16), p.x < 0 ? 0 : 16);
            }
            cp_async_commit();
            if (i + 1 < n) {
                load.next(c);
                look_up(load);
            }
            cp_async_wait<1>();
            ptx::fence_proxy_async_smem();
            if (fresh) ptx::mbar_arrive(bars + kQFull * 8);
            ptx::mbar_arrive(bars + (kKFull + stage) * 8);
            fresh = now.tile + 1 == now.tiles;
            if (fresh) ++unit;
            last = now;
            if (i + 1 < n) now.next(c);
            return true;
        };
        bool good = true;                        // (the copying warps meet n + 1 times whether they gave up or not)
        for (int i = 0; i < n; ++i) {
            place[(i & 1) * 128 + t] = found[0];
            if (t + kLoaders < kWideKeys) place[(i & 1) * 128 + t + kLoaders] = found[1];
            ptx::bar_sync(1, kLoaders);
            good = good && copy(i);
        }
        cp_async_wait<0>();
        ptx::bar_sync(1, kLoaders);              // s_odd's zero comes before any one
        if (good) signal_v(n - 1, last);
    } else if (warp == 8) {
        // ---- products
        if (ptx::elect_one()) {
            const uint32_t idesc_s = ptx::idesc_16(Pair<T>::kBf16, 128, 128, false, c.scale < 0.f);
            const uint32_t idesc_o = ptx::idesc_16(Pair<T>::kBf16, 128, D, true, false);
            uint32_t unit = 0, p_count[2] = {0, 0};
            bool fresh = true;
            auto scores = [&](int tile, int stage) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t in = (ks >> 2) * 16384 + (ks & 3) * 32;
                    ptx::mma_f16_ss(tmem + kTmemS + tile * 128, ptx::smem_desc_sw128(at + kQ + tile * kTile<D> + in),
                                    ptx::smem_desc_sw128(at + kK + stage * kTile<D> + in), idesc_s, ks > 0);
                }
                ptx::mma_commit(bars + (kSFull + tile) * 8);
            };
            auto values = [&](int tile, int stage, bool first) {
#pragma unroll
                for (int ks = 0; ks < kWideKeys / 16; ++ks)
                    ptx::mma_f16_ts(tmem + kTmemO + tile * 128, tmem + kTmemS + tile * 128 + ks * 8,
                                    ptx::smem_desc_mn_sw128(at + kV + stage * kTile<D> + ks * 2048, 16384, 1024), idesc_o, !first || ks > 0);
            };
            bool good = true;
            for (int i = 0; i < n && good; ++i) {
                const int stage = i & 1;
                const uint32_t parity = ((uint32_t)i >> 1) & 1;
                const bool two = now.at.rows > kRows, ends = now.tile + 1 == now.tiles || i + 1 == n;
                if (fresh) {
                    good = wait(kQFull, unit & 1) && wait(kKFull + stage, parity);
                    if (!good) break;
                    ptx::tc_fence_after();
                    scores(0, stage);
                    if (two) scores(1, stage);
                    ptx::mma_commit(bars + (kKEmpty + stage) * 8);
                    if (ends) ptx::mma_commit(bars + kQEmpty * 8);
                }
                const int stage1 = (i + 1) & 1;
                const uint32_t parity1 = ((uint32_t)(i + 1) >> 1) & 1;
                const bool first = fresh;
                for (int tile = 0; tile < (two ? 2 : 1); ++tile) {
                    good = wait(kPFull + tile, p_count[tile]++ & 1) && wait(kVFull + stage, parity);
                    if (!good) break;
                    ptx::tc_fence_after();
                    if (!*(volatile int*)&s_odd[stage]) values(tile, stage, first);
                    if (ends) ptx::mma_commit(bars + (kOFull + tile) * 8);
                    if (tile == (two ? 1 : 0)) ptx::mma_commit(bars + (kVEmpty + stage) * 8);
                    if (!ends) {
                        good = wait(kKFull + stage1, parity1);
                        if (!good) break;
                        ptx::tc_fence_after();
                        scores(tile, stage1);
                    }
                }
                if (!good) break;
                if (!ends) {
                    ptx::mma_commit(bars + (kKEmpty + stage1) * 8);
                    if (now.tile + 2 == now.tiles || i + 2 == n) ptx::mma_commit(bars + kQEmpty * 8);
                }
                fresh = ends;
                if (ends) ++unit;
                if (i + 1 < n) now.next(c);
            }
            if (!good) {
                // products in flight end before tensor memory is given back
                ptx::mma_commit(bars + kDrained * 8);
                for (int i = 0; i < 1 << 20 && !ptx::mbar_try_wait(bars + kDrained * 8, 0); ++i) {}
            }
        }
        __syncwarp();
    } else {
        // ---- rows
        const int tile = warp >> 2, in = tile * kRows + (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;                  // lane field of a tensor-memory address: 32 a warp
        const uint32_t s_at = tmem + lanes + kTmemS + tile * 128, o_at = tmem + lanes + kTmemO + tile * 128;
        const float scale = fabsf(c.scale);
        uint32_t s_count = 0, o_count = 0;
        bool fresh = true, whole = now.tile == 0;
        float m = -INFINITY, l = 0.f;
        int lim = 0, least = 0;
        auto all = [](bool ok) { return __all_sync(0xffffffffu, ok) != 0; };     // a warp goes on or leaves as one
        for (int i = 0; i < n; ++i) {
            const bool ends = now.tile + 1 == now.tiles || i + 1 == n;
            if (now.at.rows > tile * kRows) {
                const int row = now.at.row0 + in, tok = row / G;
                if (fresh) {
                    m = -INFINITY;
                    l = 0.f;
                    least = min(now.at.key0 + now.at.keys, now.at.limit + now.at.step * (now.at.row0 / G));
                    lim = in < now.at.rows ? min(now.at.key0 + now.at.keys, now.at.limit + now.at.step * tok) : now.at.key0 + now.at.keys;
                }
                if (!all(wait(kSFull + tile, s_count++ & 1))) break;
                ptx::tc_fence_after();
                const int key0 = now.at.key0 + now.tile * kWideKeys;
                const int seen = lim - key0;                               // of the tile's keys
                const bool masked = __any_sync(0xffffffffu, seen < kWideKeys);
                auto hide = [&](uint32_t (&r)[32], int first) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (first + j >= seen) r[j] = 0xff800000u;
                };
                uint32_t r[2][32];
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                ptx::tmem_ld_32x32b_x32(s_at, r[0]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    ptx::tmem_ld_wait_for(r[q & 1]);
                    if (q < 3) ptx::tmem_ld_32x32b_x32(s_at + 32 * (q + 1), r[(q + 1) & 1]);
                    if (masked) hide(r[q & 1], 32 * q);
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) top[e] = fmaxf(top[e], __uint_as_float(r[q & 1][j + e]));
                    }
                }
                const float highest = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * scale;
                ptx::tmem_ld_32x32b_x32(s_at, r[0]);
                bool odd = false;
                if (__any_sync(0xffffffffu, highest > m + kSlack)) {
                    const float higher = fmaxf(m, highest), alpha = m == higher ? 1.f : ex2(m - higher);
                    m = higher;
                    l *= alpha;
                    if (!fresh) {
#pragma unroll
                        for (int q = 0; q < D / 16; ++q) {
                            uint32_t o[16];
                            ptx::tmem_ld_32x32b_x16(o_at + 16 * q, o);
                            ptx::tmem_ld_wait_for(o);
#pragma unroll
                            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                            ptx::tmem_st_32x32b_x16(o_at + 16 * q, o);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.f : m;
                if (now.at.key0 + (now.tile + 1) * kWideKeys > least) {
                    if (!all(wait(kVFull + (i & 1), ((uint32_t)i >> 1) & 1))) break;
                    odd = *(volatile int*)&s_odd[i & 1] != 0;
                }
                const Two scale2 = two(scale, scale), base2 = two(-base, -base);
                Two sum[2] = {two(0.f, 0.f), two(0.f, 0.f)};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    ptx::tmem_ld_wait_for(r[q & 1]);
                    if (q < 3) ptx::tmem_ld_32x32b_x32(s_at + 32 * (q + 1), r[(q + 1) & 1]);
                    if (masked) hide(r[q & 1], 32 * q);
                    uint32_t p[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 x = apart(fma2(two(__uint_as_float(r[q & 1][2 * j]), __uint_as_float(r[q & 1][2 * j + 1])), scale2, base2));
                        const float2 w = make_float2(ex2(x.x), ex2(x.y));
                        sum[j & 1] = sum[j & 1] + two(w.x, w.y);
                        p[j] = Pair<T>::pack(w.x, w.y);
                    }
                    if (!odd) ptx::tmem_st_32x32b_x16(s_at + 16 * q, p);
                }
                const float2 total = apart(sum[0] + sum[1]);
                l += total.x + total.y;
                if (odd) {
                    // (rare) the product without the keys that a row does not see, key by key
                    const char* v_at = smem + kV + (i & 1) * kTile<D>;
                    for (int q = 0; q < D / 16; ++q) {
                        uint32_t o[16];
                        ptx::tmem_ld_32x32b_x16(o_at + 16 * q, o);
                        ptx::tmem_ld_wait_for(o);
                        if (fresh) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) o[j] = 0u;
                        }
                        for (int k0 = 0; k0 < kWideKeys; k0 += 16) {
                            uint32_t s[16];
                            ptx::tmem_ld_32x32b_x16(s_at + k0, s);
                            ptx::tmem_ld_wait_for(s);
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                if (k0 + k >= seen) continue;
                                const float w = Pair<T>::rounded(ex2(fmaf(__uint_as_float(s[k]), scale, -base)));
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    const T* v = reinterpret_cast<const T*>(v_at + swizzled(k0 + k, 2 * q + (j >> 3))) + (j & 7);
                                    o[j] = __float_as_uint(__uint_as_float(o[j]) + w * to_float(*v));
                                }
                            }
                        }
                        ptx::tmem_st_32x32b_x16(o_at + 16 * q, o);
                    }
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before();
                ptx::mbar_arrive(bars + (kPFull + tile) * 8);
                if (ends) {
                    if (!all(wait(kOFull + tile, o_count++ & 1))) break;
                    ptx::tc_fence_after();
                    const long long unit = list.steps[now.b] + (long long)now.h * now.tiles;
                    const bool direct = whole && now.tile + 1 == now.tiles && now.b >= own && c.plan.share[now.at.request].prefix < 0;
                    const bool there = in < now.at.rows;
                    const int head = now.h * G + row - tok * G;
                    T* to = static_cast<T*>(c.x.out) + (there ? (now.at.token0 + (long long)tok) * c.x.out_token + head * c.x.out_head : 0);
                    const long long piece = direct ? 0 : piece_row<true>(c, now.b, now.at, now.h, blockIdx.x, (int)(unit / each)) + in;
                    const float f = l > 0.f ? 1.f / l : l;
#pragma unroll
                    for (int q = 0; q < D / 16; ++q) {
                        uint32_t o[16];
                        ptx::tmem_ld_32x32b_x16(o_at + 16 * q, o);
                        ptx::tmem_ld_wait_for(o);
                        if (there && direct) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] = Pair<T>::pack(__uint_as_float(o[2 * j]) * f, __uint_as_float(o[2 * j + 1]) * f);
                            *reinterpret_cast<uint4*>(to + 16 * q) = make_uint4(w[0], w[1], w[2], w[3]);
                            *reinterpret_cast<uint4*>(to + 16 * q + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                        } else if (there) {
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                *reinterpret_cast<uint4*>(c.pieces.o + piece * D + 16 * q + j) = make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                        }
                    }
                    if (there) {
                        if (direct) c.x.lse[(now.at.token0 + (long long)tok) * c.x.lse_token + head] = (m + log2f(l)) * 0.6931471805599453f;
                        else c.pieces.ml[piece] = make_float2(m, l);
                    }
                    ptx::tc_fence_before();
                }
            }
            fresh = ends;
            if (ends) whole = true;
            if (i + 1 < n) now.next(c);
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 8) ptx::tmem_dealloc(tmem, kTmemColumns);
}

template <typename T, int D> bool launch(const Call& c, cudaStream_t st) {
    if (cudaFuncSetAttribute(wide_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared<D>) != cudaSuccess) return false;
    return launch_early(wide_kernel<T, D>, c.plan.wide.ctas, kThreads, 1, kShared<D>, st, c);
}
template <typename T> bool launch_width(const Call& c, int width, cudaStream_t st) {
    switch (width) {
        case 64: return launch<T, 64>(c, st);
        case 80: return launch<T, 80>(c, st);
        case 96: return launch<T, 96>(c, st);
        default: return launch<T, 128>(c, st);
    }
}

}  // namespace

bool ardiff::launch_wide(const Call& c, int32_t dtype, int width, cudaStream_t st) {
    return dtype == ARDIFF_F16 ? launch_width<__half>(c, width, st) : launch_width<__nv_bfloat16>(c, width, st);
}
