// Attention over pages for blocks of many query rows, on the tensor cores: a CTA takes 256 rows (two tiles of 128) through the
// tiles of 128 keys that are its share of the line of steps.
//
//   S_t = Q_t K^T          tcgen05, 128 x 128 in tensor memory, tile t = 0, 1
//   P_t = 2^(S_t scale - m_t), m_t a base of every row, by its running maximum (f16: 2^7 below it)
//   O_t = O_t + P_t V      tcgen05, P_t from tensor memory (16-bit, over S_t's first columns), V as it lies in the cache (keys are rows: N-major)
//
// While one tile's rows go through the exponentials the tensor cores work on the other's products, so both pipes stay busy: per step 4 x 128 x 128
// x width multiply-adds (2048 cycles at 128) and 2 x 128 x 128 exponentials (2048 cycles of 16 a clock).
// The base only moves when the maximum would grow by more than 8 (a factor 256 that P and the sums hold easily): then O is rescaled in
// tensor memory, which is rare; the product that last wrote O is done by then, since its successor S_t is issued after it.
// Measured: prompts of 841 to 1024 tokens of 32 heads over 15000 shared ones, 4 requests, width 128, 1.0 TFLOP: 0.93 ms alone, 1.03 PFLOP/s, 1.1 ms back to
// back at the clock that the power cap leaves. A step takes some 4000 cycles, 3300 of them in the issue of products that wait for
// one another and for shared memory (both operands of S come from there: 128 bytes a clock, all that it gives).
//
// Warps: 0-3 and 4-7 the rows of tile 0 and 1 (a thread a row), 8 issues products, 9 copies keys, 10 values (the rows' warps their queries). Pages of a multiple of 8 tokens
// come by TMA, in boxes of the largest power of two of tokens that divides a page (a lane looks up and copies a box). Others come by asynchronous
// 16-byte copies, 64 a lane and tile, into the same 128-byte-swizzled layout; their places warp 11 looks up, up to four steps ahead. Those
// copies tell of themselves when they have landed, and the issuing warp puts the fence between the proxies.
#include <cuda.h>
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

constexpr int kThreads = 12 * 32;               // three warps a quarter of the SM: 168 registers each
constexpr int kPlaces = 4;                       // steps whose places are known
constexpr int kRows = 128;                       // of a tile
constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemColumns = 512;

template <int D> constexpr int kSub = (D + 63) / 64;                       // blocks of 64 values of a row
template <int D> constexpr int kTile = kSub<D> * 128 * 128;                // bytes of 128 rows
template <int D> constexpr int kShared = 1024 + 6 * kTile<D> + kPlaces * kWideKeys * 16;

enum Bar { kQFull, kKFull = kQFull + 2, kKEmpty = kKFull + 2, kVFull = kKEmpty + 2, kVEmpty = kVFull + 2, kSFull = kVEmpty + 2, kPFull = kSFull + 2,
           kOFull = kPFull + 2, kVLanded = kOFull + 2, kDrained = kVLanded + 2, kPlaceFull, kPlaceEmpty = kPlaceFull + kPlaces, kBars = kPlaceEmpty + kPlaces };

// The two caches as TMA takes them; tokens 0: not that way.
struct Boxes {
    CUtensorMap k, v;
    int tokens;
};

// 2^x of two numbers, x <= 15, by the nearest whole number and a polynomial for the rest f, |f| <= 1/2 (fitted to 2^f for the least relative
// error, 2.1e-7 in fp32): a quarter of the exponentials go this way, through pipes that have room, so that the special-function unit's 16 a
// clock are not the bound. Numbers below -127 count as that, and 2^-127 comes out as 2^-149 (the lowest exponent has no leading one), which is 0 in 16
// bits: a key that is not seen adds nothing, however large its value. NaN and infinities are not taken here.
__device__ __forceinline__ float2 exp2_by_products(float2 x) {
    const Two y = two(fmaxf(x.x, -127.f), fmaxf(x.y, -127.f));
    const Two t = y + two(12582912.f, 12582912.f);             // 1.5 2^23: the whole number in the low bits
    const Two f = fma2(t + two(-12582912.f, -12582912.f), two(-1.f, -1.f), y);
    Two v = fma2(two(1.32764725e-3f, 1.32764725e-3f), f, two(9.67554096e-3f, 9.67554096e-3f));
    v = fma2(v, f, two(5.55071309e-2f, 5.55071309e-2f));
    v = fma2(v, f, two(0.240221202f, 0.240221202f));
    v = fma2(v, f, two(0.693146944f, 0.693146944f));
    v = fma2(v, f, two(1.00000012f, 1.00000012f));
    const float2 a = apart(v), n = apart(t);
    return make_float2(__int_as_float(__float_as_int(n.x) * (1 << 23) + __float_as_int(a.x)),
                       __int_as_float(__float_as_int(n.y) * (1 << 23) + __float_as_int(a.y)));
}

__device__ __forceinline__ float max3(float a, float b, float c) {                  // NaN if one is
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// A row's 128 scores from tensor memory: weights 2^(s scale - base), packed; their sum; the highest score (NaN if one is). A weight of a score that is
// -inf is 2^-149 at the most, which no sum of any other weight notices; what is NaN is the caller's to see by the highest score.
template <typename T> __device__ __forceinline__ void weights(uint32_t s_at, float scale, float base, uint32_t (&p)[64], float& sum, float& top) {
    const Two scale2 = two(scale, scale), base2 = two(-base, -base);
    uint32_t r[2][32];
    float high[2] = {-INFINITY, -INFINITY};
    Two part[2] = {two(0.f, 0.f), two(0.f, 0.f)};
    ptx::tmem_ld_32x32b_x32(s_at, r[0]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        ptx::tmem_ld_wait_for(r[q & 1]);
        if (q < 3) ptx::tmem_ld_32x32b_x32(s_at + 32 * (q + 1), r[(q + 1) & 1]);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float a = __uint_as_float(r[q & 1][2 * j]), b = __uint_as_float(r[q & 1][2 * j + 1]);
            high[j & 1] = max3(high[j & 1], a, b);
            const float2 x = apart(fma2(two(a, b), scale2, base2));
            const float2 w = (j & 3) == 3 ? exp2_by_products(x) : make_float2(ex2(x.x), ex2(x.y));
            part[j & 1] = part[j & 1] + two(w.x, w.y);
            p[16 * q + j] = Pair<T>::pack(w.x, w.y);
        }
    }
    const float2 all = apart(part[0] + part[1]);
    sum = all.x + all.y;
    top = max3(high[0], high[1], high[1]);
}

// The highest of a row's scores `hidden` <= key < seen (NaN if one is); the others become -inf, in tensor memory too where `hide` says so.
__device__ __forceinline__ float highest_seen(uint32_t s_at, int hidden, int seen, bool hide) {
    float high = -INFINITY;
#pragma unroll 1
    for (int q = 0; q < 128; q += 16) {
        uint32_t r[16];
        ptx::tmem_ld_32x32b_x16(s_at + q, r);
        ptx::tmem_ld_wait_for(r);
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            r[j] = q + j < seen && q + j >= hidden ? r[j] : 0xff800000u;
            r[j + 1] = q + j + 1 < seen && q + j + 1 >= hidden ? r[j + 1] : 0xff800000u;
            high = max3(high, __uint_as_float(r[j]), __uint_as_float(r[j + 1]));
        }
        if (hide) ptx::tmem_st_32x32b_x16(s_at + q, r);
    }
    if (hide) ptx::tmem_st_wait();
    return high;
}

// Whether some row of the block does not see all keys of a tile: keys from the first row's limit on, and those in front of the block's first key.
__device__ __forceinline__ bool some_unseen(const Block& b, int tile, const Divide& by_G) {
    const int key0 = b.key0 + tile * kWideKeys;
    return key0 < b.low || key0 + kWideKeys > min(b.key0 + b.keys, b.limit + b.step * (int)by_G.quotient(b.row0));
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) wide_kernel(const Call c, const __grid_constant__ Boxes boxes) {
    extern __shared__ char raw[];
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kQ = 0, kK = 2 * kTile<D>, kV = 4 * kTile<D>;
    // offsets of keys and of values: [2][steps][128]; odd: there is none
    long long* place = reinterpret_cast<long long*>(smem + 6 * kTile<D>);
    __shared__ __align__(8) uint64_t s_bar[kBars];
    __shared__ uint32_t s_tmem;
    __shared__ int s_stop;
    __shared__ int s_whole[kPlaces];             // whether all 128 keys of the step have a place
    __shared__ int s_odd[2];                     // values of the stage that are not finite, where some row does not see them
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bars = ptx::smem_u32(s_bar), at = ptx::smem_u32(smem);
    // (barriers and tensor memory do not wait for the kernels before)
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            int count = 1;
            if (i == kKFull || i == kKFull + 1 || i == kVFull || i == kVFull + 1 || (i >= kPlaceFull && i < kPlaceEmpty)) count = boxes.tokens ? 1 : 32;
            else if (i == kQFull || i == kQFull + 1 || i == kPFull || i == kPFull + 1) count = 128;
            else if (i >= kPlaceEmpty) count = 2;
            ptx::mbar_init(bars + i * 8, count);
        }
        s_stop = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 8) {
        ptx::tmem_alloc(ptx::smem_u32(&s_tmem), kTmemColumns);
        ptx::tmem_relinquish();
    }
    ardiff::begin_kernel();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = s_tmem;
    const List& list = c.plan.wide;
    const long long steps = list.head->steps, each = steps_each<true>(steps, list.workers), begin = each * blockIdx.x;
    const int n = (int)max(0ll, min(steps, begin + each) - begin), own = list.head->own, G = c.x.G;
    const Waits wait{bars, &s_stop, c.status};
    Cursor now;
    if (n > 0) now.start(c, find_last(list.steps, list.head->blocks, begin), begin);

    if (n == 0) {
        // nothing is left for this CTA
    } else if (warp == 11) {
        // ---- places
        for (int i = 0; i < n && !boxes.tokens; ++i) {
            const int slot = i % kPlaces;
            longlong2 found[4];
            bool whole = true;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                found[u] = place_of(c, now, u * 32 + lane);
                whole &= found[u].x >= 0;
            }
            whole = __all_sync(0xffffffffu, whole);
            if (!__all_sync(0xffffffffu, wait(kPlaceEmpty + slot, ((i / kPlaces) & 1) ^ 1))) break;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                place[slot * kWideKeys + u * 32 + lane] = found[u].x < 0 ? 1 : found[u].x;
                place[(kPlaces + slot) * kWideKeys + u * 32 + lane] = found[u].x < 0 ? 1 : found[u].y;
            }
            if (lane == 0) s_whole[slot] = whole;
            ptx::mbar_arrive(bars + (kPlaceFull + slot) * 8);
            if (i + 1 < n) now.next(c);
        }
    } else if (warp >= 9 && boxes.tokens) {
        // ---- keys or values, by boxes
        const bool v = warp == 10;
        const int full = v ? kVFull : kKFull, empty = v ? kVEmpty : kKEmpty, tokens = boxes.tokens;
        const CUtensorMap* map = v ? &boxes.v : &boxes.k;
        const uint32_t to = at + (v ? kV : kK) + lane * tokens * 128;
        Cursor load = now;                 // of the box that is looked up next
        struct Box { int id, row, head; } next;
        auto look_up = [&]() {
            const int in = load.tile * kWideKeys + lane * tokens, key = load.at.key0 + in;
            next.id = -1;
            next.head = load.h;
            if (lane * tokens < kWideKeys && in < load.at.keys) {
                const int pg = c.cache.by_page.quotient(key);
                next.row = key - pg * c.cache.page;
                next.id = c.cache.table[(long long)(pg < load.at.split ? load.at.front : load.at.request) * c.cache.width + pg];
                if (next.id < 0 || next.id >= c.cache.pages) {
                    *c.status = ARDIFF_ERR_SHAPE;
                    next.id = -1;
                }
            }
        };
        look_up();
        uint32_t landed[2] = {0, 0};
        bool good = true;
        int i = 0;
        for (; i < n; ++i) {
            const int stage = i & 1;
            const Box box = next;
            good = __all_sync(0xffffffffu, wait(empty + stage, ((i >> 1) & 1) ^ 1));
            if (!good) break;
            const bool zone = v && some_unseen(now.at, now.tile, c.x.by_G);
            const uint32_t bar = bars + ((zone ? kVLanded : full) + stage) * 8;
            const uint32_t there = __ballot_sync(0xffffffffu, box.id >= 0);
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar, __popc(there) * tokens * 128 * kSub<D>);
            __syncwarp();
            if (box.id >= 0) {
#pragma unroll
                for (int b = 0; b < kSub<D>; ++b)
                    ptx::tma_load_4d(to + stage * kTile<D> + b * 16384, map, bar, b * 64, box.row, box.head, box.id);
            }
            if (i + 1 < n) {
                load.next(c);
                look_up();
            }
            if (zone) {
                // keys that some row of the block does not see must not reach it as 0 times a value that is not finite; those behind the
                // last one, whatever they are, become zeros
                good = __all_sync(0xffffffffu, wait(kVLanded + stage, landed[stage]++ & 1));
                if (!good) {
                    for (int j = 0; j < 1 << 20 && !ptx::mbar_try_wait(bars + (kVLanded + stage) * 8, (landed[stage] - 1) & 1); ++j) {}
                    break;
                }
                const int left = now.at.keys - now.tile * kWideKeys;
                bool odd = false;
                for (int j = lane; j < kWideKeys * 8 * kSub<D>; j += 32) {
                    const int row = j & 127;
                    uint4* w = reinterpret_cast<uint4*>(smem + kV + stage * kTile<D> + swizzled(row, j >> 7));
                    if (row >= left) *w = make_uint4(0u, 0u, 0u, 0u);
                    else odd |= Pair<T>::not_finite(w->x) || Pair<T>::not_finite(w->y) || Pair<T>::not_finite(w->z) || Pair<T>::not_finite(w->w);
                }
                odd = __any_sync(0xffffffffu, odd);
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    s_odd[stage] = odd;
                    ptx::mbar_arrive(bars + (kVFull + stage) * 8);
                }
            }
            if (i + 1 < n) now.next(c);
        }
        if (!good) wait_for_copies(bars, full, i, 2);
    } else if (warp >= 9) {
        // ---- keys or values, by 16 bytes
        const bool v = warp == 10;
        const int full = v ? kVFull : kKFull, empty = v ? kVEmpty : kKEmpty;
        constexpr int kLanes = D / 8 <= 8 ? 8 : 16, kAtOnce = 32 / kLanes, kPeriod = 8 / kAtOnce;    // lanes a row, rows at once, before they repeat
        const int ch = lane % kLanes, row0 = lane / kLanes;
        const bool mine = ch < D / 8;
        const char* from = (v ? c.cache.v : c.cache.k) + ch * 16;
        uint32_t to[kPeriod];
#pragma unroll
        for (int u = 0; u < kPeriod; ++u) to[u] = at + (v ? kV : kK) + swizzled(row0 + u * kAtOnce, ch);
        for (int i = 0; i < n; ++i) {
            const int slot = i % kPlaces, stage = i & 1;
            if (!__all_sync(0xffffffffu, wait(kPlaceFull + slot, (i / kPlaces) & 1) && wait(empty + stage, ((i >> 1) & 1) ^ 1))) break;
            const long long* p = place + (v ? kPlaces + slot : slot) * kWideKeys + row0;
            const uint32_t in = stage * kTile<D>;
            // (offsets of 16 rows first: nothing is read past a copy that has been issued)
            const bool whole = s_whole[slot];
#pragma unroll 1
            for (int j = 0; j < kWideKeys / kAtOnce; j += 16) {
                long long o[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) o[u] = p[(j + u) * kAtOnce];
                const uint32_t base = in + (j / kPeriod) * 1024;
                if (whole) {
#pragma unroll
                    for (int u = 0; u < 16; ++u)
                        if (mine) cp_async16(to[u % kPeriod] + base + (u / kPeriod) * 1024, from + o[u], 16);
                } else {
#pragma unroll
                    for (int u = 0; u < 16; ++u)
                        if (mine) cp_async16(to[u % kPeriod] + base + (u / kPeriod) * 1024, from + (o[u] & 1 ? 0 : o[u]), o[u] & 1 ? 0 : 16);
                }
            }
            if (v && some_unseen(now.at, now.tile, c.x.by_G)) {
                // keys that some row of the block does not see must not reach it as 0 times a value that is not finite
                cp_async_commit();
                cp_async_wait<0>();
                __syncwarp();
                bool odd = false;
                for (int row = row0; mine && row < kWideKeys; row += kAtOnce) {
                    const uint4 w = *reinterpret_cast<const uint4*>(smem + kV + in + swizzled(row, ch));
                    odd |= Pair<T>::not_finite(w.x) || Pair<T>::not_finite(w.y) || Pair<T>::not_finite(w.z) || Pair<T>::not_finite(w.w);
                }
                odd = __any_sync(0xffffffffu, odd);
                if (lane == 0) s_odd[stage] = odd;
                ptx::mbar_arrive(bars + (full + stage) * 8);
            } else {
                cp_async_arrive(bars + (full + stage) * 8);
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bars + (kPlaceEmpty + slot) * 8);
            if (i + 1 < n) now.next(c);
        }
        cp_async_commit();
        cp_async_wait<0>();
    } else if (warp == 8) {
        // ---- products. The whole warp goes through the steps, so that addresses stay in uniform registers; one lane issues.
        const uint32_t idesc_s = ptx::idesc_16(Pair<T>::kBf16, 128, 128, false, c.scale < 0.f);
        const uint32_t idesc_o = ptx::idesc_16(Pair<T>::kBf16, 128, D, true, false);
        const uint64_t q_desc = ptx::smem_desc_sw128(at + kQ), k_desc = ptx::smem_desc_sw128(at + kK);
        const uint64_t v_desc = ptx::smem_desc_mn_sw128(at + kV, 16384, 1024);
        uint32_t units[2] = {0, 0}, p_count[2] = {0, 0};
        bool fresh = true, good = true;
        auto all = [](bool ok) { return __all_sync(0xffffffffu, ok) != 0; };
        auto commit = [&](int bar) {
            if (ptx::elect_one()) ptx::mma_commit(bars + bar * 8);
            __syncwarp();
        };
        // (a descriptor counts in 16 bytes)
        auto scores = [&](int tile, int stage) {
            const uint64_t a = q_desc + tile * (kTile<D> / 16), b = k_desc + stage * (kTile<D> / 16);
            const uint32_t to = tmem + kTmemS + tile * 128;
            if (ptx::elect_one()) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t in = (ks >> 2) * 1024 + (ks & 3) * 2;
                    ptx::mma_f16_ss(to, a + in, b + in, idesc_s, ks > 0);
                }
                ptx::mma_commit(bars + (kSFull + tile) * 8);
            }
            __syncwarp();
        };
        auto values = [&](int tile, int stage, bool first) {
            const uint64_t b = v_desc + stage * (kTile<D> / 16);
            const uint32_t to = tmem + kTmemO + tile * 128, p = tmem + kTmemS + tile * 128;
            if (ptx::elect_one()) {
#pragma unroll
                for (int ks = 0; ks < kWideKeys / 16; ++ks) ptx::mma_f16_ts(to, p + ks * 8, b + ks * 128, idesc_o, !first || ks > 0);
            }
            __syncwarp();
        };
        for (int i = 0; i < n; ++i) {
            const int stage = i & 1;
            const uint32_t parity = ((uint32_t)i >> 1) & 1;
            const bool two = now.at.rows > kRows, ends = now.tile + 1 == now.tiles || i + 1 == n;
            if (fresh) {
                for (int tile = 0; tile < (two ? 2 : 1) && good; ++tile) {
                    good = all(wait(kQFull + tile, units[tile] & 1) && wait(kKFull + stage, parity));
                    ++units[tile];
                    if (!good) break;
                    ptx::fence_proxy_async_smem();
                    ptx::tc_fence_after();
                    scores(tile, stage);
                }
                if (!good) break;
                commit(kKEmpty + stage);
            }
            const int stage1 = (i + 1) & 1;
            const uint32_t parity1 = ((uint32_t)(i + 1) >> 1) & 1;
            const bool zone = some_unseen(now.at, now.tile, c.x.by_G);
#pragma unroll
            for (int tile = 0; tile < 2; ++tile) {
                if (tile == 1 && !two) break;
                if (tile == 0) {
                    good = all(wait(kVFull + stage, parity));
                    if (!boxes.tokens) ptx::fence_proxy_async_smem();          // (TMA writes where products read)
                }
                good = good && all(wait(kPFull + tile, p_count[tile] & 1));
                ++p_count[tile];
                if (!good) break;
                ptx::tc_fence_after();
                if (!zone || !*(volatile int*)&s_odd[stage]) values(tile, stage, fresh);
                if (ends) commit(kOFull + tile);
                if (tile == (two ? 1 : 0)) commit(kVEmpty + stage);
                if (!ends) {
                    if (tile == 0) {
                        good = all(wait(kKFull + stage1, parity1));
                        if (!good) break;
                        if (!boxes.tokens) ptx::fence_proxy_async_smem();
                        ptx::tc_fence_after();
                    }
                    scores(tile, stage1);
                }
            }
            if (!good) break;
            if (!ends) commit(kKEmpty + stage1);
            fresh = ends;
            if (i + 1 < n) now.next(c);
        }
        if (!good) {
            // products in flight end before tensor memory is given back
            commit(kDrained);
            for (int i = 0; i < 1 << 20 && !ptx::mbar_try_wait(bars + kDrained * 8, 0); ++i) {}
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
        float m = -INFINITY, l = 0.f, recent = 0.f;                        // sums of weights, of the last 32 tiles apart: roundings add up less
        int lim = 0;
        auto all = [](bool ok) { return __all_sync(0xffffffffu, ok) != 0; };     // a warp goes on or leaves as one
        for (int i = 0; i < n; ++i) {
            const bool ends = now.tile + 1 == now.tiles || i + 1 == n;
            if (now.at.rows > tile * kRows) {
                const int row = now.at.row0 + in, tok = row / G;
                if (fresh) {
                    // the warp's rows of queries (the last unit's products are done: its results have been read)
                    constexpr int kLanes = D / 8 <= 8 ? 8 : 16;
                    const T* base = static_cast<const T*>(c.x.q) + (long long)now.at.token0 * c.x.q_token + (long long)now.h * G * c.x.q_head + (lane % kLanes) * 8;
#pragma unroll 4
                    for (int u = lane / kLanes; u < 32; u += 32 / kLanes) {
                        const int j = in - lane + u;
                        const unsigned r = now.at.row0 + j, t = c.x.by_G.quotient(r);
                        const T* from = base + (j < now.at.rows ? t * c.x.q_token + (r - t * G) * c.x.q_head : 0);
                        if (lane % kLanes < D / 8) cp_async16(at + kQ + tile * kTile<D> + swizzled(j & 127, lane % kLanes), from, j < now.at.rows ? 16 : 0);
                    }
                    cp_async_arrive(bars + (kQFull + tile) * 8);
                    m = -INFINITY;
                    l = recent = 0.f;
                    lim = in < now.at.rows ? min(now.at.key0 + now.at.keys, now.at.limit + now.at.step * tok) : now.at.key0 + now.at.keys;
                }
                if (!all(wait(kSFull + tile, s_count++ & 1))) break;
                ptx::tc_fence_after();
                const int key0 = now.at.key0 + now.tile * kWideKeys;
                const int seen = lim - key0, hidden = now.at.low - key0;   // of the tile's keys
                const bool masked = __any_sync(0xffffffffu, seen < kWideKeys || hidden > 0);
                // Weights by the maximum so far, in the hope that it holds, and kept in registers until it is known to: S is still there for another
                // try with a higher one. A unit's first tile, and tiles that some row does not see all of, are looked through before.
                uint32_t p[64];
                float top = 0.f;
                bool look = fresh || masked;
                if (look) top = highest_seen(s_at, hidden, seen, masked);
                for (;;) {
                    const float highest = top * scale;
                    if (look && __any_sync(0xffffffffu, highest > m + Pair<T>::kSlack || (fresh && highest > m))) {
                        const float higher = fmaxf(m, highest - Pair<T>::kLift), alpha = m == higher ? 1.f : ex2(m - higher);
                        m = higher;
                        l *= alpha;
                        recent *= alpha;
                        if (!fresh) {
#pragma unroll 1
                            for (int q = 0; q < D; q += 16) {
                                uint32_t o[16];
                                ptx::tmem_ld_32x32b_x16(o_at + q, o);
                                ptx::tmem_ld_wait_for(o);
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                                ptx::tmem_st_32x32b_x16(o_at + q, o);
                            }
                            ptx::tmem_st_wait();               // (the product key by key reads them again)
                        }
                    }
                    float sum;
                    weights<T>(s_at, scale, m == -INFINITY ? 0.f : m, p, sum, top);
                    // NaN and +inf have no weights: the row's results are NaN
                    const bool lost = !(top * scale < INFINITY) && !(top == -INFINITY);
                    if (look || __all_sync(0xffffffffu, lost || top * scale <= m + Pair<T>::kSlack || top == -INFINITY)) {
                        recent += lost ? NAN : sum;
                        break;
                    }
                    look = true;
                }
                bool odd = false;
                if (some_unseen(now.at, now.tile, c.x.by_G)) {
                    if (!all(wait(kVFull + (i & 1), ((uint32_t)i >> 1) & 1))) break;
                    odd = *(volatile int*)&s_odd[i & 1] != 0;
                }
                if (!odd) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t part[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) part[j] = p[16 * q + j];
                        ptx::tmem_st_32x32b_x16(s_at + 16 * q, part);
                    }
                }
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
                                if (k0 + k >= seen || k0 + k < hidden) continue;
                                const float w = Pair<T>::rounded(ex2(fmaf(__uint_as_float(s[k]), scale, m == -INFINITY ? 0.f : -m)));
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
                if (ends || (i & 31) == 31) {
                    l += recent;
                    recent = 0.f;
                }
                if (ends) {
                    if (!all(wait(kOFull + tile, o_count++ & 1))) break;
                    ptx::tc_fence_after();
                    const long long unit = now.at.first_step + (long long)now.h * now.tiles;
                    const bool direct = whole && now.tile + 1 == now.tiles && now.b >= own && c.plan.share[now.at.request].prefix < 0;
                    const bool there = in < now.at.rows;
                    const int head = now.h * G + row - tok * G;
                    T* to = static_cast<T*>(c.x.out) + (there ? (now.at.token0 + (long long)tok) * c.x.out_token + head * c.x.out_head : 0);
                    const long long piece = direct ? 0 : piece_row<true>(c, list.head->rows_before, now.at, now.h, blockIdx.x, quotient_of(unit, each));
                    if (m == -INFINITY) l = l == l ? 0.f : l;                // no key was seen
                    const float f = l > 0.f ? 1.f / l : l;
#pragma unroll 1
                    for (int q = 0; q < D; q += 16) {
                        uint32_t o[16];
                        ptx::tmem_ld_32x32b_x16(o_at + q, o);
                        ptx::tmem_ld_wait_for(o);
                        if (there && direct) {
                            uint32_t w[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] = Pair<T>::pack(__uint_as_float(o[2 * j]) * f, __uint_as_float(o[2 * j + 1]) * f);
                            *reinterpret_cast<uint4*>(to + q) = make_uint4(w[0], w[1], w[2], w[3]);
                            *reinterpret_cast<uint4*>(to + q + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                        } else if (there) {
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                *reinterpret_cast<uint4*>(piece_values(c, piece, D, now.at.rows, in, q + j)) = make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                        }
                    }
                    if (there) {
                        if (direct) c.x.lse[(now.at.token0 + (long long)tok) * c.x.lse_token + head] = (m + log2f(l)) * 0.6931471805599453f;
                        else c.pieces.ml[piece + in] = make_float2(m, l);
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

template <typename T, int D> bool launch(const Call& c, const Boxes& boxes, cudaStream_t st) {
    static std::atomic<uint64_t> ready{0};
    return shared_memory(wide_kernel<T, D>, kShared<D>, ready) &&
           launch_early(wide_kernel<T, D>, c.plan.wide.workers, kThreads, 1, kShared<D>, st, c, boxes);
}
template <typename T> bool launch_width(const Call& c, int width, const Boxes& boxes, cudaStream_t st) {
    switch (width) {
        case 64: return launch<T, 64>(c, boxes, st);
        case 80: return launch<T, 80>(c, boxes, st);
        case 96: return launch<T, 96>(c, boxes, st);
        default: return launch<T, 128>(c, boxes, st);
    }
}

}  // namespace

namespace {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encoder() {
    static std::atomic<EncodeTiled> known{nullptr};
    EncodeTiled f = known.load(std::memory_order_relaxed);
    if (!f) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
        f = reinterpret_cast<EncodeTiled>(p);
        known.store(f, std::memory_order_relaxed);
    }
    return f;
}

}  // namespace

int ardiff::box_tokens(int page) {
    int tokens = 1;
    while (tokens < 128 && page % (2 * tokens) == 0) tokens *= 2;
    return tokens >= 8 ? tokens : 0;
}

bool ardiff::describe(CUtensorMap* map, const char* base, bool bf16, int width, int tokens, const Pages& p, uint32_t token, uint32_t head, uint32_t page) {
    // (a stride of 0 where there is more than one: the same rows under several names)
    if (p.pages < 1 || (!token && p.page > 1) || (!head && p.heads > 1) || (!page && p.pages > 1)) return false;
    const EncodeTiled f = encoder();
    if (!f) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)width, (cuuint64_t)p.page, (cuuint64_t)p.heads, (cuuint64_t)p.pages};
    const cuuint64_t strides[3] = {16 * (cuuint64_t)(token ? token : 1), 16 * (cuuint64_t)(head ? head : 1), 16 * (cuuint64_t)(page ? page : 1)};
    const cuuint32_t box[4] = {64, (cuuint32_t)tokens, 1, 1}, ones[4] = {1, 1, 1, 1};
    return f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<char*>(base), dims, strides, box, ones,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool ardiff::describe_queries(CUtensorMap* map, const Queries& x, bool bf16, int width, int rows) {
    if (x.tokens < 1 || rows % x.G || x.q_token < 0 || x.q_head < 0 || (x.q_token | x.q_head) >> 38) return false;
    if ((!x.q_token && x.tokens > 1) || (!x.q_head && x.heads > 1)) return false;
    const EncodeTiled f = encoder();
    if (!f) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)x.heads, (cuuint64_t)x.tokens};
    const cuuint64_t strides[2] = {x.heads > 1 ? 2 * (cuuint64_t)x.q_head : 16, x.tokens > 1 ? 2 * (cuuint64_t)x.q_token : 16};
    const cuuint32_t box[3] = {64, (cuuint32_t)x.G, (cuuint32_t)(rows / x.G)}, ones[3] = {1, 1, 1};
    return f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(x.q), dims, strides, box, ones,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool ardiff::launch_wide(const Call& c, int32_t dtype, int width, cudaStream_t st) {
    Boxes boxes;
    memset(&boxes, 0, sizeof(boxes));
    const int tokens = box_tokens(c.cache.page);
    const bool bf16 = dtype == ARDIFF_BF16;
    if (tokens && describe(&boxes.k, c.cache.k, bf16, width, tokens, c.cache, c.cache.k_token, c.cache.k_head, c.cache.k_page) &&
        describe(&boxes.v, c.cache.v, bf16, width, tokens, c.cache, c.cache.v_token, c.cache.v_head, c.cache.v_page))
        boxes.tokens = tokens;
    return bf16 ? launch_width<__nv_bfloat16>(c, width, boxes, st) : launch_width<__half>(c, width, boxes, st);
}
