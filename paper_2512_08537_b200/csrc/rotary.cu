// Rotary positions with several axes:
//   ardiff_rotary           queries and keys turned by their positions (forward);
//   ardiff_rotary_backward  their gradients turned back (a rotation's transpose is the rotation by the negative angle);
//   ardiff_rotary_append    queries turned, keys turned and written with their values into the slots of a paged cache.
//
// Token t turns pair i of every head by angle(t, i) = position[axis_i][t] * freq_i. The angle belongs to the token and the pair alone, so a
// CTA works out cosine and sine of its tokens once, into shared memory, and uses them for all heads. A far position has an angle of
// 10^5 turns and more, of which fp32 would keep no fraction; so turns are formed and reduced in fp64 (three operations a token and pair,
// against 2 x 40 heads that use them) and only the fraction, at most half a turn, goes on in fp32. Rotations are fp32, rounded once.
//
// Bound by memory: every value is read once and written once. Two kernels:
//   rows_kernel    rows on 16-byte boundaries, of up to 512 bytes: a lane has one 16-byte chunk of a row, two to four rows a warp side by side, and the
//                  cosines of that chunk in registers for all heads of the token; the other halves of pairs come by shuffles, whatever the number
//                  of pairs (a window of two lanes' chunks, shifted). Four rows a lane under way, three CTAs an SM (two or four: 148 and 153 us
//                  instead of 122 for the gradients of 32768 tokens of 40 heads of 128 f16 values, 671 MB, which is 5.5 TB/s). Halves that are no
//                  whole chunks cost 16 shuffles and shifts where others take four: 16384 tokens of 48 heads of 80 values, 35 pairs:
//                  252 MB in 71 us, 3.6 TB/s.
//   rotary_kernel  all others: an item is a chunk of VEC pairs (two loads and two stores) or of VEC values that no pair covers; VEC is the
//                  widest that the alignment of rows, halves and pointers allows.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/ardiff.h"
#include "common.cuh"
#include "launch.cuh"
#include "rows.cuh"

namespace {

using namespace ardiff;

constexpr int kThreads = 256;
constexpr int kItems = 4;                        // items of a thread under way together
constexpr float kStill = 2.f;                    // in the place of a cosine: a pair of no axis stands still, whatever its values are (0 times an infinity would be NaN)

// n / d for n * d < 2^32, by the number 2^32 / d rounded up (here n < 2^20, since a CTA has at most 2048 items or one token's, and d <= 1024)
struct Divide {
    uint32_t d, m;
};
Divide divide_by(uint32_t d) { return Divide{d, d > 1 ? (uint32_t)((((uint64_t)1 << 32) + d - 1) / d) : 0u}; }
__device__ __forceinline__ uint32_t quotient(uint32_t n, Divide by) { return by.d > 1 ? __umulhi(n, by.m) : n; }

struct Side {                                    // queries, keys or values: strides in values
    const void* in;
    void* out;
    long long in_token, in_head, out_token, out_head;
    int heads;
};

struct Rotary {
    Side q, k, v;                                // v: copied, only with a cache
    const int32_t* position;                     // [axes][n], rows position_ld apart
    long long position_ld;
    const float* freq;
    const int32_t* axis;
    const int64_t* slot;                         // the cache's: place of every token
    const int32_t* count;
    long long n, slots;
    long long k_page, v_page;                    // strides of the cache's pages; out_token is that of tokens in a page
    int page, axes, width, pairs, tokens;        // tokens: of a CTA
    Divide by_chunks, by_copies, by_q, by_k, by_token;   // chunks of a row, of a value's row; heads; pairs
    float sign;
};

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Chunk { T x[VEC]; };

// With a cache, keys and values of token t go to page slot / page, place slot % page.
template <typename T, int VEC, bool kNeighbours, bool kAppend>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const Rotary a) {
    extern __shared__ char smem[];
    float2* cs = reinterpret_cast<float2*>(smem);                                   // [tokens][pairs]
    long long* k_at = reinterpret_cast<long long*>(cs + (size_t)a.tokens * a.pairs);    // [tokens], -1: not written
    long long* v_at = k_at + a.tokens;
    ardiff::begin_kernel();
    const long long t0 = (long long)blockIdx.x * a.tokens;
    long long n = a.n;
    if (kAppend && a.count) n = min(n, (long long)*a.count);
    const int tokens = (int)max(0ll, min((long long)a.tokens, n - t0));
    if (tokens == 0) return;

    for (uint32_t j = threadIdx.x; j < (uint32_t)(tokens * a.pairs); j += kThreads) {
        const uint32_t t = quotient(j, a.by_token), i = j - t * a.pairs;
        const int axis = a.axis ? a.axis[i] : 0;
        float s = 0.f, c = kStill;
        if (axis >= 0 && axis < a.axes) {
            double turns = (double)a.position[axis * a.position_ld + t0 + t] * ((double)a.freq[i] * 0.15915494309189533577);
            turns -= rint(turns);
            sincospif(2.f * (float)turns, &s, &c);
        }
        cs[j] = make_float2(c, s * a.sign);
    }
    if (kAppend) {
        for (int t = threadIdx.x; t < tokens; t += kThreads) {
            const long long slot = a.slot[t0 + t];
            long long k = -1, v = -1;
            if (slot >= 0 && slot < a.slots) {
                const long long pg = slot / a.page, in = slot - pg * a.page;
                k = pg * a.k_page + in * a.k.out_token;
                v = pg * a.v_page + in * a.v.out_token;
            }
            k_at[t] = k;
            v_at[t] = v;
        }
    }
    __syncthreads();

    using C = Chunk<T, VEC>;
    const uint32_t pair_chunks = a.pairs / VEC, chunks = a.by_chunks.d;             // chunks of a row of queries or keys
    const uint32_t queries = tokens * a.q.heads * chunks, turned = queries + tokens * a.k.heads * chunks;
    const uint32_t items = turned + (kAppend ? tokens * a.k.heads * a.by_copies.d : 0u);
    for (uint32_t base = threadIdx.x; base < items; base += kThreads * kItems) {
        C lo[kItems], hi[kItems];
        T* to[kItems];
        int32_t table[kItems];                   // place of the cosines of an item that turns; -1: copied
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const uint32_t item = base + u * kThreads;
            to[u] = nullptr;
            table[u] = -1;
            if (item >= items) continue;
            // all tokens' queries, then all tokens' keys, then, with a cache, all tokens' values
            const bool is_q = item < queries, is_v = kAppend && item >= turned;
            const uint32_t at = is_q ? item : is_v ? item - turned : item - queries;
            uint32_t row = quotient(at, is_v ? a.by_copies : a.by_chunks);
            const uint32_t c = at - row * (is_v ? a.by_copies.d : chunks);
            const uint32_t t = quotient(row, is_q ? a.by_q : a.by_k);
            row -= t * (is_q ? a.by_q.d : a.by_k.d);
            const T* in = static_cast<const T*>(is_q ? a.q.in : is_v ? a.v.in : a.k.in) +
                          (t0 + t) * (is_q ? a.q.in_token : is_v ? a.v.in_token : a.k.in_token) +
                          (long long)row * (is_q ? a.q.in_head : is_v ? a.v.in_head : a.k.in_head);
            T* out = static_cast<T*>(is_q ? a.q.out : is_v ? a.v.out : a.k.out) +
                     (long long)row * (is_q ? a.q.out_head : is_v ? a.v.out_head : a.k.out_head);
            if (kAppend && !is_q) {
                const long long place = is_v ? v_at[t] : k_at[t];
                if (place < 0) continue;
                out += place;
            } else {
                out += (t0 + t) * (is_q ? a.q.out_token : a.k.out_token);
            }
            if (!is_v && c < pair_chunks) {
                const int first = kNeighbours ? 2 * c * VEC : c * VEC;
                lo[u] = *reinterpret_cast<const C*>(in + first);
                hi[u] = *reinterpret_cast<const C*>(in + (kNeighbours ? first + VEC : first + a.pairs));
                to[u] = out + first;
                table[u] = t * a.pairs + c * VEC;
            } else {
                const int first = is_v ? c * VEC : 2 * a.pairs + (c - pair_chunks) * VEC;
                lo[u] = *reinterpret_cast<const C*>(in + first);
                to[u] = out + first;
            }
        }
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            if (!to[u]) continue;
            if (table[u] >= 0) {
                const float2* p = cs + table[u];
                T v[2 * VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float2 w = p[e];
                    T &a0 = kNeighbours ? (2 * e < VEC ? lo[u].x[2 * e < VEC ? 2 * e : 0] : hi[u].x[2 * e >= VEC ? 2 * e - VEC : 0]) : lo[u].x[e];
                    T &b0 = kNeighbours ? (2 * e + 1 < VEC ? lo[u].x[2 * e + 1 < VEC ? 2 * e + 1 : 0] : hi[u].x[2 * e + 1 >= VEC ? 2 * e + 1 - VEC : 0]) : hi[u].x[e];
                    const float x = ardiff::to_float(a0), y = ardiff::to_float(b0);
                    v[2 * e] = w.x == kStill ? a0 : ardiff::from_float<T>(x * w.x - y * w.y);
                    v[2 * e + 1] = w.x == kStill ? b0 : ardiff::from_float<T>(x * w.y + y * w.x);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    lo[u].x[e] = kNeighbours ? v[e] : v[2 * e];
                    hi[u].x[e] = kNeighbours ? v[VEC + e] : v[2 * e + 1];
                }
                *reinterpret_cast<C*>(to[u] + (kNeighbours ? VEC : a.pairs)) = hi[u];
            }
            *reinterpret_cast<C*>(to[u]) = lo[u];
        }
    }
}

// ---- rows on 16-byte boundaries ----
constexpr int kUnroll = 4;                       // rows of a lane under way together
constexpr int kWarps = kThreads / 32;

struct Words {
    uint32_t w[4];
};
__device__ __forceinline__ Words shuffle(const uint4& x, int lane) {
    return Words{{__shfl_sync(0xffffffffu, x.x, lane), __shfl_sync(0xffffffffu, x.y, lane), __shfl_sync(0xffffffffu, x.z, lane), __shfl_sync(0xffffffffu, x.w, lane)}};
}

// The 16 bytes from 2 s (s < 8) bytes into the chunk of lane `lane` on, the next lane's behind them.
__device__ __forceinline__ Words window(const uint4& x, int lane, int s) {
    const Words a = shuffle(x, lane), b = shuffle(x, lane + 1);
    uint32_t w[8] = {a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3]};
    if (s & 4) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (s & 2) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (s & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    return Words{{w[0], w[1], w[2], w[3]}};
}

__device__ __forceinline__ uint4 to_chunk(const Words& w) { return make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]); }

// kNeighbours: pairs 2 i, 2 i + 1. Else kAligned: the number of pairs fills whole chunks, so that a chunk's other halves are one other chunk.
// `split` warps share a token.
template <typename T, bool kNeighbours, bool kAligned, bool kAppend>
__global__ void __launch_bounds__(kThreads, 3) rows_kernel(const Rotary a, int lanes, int split) {
    constexpr int N = Piece<T>::N;               // values of a chunk
    extern __shared__ char smem[];
    float2* cs = reinterpret_cast<float2*>(smem);                                   // [tokens][pairs]
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long t0 = (long long)blockIdx.x * a.tokens;
    long long n = a.n;
    if (kAppend && a.count) n = min(n, (long long)*a.count);
    const int tokens = (int)max(0ll, min((long long)a.tokens, n - t0));
    if (tokens == 0) return;
    const int side = 32 / lanes, c = lane % lanes, sub = lane / lanes;              // rows side by side; chunk; which row
    const bool mine = sub < side;
    const int mt = warp / split;                 // of the CTA's tokens
    const long long t = t0 + mt;
    const int rows = a.q.heads + a.k.heads, step = side * split;
    const T* q_in = static_cast<const T*>(a.q.in) + t * a.q.in_token + c * N;
    const T* k_in = static_cast<const T*>(a.k.in) + t * a.k.in_token + c * N;
    T* q_out = static_cast<T*>(a.q.out) + t * a.q.out_token + c * N;
    T* k_out = static_cast<T*>(a.k.out) + c * N;
    bool keys = true;                            // to be written
    const bool there = mt < tokens;
    if (kAppend) {
        const long long slot = there ? a.slot[t] : -1;
        keys = slot >= 0 && slot < a.slots;
        if (keys) {
            const long long pg = slot / a.page, in = slot - pg * a.page;
            k_out += pg * a.k_page + in * a.k.out_token;
            // values: copied as they are
            const T* v_in = static_cast<const T*>(a.v.in) + t * a.v.in_token + c * N;
            T* v_out = static_cast<T*>(a.v.out) + pg * a.v_page + in * a.v.out_token + c * N;
            for (int r = (warp % split) * side + sub; mine && r < a.v.heads; r += kUnroll * step) {
                uint4 x[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    if (r + u * step < a.v.heads) x[u] = *reinterpret_cast<const uint4*>(v_in + (long long)(r + u * step) * a.v.in_head);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    if (r + u * step < a.v.heads) *reinterpret_cast<uint4*>(v_out + (long long)(r + u * step) * a.v.out_head) = x[u];
            }
        }
    } else {
        k_out += t * a.k.out_token;
    }
    auto load = [&](int r) -> uint4 {
        if (!mine || !there || r >= rows) return make_uint4(0u, 0u, 0u, 0u);
        return *reinterpret_cast<const uint4*>(r < a.q.heads ? q_in + (long long)r * a.q.in_head : k_in + (long long)(r - a.q.heads) * a.k.in_head);
    };
    uint4 x[kUnroll];
    const int first = (warp % split) * side + sub;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) x[u] = load(first + u * step);

    for (uint32_t j = tid; j < (uint32_t)(tokens * a.pairs); j += kThreads) {
        const uint32_t tok = quotient(j, a.by_token), i = j - tok * a.pairs;
        const int axis = a.axis ? a.axis[i] : 0;
        float s = 0.f, co = kStill;
        if (axis >= 0 && axis < a.axes) {
            double turns = (double)a.position[axis * a.position_ld + t0 + tok] * ((double)a.freq[i] * 0.15915494309189533577);
            turns -= rint(turns);
            sincospif(2.f * (float)turns, &s, &co);
        }
        cs[j] = make_float2(co, s * a.sign);
    }
    __syncthreads();
    if (!there) return;

    // out = x cos + y sin', y the pair's other value: masks say where it comes from a later place (up) or an earlier one (down), if at all
    float co[N], si[N];
    uint32_t up[4] = {0u, 0u, 0u, 0u}, down[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int j = c * N + e;
        const bool early = kNeighbours ? !(e & 1) : j < a.pairs;
        const float2 w = j < 2 * a.pairs && mine ? cs[mt * a.pairs + (kNeighbours ? j >> 1 : early ? j : j - a.pairs)] : make_float2(kStill, 0.f);
        const bool pair = w.x != kStill;
        co[e] = pair ? w.x : 1.f;
        si[e] = !pair ? -0.f : early ? -w.y : w.y;               // (x - 0 is x, whatever x is)
        const uint32_t bits = N == 4 ? 0xffffffffu : e & 1 ? 0xffff0000u : 0xffffu;
        if (pair && early) up[e * 4 / N] |= bits;
        if (pair && !early) down[e * 4 / N] |= bits;
    }
    const int s = a.pairs % N, chunks = a.pairs / N, row_lane = lane - c;
    const int half = c < chunks ? lane + chunks : lane - chunks;                    // (aligned) the other half's lane
    for (int r0 = first; r0 - sub < rows; r0 += kUnroll * step) {
        uint4 next[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) next[u] = load(r0 + (kUnroll + u) * step);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            Words y;
            if (kNeighbours) {
                y = N == 4 ? Words{{x[u].y, x[u].x, x[u].w, x[u].z}}
                           : Words{{__funnelshift_r(x[u].x, x[u].x, 16), __funnelshift_r(x[u].y, x[u].y, 16), __funnelshift_r(x[u].z, x[u].z, 16), __funnelshift_r(x[u].w, x[u].w, 16)}};
#pragma unroll
                for (int i = 0; i < 4; ++i) y.w[i] &= up[i] | down[i];
            } else if (kAligned) {
                y = shuffle(x[u], half);
#pragma unroll
                for (int i = 0; i < 4; ++i) y.w[i] &= up[i] | down[i];
            } else {
                const int shift = N == 4 ? 2 * s : s;
                const Words later = window(x[u], row_lane + c + chunks, shift), earlier = window(x[u], row_lane + c - chunks - 1, 8 - shift);
#pragma unroll
                for (int i = 0; i < 4; ++i) y.w[i] = (later.w[i] & up[i]) | (earlier.w[i] & down[i]);
            }
            const int r = r0 + u * step;
            if (!mine || r >= rows || (kAppend && r >= a.q.heads && !keys)) continue;
            float xs[N], ys[N];
            unpack(x[u], xs, T());
            unpack(to_chunk(y), ys, T());
#pragma unroll
            for (int e = 0; e < N; ++e) xs[e] = xs[e] * co[e] + ys[e] * si[e];
            *reinterpret_cast<uint4*>(r < a.q.heads ? q_out + (long long)r * a.q.out_head : k_out + (long long)(r - a.q.heads) * a.k.out_head) = pack(xs, T());
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) x[u] = next[u];
    }
}

template <typename T, bool kNeighbours, bool kAligned> bool launch_rows(const Rotary& a, bool append, unsigned grid, size_t smem, int lanes, int split, cudaStream_t st) {
    return append ? ardiff::launch_early(rows_kernel<T, kNeighbours, kAligned, true>, grid, kThreads, 1, smem, st, a, lanes, split)
                  : ardiff::launch_early(rows_kernel<T, kNeighbours, kAligned, false>, grid, kThreads, 1, smem, st, a, lanes, split);
}
template <typename T> bool launch_rows_of(const Rotary& a, bool neighbours, bool append, unsigned grid, size_t smem, int lanes, int split, cudaStream_t st) {
    if (neighbours) return launch_rows<T, true, true>(a, append, grid, smem, lanes, split, st);
    return a.pairs % Piece<T>::N ? launch_rows<T, false, false>(a, append, grid, smem, lanes, split, st)
                                 : launch_rows<T, false, true>(a, append, grid, smem, lanes, split, st);
}

template <typename T, int VEC> bool launch(const Rotary& a, bool neighbours, bool append, unsigned grid, size_t smem, cudaStream_t st) {
    if (append) {
        return neighbours ? ardiff::launch_early(rotary_kernel<T, VEC, true, true>, grid, kThreads, 1, smem, st, a)
                          : ardiff::launch_early(rotary_kernel<T, VEC, false, true>, grid, kThreads, 1, smem, st, a);
    }
    return neighbours ? ardiff::launch_early(rotary_kernel<T, VEC, true, false>, grid, kThreads, 1, smem, st, a)
                      : ardiff::launch_early(rotary_kernel<T, VEC, false, false>, grid, kThreads, 1, smem, st, a);
}

template <typename T> bool launch_type(const Rotary& a, int vec, bool neighbours, bool append, unsigned grid, size_t smem, cudaStream_t st) {
    if (sizeof(T) == 2 && vec == 8) return launch<T, sizeof(T) == 2 ? 8 : 4>(a, neighbours, append, grid, smem, st);
    if (vec >= 4) return launch<T, 4>(a, neighbours, append, grid, smem, st);
    if (vec >= 2) return launch<T, 2>(a, neighbours, append, grid, smem, st);
    return launch<T, 1>(a, neighbours, append, grid, smem, st);
}

// The strides and the pointer of rows, as far as their alignment goes: what a power of two that divides all of them divides.
uint64_t places(const void* p, int size, long long token, long long head) {
    return (uint64_t)reinterpret_cast<uintptr_t>(p) / size | (uint64_t)token | (uint64_t)head;
}

int rotary(Rotary& a, int32_t dtype, int32_t neighbours, bool append, cudaStream_t st) {
    const int size = ardiff::value_size(dtype);
    if (a.n < 0 || a.n >= (int64_t)1 << 31 || a.q.heads < 0 || a.k.heads < 0 || a.q.heads > ARDIFF_ROTARY_MAX_HEADS || a.k.heads > ARDIFF_ROTARY_MAX_HEADS || a.width < 1 ||
        a.width > ARDIFF_ROTARY_MAX_WIDTH || a.pairs < 0 || 2 * a.pairs > a.width || a.axes < 1 || a.axes > 65535 || a.position_ld < 0)
        return ARDIFF_ERR_SHAPE;
    if (!size) return ARDIFF_ERR_UNSUPPORTED;
    ardiff::set_launch_count(0);
    if (a.n == 0 || (a.q.heads == 0 && a.k.heads == 0)) return ARDIFF_OK;
    if (!a.position || (a.pairs > 0 && !a.freq) || (append && !a.slot)) return ARDIFF_ERR_NULL;
    uint64_t bits = (uint64_t)a.width | (uint64_t)a.pairs, bits_rows = 0;    // what a power of two divides where it divides all
    const Side* sides[3] = {&a.q, &a.k, &a.v};
    for (int i = 0; i < (append ? 3 : 2); ++i) {
        const Side& s = *sides[i];
        if (s.heads == 0) continue;
        if (!s.in || !s.out) return ARDIFF_ERR_NULL;
        if ((reinterpret_cast<uintptr_t>(s.in) | reinterpret_cast<uintptr_t>(s.out)) & (size - 1)) return ARDIFF_ERR_ALIGN;
        if (s.in == s.out && ((a.n > 1 && s.in_token != s.out_token) || (s.heads > 1 && s.in_head != s.out_head))) return ARDIFF_ERR_UNSUPPORTED;
        bits_rows |= places(s.in, size, s.in_token, s.heads > 1 ? s.in_head : 0) | places(s.out, size, s.out_token, s.heads > 1 ? s.out_head : 0);
    }
    if (append) bits_rows |= (uint64_t)a.k_page | (uint64_t)a.v_page;
    bits |= bits_rows;
    int vec = 16 / size;
    while (vec > 1 && (bits & (vec - 1))) vec >>= 1;
    a.by_token = divide_by(a.pairs > 0 ? a.pairs : 1);
    // rows of whole 16-byte chunks (neighbouring pairs never cross one)
    const int lanes = a.width * size / 16;
    if (lanes >= 1 && lanes <= 32 && !((bits_rows * size | (uint64_t)a.width * size) & 15)) {
        // a warp a token; few tokens are shared by more, so that a warp's rows are few as well
        int split = 1;
        while (split < kWarps && a.n * split < 2368) split *= 2;
        a.tokens = kWarps / split;
        const unsigned grid = (unsigned)((a.n + a.tokens - 1) / a.tokens);
        const size_t smem = (size_t)a.tokens * a.pairs * sizeof(float2);
        const bool ok = dtype == ARDIFF_F32 ? launch_rows_of<float>(a, neighbours != 0, append, grid, smem, lanes, split, st)
                      : dtype == ARDIFF_F16 ? launch_rows_of<__half>(a, neighbours != 0, append, grid, smem, lanes, split, st)
                                            : launch_rows_of<__nv_bfloat16>(a, neighbours != 0, append, grid, smem, lanes, split, st);
        ardiff::set_launch_count(1);
        return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
    }
    const uint32_t chunks = a.pairs / vec + (a.width - 2 * a.pairs) / vec;
    const long long copies = append ? (long long)a.k.heads * (a.width / vec) : 0;
    const long long of_token = (long long)(a.q.heads + a.k.heads) * chunks + copies;
    // About 2048 items a CTA: two rounds of its threads, so that loads of one are under way while the other computes; few tokens spread
    // over as many CTAs as there are.
    long long tokens = 2048 / of_token;
    if (tokens > a.n / 296) tokens = a.n / 296;
    a.tokens = (int)(tokens < 1 ? 1 : tokens > 16 ? 16 : tokens);
    a.by_chunks = divide_by(chunks);
    a.by_q = divide_by(a.q.heads > 0 ? a.q.heads : 1);
    a.by_k = divide_by(a.k.heads > 0 ? a.k.heads : 1);
    a.by_copies = divide_by((uint32_t)(a.width / vec));
    const size_t smem = (size_t)a.tokens * (a.pairs * sizeof(float2) + 16);
    const unsigned grid = (unsigned)((a.n + a.tokens - 1) / a.tokens);
    const bool ok = dtype == ARDIFF_F32 ? launch_type<float>(a, vec, neighbours != 0, append, grid, smem, st)
                  : dtype == ARDIFF_F16 ? launch_type<__half>(a, vec, neighbours != 0, append, grid, smem, st)
                                        : launch_type<__nv_bfloat16>(a, vec, neighbours != 0, append, grid, smem, st);
    ardiff::set_launch_count(1);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}

// What both structures say, of queries, keys and angles.
template <typename C> Rotary arguments(const C& c, float sign) {
    Rotary a;
    memset(&a, 0, sizeof(a));
    a.q.in = c.q; a.q.in_token = c.q_token; a.q.in_head = c.q_head; a.q.heads = (int)c.q_heads;
    a.q.out = c.q_out; a.q.out_token = c.q_out_token; a.q.out_head = c.q_out_head;
    a.k.in = c.k; a.k.in_token = c.k_token; a.k.in_head = c.k_head; a.k.heads = (int)c.k_heads;
    a.n = c.n; a.width = (int)c.width; a.position = c.position; a.position_ld = c.position_ld; a.axes = (int)c.axes; a.freq = c.freq; a.axis = c.axis;
    a.pairs = (int)c.pairs; a.sign = sign;
    return a;
}

int turned(const ardiff_rotary_call* call, float sign, void* stream) {
    if (!call) return ARDIFF_ERR_NULL;
    const ardiff_rotary_call& c = *call;
    if (!ardiff::in_32_bits({c.q_heads, c.k_heads, c.dtype, c.width, c.axes, c.pairs, c.neighbours})) return ARDIFF_ERR_SHAPE;
    Rotary a = arguments(c, sign);
    a.k.out = c.k_out; a.k.out_token = c.k_out_token; a.k.out_head = c.k_out_head;
    return rotary(a, (int32_t)c.dtype, (int32_t)c.neighbours, false, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" int ardiff_rotary(const ardiff_rotary_call* call, void* stream) { return turned(call, 1.f, stream); }

extern "C" int ardiff_rotary_backward(const ardiff_rotary_call* call, void* stream) { return turned(call, -1.f, stream); }

extern "C" int ardiff_rotary_append(const ardiff_rotary_append_call* call, void* stream) {
    if (!call) return ARDIFF_ERR_NULL;
    const ardiff_rotary_append_call& c = *call;
    if (!ardiff::in_32_bits({c.q_heads, c.k_heads, c.dtype, c.width, c.axes, c.pairs, c.neighbours, c.pages, c.page})) return ARDIFF_ERR_SHAPE;
    if (c.pages < 0 || c.page < 1) return ARDIFF_ERR_SHAPE;
    Rotary a = arguments(c, 1.f);
    a.k.out = c.k_cache; a.k.out_token = c.k_cache_token; a.k.out_head = c.k_cache_head; a.k_page = c.k_cache_page;
    a.v.in = c.v; a.v.in_token = c.v_token; a.v.in_head = c.v_head; a.v.heads = a.k.heads;
    a.v.out = c.v_cache; a.v.out_token = c.v_cache_token; a.v.out_head = c.v_cache_head; a.v_page = c.v_cache_page;
    a.slot = c.slot; a.count = c.count; a.page = (int)c.page; a.slots = (long long)c.pages * c.page;
    return rotary(a, (int32_t)c.dtype, (int32_t)c.neighbours, true, static_cast<cudaStream_t>(stream));
}
