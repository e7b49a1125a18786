// The next token of every row of logits: temperature, top-k, top-p and min-p, then one draw with a given uniform number.
//
// With w_i = exp((x_i - max) / T), the kept tokens are a prefix of the order (logit descending, index ascending): the first
// top_k, of these the shortest prefix whose mass reaches top_p of theirs, of these the ones with w >= min_p. The token is the
// first kept one, in order of index, at which the sum of w passes u times the kept sum.
//
// Which token that is hangs on borders between sums, and a flat row of a large vocabulary has its borders closer together than
// fp32 sums are exact: all weights that decide are formed and summed in fp64 (polynomial of degree 9 after splitting off the
// integer part, 4e-14 relative), in an order that depends on sizes only.
//
// A row belongs to a cluster of one to eight CTAs and is read once, into shared memory, a contiguous part a CTA, of that a
// contiguous segment a warp. What is done with it depends on its settings:
//   T = 0                the largest logit's lowest index
//   top-k, small nuclei  "list": the threads' own largest logits (512 a CTA) bound the k-th largest from below (at least k logits
//                        lie above the k-th largest of them), and the mass above a bound as well; the few logits above the bound
//                        go to the first CTA, which sorts them and does the rest alone
//   no prefix            the segments' sums, then the one segment in which the draw ends
//   large k or nuclei    "search" for the prefix's last element: histograms narrow a range of logits until it holds few, an exact
//                        pass sums what lies above it and lists what lies in it, and the sums say whether the range was right
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/ardiff.h"
#include "common.cuh"
#include "rows.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2 * kThreads;      // of a histogram, two a thread
constexpr int kList = 2 * kThreads;      // logits that the first CTA sorts, two a thread
constexpr int kMaxParts = 8;
constexpr double kFar = -100.0;          // weights below 2^kFar count as nothing: all of a row's add up to less than 2^-75 of its sum

struct Args {
    const void* x;
    int64_t ld;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* token;
    float* logprob;
    int32_t V, parts;
};

struct Shared {
    float thread_max[kThreads];
    float warp_max[kWarps];
    int warp_first[kWarps];
    double seg[2][kWarps];               // sums of the warps' segments; two, so that one may still be read by another CTA
    double scan[kWarps];
    unsigned uscan[kWarps];
    double total, before;
    int owner;                           // segment in which a sum passes its target, of all CTAs'
    int found, last;
    float cta_max;
    int cta_first;
    unsigned count;                      // entries of `list` (of the first CTA)
    unsigned kmin, kmax;
    int pick_first, pick_last;
    unsigned pick_before, pick_after;
    int verdict;
    unsigned cut_key;
    int cut_index;
    double mass_above, mass_in;
    unsigned long long list[kList];
    union {
        unsigned hist[kBins];
        double w[kList];
    };
};

// logits in their order as whole numbers; both zeros are one
__device__ __forceinline__ unsigned key_of(float x) {
    const unsigned b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// Kept: everything before this element in the order (descending, lowest index first), and it.
struct Cut {
    unsigned key;
    int index;
};
__device__ __forceinline__ Cut no_cut() { return Cut{0u, INT_MAX}; }

__device__ __forceinline__ float max_nan(float a, float b) {       // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 2^y of y = d a, d <= 0: y = k + r, |r| <= 1/2, 2^r = 1 + r P(r), P of degree 8 by interpolation at the Chebyshev nodes (3.7e-14
// relative; exactly 1 at 0). 0 below 2^kFar, also for d = -inf.
__device__ __forceinline__ double pow2(double d, double a) {
    constexpr double kRound = 6755399441055744.0;                  // 1.5 2^52: adding it leaves the nearest integer
    const double t = fma(d, a, kRound);
    const double k = t - kRound;
    const double r = fma(d, a, -k);
    double p = 1.0203121063391729e-07;
    p = fma(p, r, 1.3255224878668817e-06);
    p = fma(p, r, 1.525268684626772e-05);
    p = fma(p, r, 0.00015403455852453838);
    p = fma(p, r, 0.0013333558179043112);
    p = fma(p, r, 0.009618129159402558);
    p = fma(p, r, 0.055504108664760424);
    p = fma(p, r, 0.2402265069581299);
    p = fma(p, r, 0.6931471805599453);
    p = fma(p, r, 1.0);
    const double v = __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
    return k >= kFar ? v : 0.0;
}
// u = 0 asks for the first kept token with any weight at all, down to fp64's smallest.
__device__ __noinline__ double pow2_far(double d, double a) { return d == -INFINITY ? 0.0 : exp2(d * a); }

template <typename T>
struct Part {                            // this CTA's part of its row
    static constexpr int N = ardiff::Piece<T>::N;
    const uint4* piece;                  // in shared memory; -inf in the places outside the row
    int pieces, segment;                 // pieces, and pieces a warp
    int first;                           // index of the part's first value in the row (negative in front of the row)
    int rank, parts, V;
    float m;
    double a;                            // log2(e) / T
    float a32;                           // the same in fp32, finite
    bool tiny;                           // u = 0
    Shared* s;

    __device__ __forceinline__ double weight(float x) const { return pow2((double)x - (double)m, a); }
    __device__ __forceinline__ double weight_drawn(float x) const {        // of a draw that may end at any weight above 0
        const double w = weight(x);
        return tiny && w == 0.0 ? pow2_far((double)x - (double)m, a) : w;
    }
    __device__ __forceinline__ void sync() const {
        if (parts > 1) cg::this_cluster().sync(); else __syncthreads();
    }
    template <typename U> __device__ __forceinline__ U* at(U* p, int r) const {
        return parts > 1 ? cg::this_cluster().map_shared_rank(p, r) : p;
    }
    // f(value, index) for every value of the calling warp's segment, lanes taking pieces in turn
    template <typename F> __device__ __forceinline__ void each(F&& f) const {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const int end = min(pieces, (warp + 1) * segment);
        for (int p = warp * segment + lane; p < end; p += 32) {
            float v[N];
            ardiff::unpack(piece[p], v, T());
#pragma unroll
            for (int i = 0; i < N; ++i) f(v[i], first + p * N + i);
        }
    }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Exclusive sums over the CTA's threads; *total: of all.
__device__ __forceinline__ double cta_scan(Shared& s, double v, double* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
    }
    double ex = __shfl_up_sync(0xffffffffu, inc, 1);
    if (lane == 0) ex = 0.0;
    __syncthreads();
    if (lane == 31) s.scan[warp] = inc;
    __syncthreads();
    double before = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) before = all;
        all += s.scan[w];
    }
    *total = all;
    return before + ex;
}
__device__ __forceinline__ unsigned cta_scan(Shared& s, unsigned v, unsigned* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
    }
    __syncthreads();
    if (lane == 31) s.uscan[warp] = inc;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) before = all;
        all += s.uscan[w];
    }
    *total = all;
    return before + inc - v;
}

// Sums of f(value, index) over the segments, in s.seg[buf]; afterwards every CTA knows their sum (returned) and, with target >= 0, the
// first segment at whose end the running sum is above the target (the last one with anything, if none is: s.owner) and the
// sum before it (s.before). Two calls in a row use different buffers.
template <typename T, typename F>
__device__ __forceinline__ double sum_segments(const Part<T>& a, int buf, double share, F&& f) {
    Shared& s = *a.s;
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int end = min(a.pieces, (warp + 1) * a.segment);
    for (int p = warp * a.segment + lane; p < end; p += 32) {
        float v[Part<T>::N];
        ardiff::unpack(a.piece[p], v, T());
#pragma unroll
        for (int i = 0; i < Part<T>::N; ++i) acc[i & 3] += f(v[i], a.first + p * Part<T>::N + i);
    }
    const double mine = warp_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
    if (lane == 0) s.seg[buf][warp] = mine;
    a.sync();
    if (warp == 0) {
        constexpr int kPer = kMaxParts * kWarps / 32;
        double v[kPer], own = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int g = lane * kPer + i;
            v[i] = g < a.parts * kWarps ? *a.at(&s.seg[buf][g % kWarps], g / kWarps) : 0.0;
            own += v[i];
        }
        double inc = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double up = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += up;
        }
        const double all = __shfl_sync(0xffffffffu, inc, 31);
        const double target = share * all;
        double before = __shfl_up_sync(0xffffffffu, inc, 1);
        if (lane == 0) before = 0.0;
        int first = INT_MAX, last = -1;
        double first_before = 0.0, last_before = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const double after = before + v[i];
            if (v[i] > 0.0) {
                last = lane * kPer + i;
                last_before = before;
                if (after > target && first == INT_MAX) {
                    first = last;
                    first_before = before;
                }
            }
            before = after;
        }
        const int f_all = __reduce_min_sync(0xffffffffu, first), l_all = __reduce_max_sync(0xffffffffu, last);
        const int pick = f_all != INT_MAX ? f_all : l_all;
        if (first == pick || (f_all == INT_MAX && last == pick && last >= 0)) {
            s.owner = pick;
            s.before = first == pick ? first_before : last_before;
        }
        if (lane == 0) {
            if (pick < 0) s.owner = 0, s.before = 0.0;
            s.total = all;
        }
    }
    __syncthreads();
    return s.total;
}

// In the CTA that owns segment s.owner: the index of the first value at which the running sum of f passes share * total (the last value
// with anything, if none does). All threads of that CTA call it.
template <typename T, typename F>
__device__ __forceinline__ int locate(const Part<T>& a, double target, F&& f) {
    Shared& s = *a.s;
    const int g = s.owner % kWarps;
    const int begin = g * a.segment, end = min(a.pieces, begin + a.segment);
    double carry = s.before;
    if (threadIdx.x == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    for (int p0 = begin; p0 < end; p0 += kThreads) {
        const int p = p0 + threadIdx.x;
        double w[Part<T>::N], own = 0.0;
        const int e = a.first + p * Part<T>::N;
        if (p < end) {
            float v[Part<T>::N];
            ardiff::unpack(a.piece[p], v, T());
#pragma unroll
            for (int i = 0; i < Part<T>::N; ++i) {
                w[i] = f(v[i], e + i);
                own += w[i];
            }
        }
        double total;
        double run = carry + cta_scan(s, own, &total);             // (its barriers put s.found's start before its use)
        if (p < end && own > 0.0) {
#pragma unroll
            for (int i = 0; i < Part<T>::N; ++i) {
                run += w[i];
                if (w[i] > 0.0) {
                    atomicMax(&s.last, e + i);
                    if (run > target) atomicMin(&s.found, e + i);
                }
            }
        }
        carry += total;
        __syncthreads();
        if (s.found != INT_MAX) break;
    }
    return s.found != INT_MAX ? s.found : s.last;
}

// Sorts s.list[0 .. n), ascending, n <= kList; entries behind are overwritten.
__device__ __forceinline__ void sort_list(Shared& s, int n) {
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kThreads) s.list[i] = ~0ull;
    __syncthreads();
    const int pairs = size / 2;
    const bool one_warp = pairs <= 32;
    if (!one_warp || threadIdx.x < 32) {
        for (int span = 2; span <= size; span *= 2) {
            for (int step = span / 2; step > 0; step /= 2) {
                const int i = threadIdx.x;
                if (i < pairs) {
                    const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
                    const unsigned long long x = s.list[lo], y = s.list[hi];
                    if ((x > y) == ((lo & span) == 0)) {
                        s.list[lo] = y;
                        s.list[hi] = x;
                    }
                }
                if (one_warp) __syncwarp(); else __syncthreads();
            }
        }
    }
    __syncthreads();
}

__device__ __forceinline__ unsigned long long entry(float x, int index) {
    return (unsigned long long)(~key_of(x)) << 32 | (unsigned)index;
}
__device__ __forceinline__ float entry_value(unsigned long long e) { return value_of(~(unsigned)(e >> 32)); }

struct Settings {
    float T, p, mp, u;
    int k;
    bool use_k, use_p, use_m;
};

__device__ __forceinline__ void answer(const Args& a, int64_t row, int token, float logprob) {
    a.token[row] = token;
    a.logprob[row] = logprob;
}

// The first CTA alone: s.list[0 .. n) holds every logit that may be kept (and no other CTA's memory is needed). `whole`: the mass that
// top-p is a share of, where no top-k makes it the list's own.
template <typename T>
__device__ __forceinline__ void finish_list(const Args& args, int64_t row, const Part<T>& a, const Settings& o, int n, double whole,
                                            bool all_listed) {
    Shared& s = *a.s;
    sort_list(s, n);
    const int j0 = 2 * threadIdx.x, j1 = j0 + 1;
    const int limit = o.use_k ? min(o.k, n) : n;
    unsigned long long e0 = ~0ull, e1 = ~0ull;
    double w0 = 0.0, w1 = 0.0, total;
    if (j0 < limit) e0 = s.list[j0], w0 = a.weight_drawn(entry_value(e0));
    if (j1 < limit) e1 = s.list[j1], w1 = a.weight_drawn(entry_value(e1));
    const double before = cta_scan(s, w0 + w1, &total);
    bool keep0 = j0 < limit, keep1 = j1 < limit;
    if (o.use_p) {
        const double enough = (double)o.p * (o.use_k || all_listed ? total : whole);
        keep0 = keep0 && (j0 == 0 || before < enough);
        keep1 = keep1 && before + w0 < enough;
    }
    if (o.use_m) {
        keep0 = keep0 && w0 >= (double)o.mp;
        keep1 = keep1 && w1 >= (double)o.mp;
    }
    if (threadIdx.x == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    // what is kept, in order of index
    const int kept = __syncthreads_count(keep0) + __syncthreads_count(keep1);
    s.list[j0] = keep0 ? (e0 & 0xffffffffull) << 32 | (unsigned)j0 : ~0ull;
    s.list[j1] = keep1 ? (e1 & 0xffffffffull) << 32 | (unsigned)j1 : ~0ull;
    s.w[j0] = keep0 ? w0 : 0.0;
    s.w[j1] = keep1 ? w1 : 0.0;
    const float x0 = entry_value(e0), x1 = entry_value(e1);
    sort_list(s, limit);
    double v0 = 0.0, v1 = 0.0;
    if (j0 < kept) v0 = s.w[(unsigned)s.list[j0]];
    if (j1 < kept) v1 = s.w[(unsigned)s.list[j1]];
    const double run = cta_scan(s, v0 + v1, &total);
    const double target = (double)o.u * total;
    if (v0 > 0.0) {
        atomicMax(&s.last, j0);
        if (run + v0 > target) atomicMin(&s.found, j0);
    }
    if (v1 > 0.0) {
        atomicMax(&s.last, j1);
        if (run + v0 + v1 > target) atomicMin(&s.found, j1);
    }
    __syncthreads();
    const int at = s.found != INT_MAX ? s.found : s.last;
    const unsigned long long e = s.list[at];
    const int j = (int)(unsigned)e;
    if (j == j0 || j == j1) {
        const double y = ((double)(j == j0 ? x0 : x1) - (double)a.m) * a.a;
        answer(args, row, (int)(e >> 32), (float)(y * 0.69314718055994530942 - log(total)));
    }
}

// Logits at a distance d below the largest, by the bits of d: 32 bins an octave, from 2^-16 to 2^16; the last bin is beyond them.
__device__ __forceinline__ int distance_bin(float d) {
    const int b = (int)(__float_as_uint(d) >> 18) - (int)(111u << 5);
    return min(max(b, 0), kBins - 1);
}
__device__ __forceinline__ float distance_edge(int b) { return __uint_as_float((unsigned)(b + (111 << 5)) << 18); }

// What a histogram says about where a prefix ends: the bins, first to last (larger logits first), that hold its last element, the
// elements before them and in them, and the mass before them by the bins' middles.
struct Range {
    int first, last;
    unsigned before, in;
    double mass;
};

// Adds up the CTAs' histograms and picks the bin in which the count passes k (COUNT), the estimated mass `enough`, or the count half of
// all (HALF: where estimates did not help). A bin that was found by an estimate comes with its neighbours, as far as the list
// has room. before, mass: in front of the histogram. middle(b): a weight of bin b. False: there is nothing.
template <typename T, bool COUNT, typename F>
__device__ __forceinline__ bool pick(const Part<T>& a, unsigned k, double enough, bool half, unsigned before, double mass, F&& middle,
                                     Range& r) {
    Shared& s = *a.s;
    const int b0 = 2 * threadIdx.x, b1 = b0 + 1;
    unsigned c0 = 0, c1 = 0, total;
    for (int p = 0; p < a.parts; ++p) {
        const unsigned* h = a.at(s.hist, p);
        c0 += h[b0];
        c1 += h[b1];
    }
    if (threadIdx.x == 0) {
        s.found = s.pick_first = INT_MAX;
        s.last = s.pick_last = -1;
    }
    const unsigned n0 = before + cta_scan(s, c0 + c1, &total), n1 = n0 + c0, n2 = n1 + c1;
    if (total == 0u) return false;
    if (COUNT && before + total < k) {                       // not as many
        r = Range{0, 0, before, total, 0.0};
        return true;
    }
    double m0 = mass, m1 = mass;
    if (COUNT || half) {
        const unsigned goal = COUNT ? k : before + (total + 1) / 2;
        if (n0 < goal && n1 >= goal) s.found = b0;
        else if (n1 < goal && n2 >= goal) s.found = b1;
    } else {
        double w0 = 0.0, w1 = 0.0, all;
        if (c0) w0 = c0 * middle(b0);
        if (c1) w1 = c1 * middle(b1);
        m0 = mass + cta_scan(s, w0 + w1, &all);
        m1 = m0 + w0;
        if (c0 && m1 >= enough) atomicMin(&s.found, b0);
        else if (c1 && m1 + w1 >= enough) atomicMin(&s.found, b1);
        if (c0 | c1) atomicMax(&s.last, c1 ? b1 : b0);
    }
    __syncthreads();
    const int found = s.found != INT_MAX ? s.found : s.last;
    if (found == b0) s.pick_before = n0, s.pick_after = n1;
    else if (found == b1) s.pick_before = n1, s.pick_after = n2;
    __syncthreads();
    const unsigned lo = s.pick_before, hi = s.pick_after, in = hi - lo;
    const unsigned more = COUNT || in > (unsigned)kList ? 0u : ((unsigned)kList - in) / 2;
    if (more == 0u) {
        if (threadIdx.x == 0) s.pick_first = s.pick_last = found;
    } else if (b0 <= found && n0 + more >= lo) atomicMin(&s.pick_first, b0);
    else if (b1 <= found && n1 + more >= lo) atomicMin(&s.pick_first, b1);
    if (more != 0u && b1 >= found && n2 <= hi + more) atomicMax(&s.pick_last, b1);
    else if (more != 0u && b0 >= found && n1 <= hi + more) atomicMax(&s.pick_last, b0);
    __syncthreads();
    r.first = s.pick_first;
    r.last = s.pick_last;
    if (r.first == b0) s.pick_before = n0, s.mass_above = m0;
    else if (r.first == b1) s.pick_before = n1, s.mass_above = m1;
    if (r.last == b0) s.pick_after = n1;
    else if (r.last == b1) s.pick_after = n2;
    __syncthreads();
    r.before = s.pick_before;
    r.in = s.pick_after - r.before;
    r.mass = s.mass_above;
    return true;
}

// The search for a prefix's last element among what `cut` keeps: the k-th (COUNT), or the first at which the mass reaches `enough`.
template <typename T, bool COUNT>
__device__ __noinline__ Cut search(const Part<T>& a, const Cut cut, unsigned k, double enough, int& buf) {
    Shared& s = *a.s;
    const float cut_value = value_of(cut.key);
    auto kept = [&](float x, int i) { return x > cut_value || (x == cut_value && i <= cut.index) || cut.key == 0u; };
    const float a32 = a.a32;
    unsigned lo_key = key_of(-INFINITY) + 1, hi_key = key_of(a.m);       // where the element can be; masked logits are none
    double hi_mass = 0.0;                                                // above hi_key
    // a first histogram by the distance from the largest: its logarithm where elements are counted, linear over 64 octaves of the
    // weight where their mass is
    const float width = 64.0f / (float)kBins / a32;
    auto bin_of = [&](float d) { return COUNT ? distance_bin(d) : (int)fminf(d / width, (float)(kBins - 1)); };
    __syncthreads();                                                     // s.found and the histogram have been read
    s.hist[2 * threadIdx.x] = s.hist[2 * threadIdx.x + 1] = 0u;
    if (threadIdx.x == 0) {
        s.kmin = UINT_MAX;
        s.kmax = 0u;
    }
    __syncthreads();
    a.each([&](float x, int i) {
        if (x > -INFINITY && kept(x, i)) atomicAdd(&s.hist[bin_of(a.m - x)], 1u);
    });
    a.sync();
    Range r;
    pick<T, COUNT>(a, k, enough, false, 0u, 0.0, [&](int b) { return (double)ardiff::ex2(-((float)b + 0.5f) * width * a32); }, r);
    if (COUNT && r.before + r.in < k) {                                  // there are no more than k
        a.sync();
        return cut;
    }
    // the range as keys: those of its elements' extremes
    {
        unsigned lo = UINT_MAX, hi = 0u;
        a.each([&](float x, int i) {
            if (x > -INFINITY && kept(x, i)) {
                const int b = bin_of(a.m - x);
                if (b >= r.first && b <= r.last) {
                    const unsigned q = key_of(x);
                    lo = min(lo, q);
                    hi = max(hi, q);
                }
            }
        });
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        if ((threadIdx.x & 31) == 0) {
            atomicMin(&s.kmin, lo);
            atomicMax(&s.kmax, hi);
        }
    }
    a.sync();
    unsigned kmin = UINT_MAX, kmax = 0u;
    for (int p = 0; p < a.parts; ++p) {
        kmin = min(kmin, *a.at(&s.kmin, p));
        kmax = max(kmax, *a.at(&s.kmax, p));
    }
    a.sync();
    // The range shrinks to one bin of the histogram before it, or fits the list, at every step of the inner loop; with a wrong
    // estimate everything on one side of it is done with, from the third time on half of the elements or more.
    for (int turn = 0; turn < 64; ++turn) {
        // histograms over the keys, until few are left or all are equal
        while (r.in == UINT_MAX || (r.in > (unsigned)kList && kmin < kmax)) {
            int shift = 0;
            while (((kmax - kmin) >> shift) >= (unsigned)kBins) ++shift;
            s.hist[2 * threadIdx.x] = s.hist[2 * threadIdx.x + 1] = 0u;
            __syncthreads();
            a.each([&](float x, int i) {
                const unsigned q = key_of(x);
                if (q >= kmin && q <= kmax && kept(x, i)) atomicAdd(&s.hist[(kmax - q) >> shift], 1u);     // largest first
            });
            a.sync();
            const bool any = pick<T, COUNT>(a, k, enough, turn > 2, r.before, r.mass, [&](int b) {
                const unsigned down = ((unsigned)b << shift) + (shift ? 1u << (shift - 1) : 0u);
                return (double)ardiff::ex2((value_of(kmax - min(down, kmax - kmin)) - a.m) * a32);
            }, r);
            a.sync();                                        // the histograms have been read
            if (!any) return Cut{hi_key + 1, INT_MAX};       // nothing there: by the exact sums all above it is kept
            const unsigned top = kmax - ((unsigned)r.first << shift);
            const unsigned long long below = (unsigned long long)(r.last + 1) << shift;      // (up to 2^32)
            if (kmax - kmin >= below) kmin = kmax - (unsigned)below + 1;
            kmax = top;
        }
        // the exact sum above the range; the range's elements to the first CTA
        const float top = value_of(kmax), bottom = value_of(kmin);
        const bool ties = r.in > (unsigned)kList;
        if (threadIdx.x == 0) s.count = 0u;
        a.sync();
        double sure = 0.0;
        if (!COUNT) {
            sure = sum_segments(a, buf, 2.0, [&](float x, int i) { return x > top && kept(x, i) ? a.weight(x) : 0.0; });
            buf ^= 1;
        }
        if (!ties) {
            a.each([&](float x, int i) {
                if (x >= bottom && x <= top && kept(x, i)) {
                    const unsigned at = atomicAdd(a.at(&s.count, 0), 1u);
                    if (at < (unsigned)kList) *a.at(&s.list[at], 0) = entry(x, i);
                }
            });
            a.sync();
            if (a.rank == 0) {
                const int n = (int)min(s.count, (unsigned)kList);
                sort_list(s, n);
                if (COUNT) {
                    if (threadIdx.x == 0) {
                        const unsigned long long e = s.list[k - r.before - 1];
                        s.cut_key = ~(unsigned)(e >> 32);
                        s.cut_index = (int)(unsigned)e;
                        s.verdict = 0;
                    }
                } else {
                    if (threadIdx.x == 0) s.found = INT_MAX;
                    const int j0 = 2 * threadIdx.x;
                    double w0 = 0.0, w1 = 0.0, all;
                    if (j0 < n) w0 = a.weight(entry_value(s.list[j0]));
                    if (j0 + 1 < n) w1 = a.weight(entry_value(s.list[j0 + 1]));
                    const double run = sure + cta_scan(s, w0 + w1, &all);
                    if (j0 < n && run + w0 >= enough) atomicMin(&s.found, j0);
                    else if (j0 + 1 < n && run + w0 + w1 >= enough) atomicMin(&s.found, j0 + 1);
                    __syncthreads();
                    if (threadIdx.x == 0) {
                        s.mass_in = sure + all;
                        if (sure >= enough) {
                            s.verdict = 1;                               // it lies above
                        } else if (s.found == INT_MAX) {
                            s.verdict = 2;                               // below
                        } else {
                            const unsigned long long e = s.list[s.found];
                            s.cut_key = ~(unsigned)(e >> 32);
                            s.cut_index = (int)(unsigned)e;
                            s.verdict = 0;
                        }
                    }
                }
            }
        } else {
            // one value, more often than the list is long: as many of it as are needed, lowest indices first
            double need = (double)(k - r.before);
            const double w = COUNT ? 1.0 : a.weight(top);
            int verdict = 0;
            if (!COUNT) {
                need = fmin(ceil((enough - sure) / w), (double)r.in + 1.0);
                while (need > 1.0 && sure + (need - 1.0) * w >= enough) need -= 1.0;
                while (need <= (double)r.in && sure + need * w < enough) need += 1.0;
                verdict = sure >= enough ? 1 : need > (double)r.in ? 2 : 0;
            }
            auto one = [&](float x, int i) { return x == top && kept(x, i) ? 1.0 : 0.0; };
            // (the sum over all is r.in: the share of it is a whole number less a half, up to rounding)
            sum_segments(a, buf, (need - 0.5) / (double)r.in, one);
            buf ^= 1;
            const int owner = s.owner / kWarps;
            if (verdict == 0 && owner == a.rank) {
                const int at = locate(a, need - 0.5, one);
                if (threadIdx.x == 0) s.cut_index = at;
            }
            a.sync();
            if (a.rank == 0 && threadIdx.x == 0) {
                s.cut_key = kmax;
                s.cut_index = *a.at(&s.cut_index, owner);
                s.verdict = verdict;
                s.mass_in = sure + r.in * w;
            }
        }
        a.sync();
        const int verdict = *a.at(&s.verdict, 0);
        const Cut found{*a.at(&s.cut_key, 0), *a.at(&s.cut_index, 0)};
        const double with = *a.at(&s.mass_in, 0);
        a.sync();
        if (verdict == 0) return found;
        // the estimates were wrong about the range: the exact sums say on which side of it the element lies
        if (verdict == 1) {
            lo_key = kmax + 1;
        } else {
            hi_key = kmin - 1;
            hi_mass = with;
        }
        if (lo_key > hi_key) return Cut{hi_key + 1, INT_MAX};            // sums that differ in their last bit
        kmin = lo_key;
        kmax = hi_key;
        r.in = UINT_MAX;                                     // not known: a histogram at least
        r.before = 0;
        r.mass = hi_mass;
    }
    return Cut{hi_key + 1, INT_MAX};                         // (2^18 elements are halved 18 times)
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const Args args) {
    constexpr int N = ardiff::Piece<T>::N;
    extern __shared__ __align__(16) uint4 s_piece[];
    __shared__ Shared s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x / args.parts;
    Settings o;
    o.u = args.u[row];
    o.T = args.temperature ? args.temperature[row] : 1.f;
    o.k = args.top_k ? args.top_k[row] : 0;
    o.p = args.top_p ? args.top_p[row] : 1.f;
    o.mp = args.min_p ? args.min_p[row] : 0.f;
    const bool valid = o.u >= 0.f && o.u < 1.f && o.T >= 0.f && o.T < INFINITY && o.p == o.p && o.mp == o.mp;
    o.use_k = o.k > 0 && o.k < args.V;
    o.use_p = o.p < 1.f;
    o.use_m = o.mp > 0.f;
    o.mp = fminf(o.mp, 1.f);

    Part<T> a;
    a.s = &s;
    a.rank = blockIdx.x % args.parts;
    a.parts = args.parts;
    a.V = args.V;
    a.piece = s_piece;
    a.tiny = o.u == 0.f;
    // the aligned pieces that cover the row; `shift` places in front of it belong to none of them
    const T* x = static_cast<const T*>(args.x) + row * args.ld;
    const int shift = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
    const int pieces = (shift + args.V + N - 1) / N;
    const int per = (pieces + a.parts - 1) / a.parts;
    const int p0 = min(pieces, a.rank * per);
    a.pieces = min(pieces, p0 + per) - p0;
    a.segment = (a.pieces + kWarps - 1) / kWarps;
    a.first = p0 * N - shift;
    float top = -INFINITY;
    {
        const int end = min(a.pieces, (warp + 1) * a.segment);
        for (int p = warp * a.segment + lane; p < end; p += 32) {
            const int e = a.first + p * N;
            uint4 v;
            if (e >= 0 && e + N <= args.V) {
                v = __ldg(reinterpret_cast<const uint4*>(x + e));
            } else {
                T t[N];
#pragma unroll
                for (int i = 0; i < N; ++i)
                    t[i] = e + i >= 0 && e + i < args.V ? x[e + i] : ardiff::from_float<T>(-INFINITY);
                float f[N];
#pragma unroll
                for (int i = 0; i < N; ++i) f[i] = ardiff::to_float(t[i]);
                v = ardiff::pack(f, T());
            }
            s_piece[p] = v;
            float f[N];
            ardiff::unpack(v, f, T());
#pragma unroll
            for (int i = 0; i < N; ++i) top = max_nan(top, f[i]);
        }
    }
    s.thread_max[tid] = top;
    float wtop = top;
#pragma unroll
    for (int q = 16; q > 0; q >>= 1) wtop = max_nan(wtop, __shfl_xor_sync(0xffffffffu, wtop, q));
    if (lane == 0) s.warp_max[warp] = wtop;
    if (tid == 0) s.count = 0u;
    __syncthreads();
    float own = s.warp_max[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) own = max_nan(own, s.warp_max[w]);
    const bool greedy = o.T == 0.f;
    if (greedy) {                                            // the lowest index of this part's largest
        int first = INT_MAX;
        if (top == own)
            a.each([&](float v, int i) { if (v == own) first = min(first, i); });
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0) s.warp_first[warp] = first;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kWarps; ++w) first = min(first, s.warp_first[w]);
            s.cta_first = first;
        }
    }
    if (tid == 0) s.cta_max = own;
    a.sync();
    a.m = own;
    for (int r = 0; r < a.parts; ++r) a.m = max_nan(a.m, *a.at(&s.cta_max, r));
    if (!valid || !(fabsf(a.m) < INFINITY) || greedy) {
        if (a.rank == 0 && tid == 0) {
            int token = -1;
            if (valid && fabsf(a.m) < INFINITY) {
                token = INT_MAX;
                for (int r = 0; r < a.parts; ++r)
                    if (*a.at(&s.cta_max, r) == a.m) token = min(token, *a.at(&s.cta_first, r));
            }
            answer(args, row, token, token >= 0 ? 0.f : NAN);
        }
        a.sync();
        return;
    }
    a.a = 1.4426950408889634074 / (double)o.T;
    a.a32 = (float)fmin(a.a, 3e38);
    int buf = 0;
    Cut cut = no_cut();
    if (o.use_k || o.use_p) {
        // a distance below the largest logit within which everything that is kept lies, but few others
        float reach = -1.f;
        double whole = 0.0;
        const bool all = args.V <= kList;
        if (all) {
            reach = INFINITY;
        } else {
            if (!o.use_k) {
                whole = sum_segments(a, buf, 2.0, [&](float v, int) { return a.weight(v); });
                buf ^= 1;
            }
            s.hist[2 * tid] = s.hist[2 * tid + 1] = 0u;
            if (tid == 0) s.found = INT_MAX;
            __syncthreads();
            for (int r = 0; r < a.parts; ++r) {
                const float d = a.m - *a.at(&s.thread_max[tid], r);
                const int b = distance_bin(d);
                if (b < kBins - 1) atomicAdd(&s.hist[b], 1u);
            }
            __syncthreads();
            const unsigned c0 = s.hist[2 * tid], c1 = s.hist[2 * tid + 1];
            unsigned total;
            const unsigned before = cta_scan(s, c0 + c1, &total);
            if (o.use_k) {
                if (before < (unsigned)o.k && before + c0 >= (unsigned)o.k) s.found = 2 * tid;
                else if (before + c0 < (unsigned)o.k && before + c0 + c1 >= (unsigned)o.k) s.found = 2 * tid + 1;
            } else {
                // weights at the bins' far edges, less what fp32 may have added to them: no more than the logits have
                const double m0 = c0 * 0.9999 * (double)ardiff::ex2(-distance_edge(2 * tid + 1) * a.a32);
                const double m1 = c1 * 0.9999 * (double)ardiff::ex2(-distance_edge(2 * tid + 2) * a.a32);
                double sum;
                const double run = cta_scan(s, m0 + m1, &sum);
                const double enough = (double)o.p * whole;
                if (c0 && run + m0 >= enough) atomicMin(&s.found, 2 * tid);
                else if (c1 && run + m0 + m1 >= enough) atomicMin(&s.found, 2 * tid + 1);
            }
            __syncthreads();
            if (s.found != INT_MAX) reach = distance_edge(s.found + 1);
        }
        if (reach >= 0.f) {
            if (a.m - top < reach || (all && top > -INFINITY))
                a.each([&](float v, int i) {
                    if (v > -INFINITY && (all || a.m - v < reach)) {
                        const unsigned at = atomicAdd(a.at(&s.count, 0), 1u);
                        if (at < (unsigned)kList) *a.at(&s.list[at], 0) = entry(v, i);
                    }
                });
            a.sync();
            const unsigned n = *a.at(&s.count, 0);
            a.sync();
            if (n <= (unsigned)kList) {
                if (a.rank == 0) finish_list(args, row, a, o, (int)n, whole, all);
                return;
            }
        }
        if (o.use_k) cut = search<T, true>(a, cut, (unsigned)o.k, 0.0, buf);
        if (o.use_p) {
            const float c = value_of(cut.key);
            if (o.use_k) {
                whole = sum_segments(a, buf, 2.0, [&](float v, int i) {
                    return cut.key == 0u || v > c || (v == c && i <= cut.index) ? a.weight(v) : 0.0;
                });
                buf ^= 1;
            }
            cut = search<T, false>(a, cut, 0u, fmax((double)o.p * whole, 1e-300), buf);       // at least one
        }
    }
    // the draw among what the cut keeps
    const float c = value_of(cut.key);
    const float half = 0.5f * a.m;                           // (halves: a difference of two logits can pass fp32's range)
    const float floor_ = o.use_m ? 0.5f * (log2f(o.mp) - 0.01f) : -INFINITY;
    auto kept = [&](float v, int i) {
        return (cut.key == 0u || v > c || (v == c && i <= cut.index)) && (!o.use_m || (0.5f * v - half) * a.a32 >= floor_);
    };
    auto weight = [&](float v, int i) {
        if (!kept(v, i)) return 0.0;
        const double w = a.weight(v);
        return o.use_m && w < (double)o.mp ? 0.0 : w;
    };
    auto weight_drawn = [&](float v, int i) {
        if (!kept(v, i)) return 0.0;
        const double w = a.weight_drawn(v);
        return o.use_m && w < (double)o.mp ? 0.0 : w;
    };
    const double total = a.tiny ? sum_segments(a, buf, (double)o.u, weight_drawn) : sum_segments(a, buf, (double)o.u, weight);
    a.sync();                                                // every CTA has read the others' sums
    if (s.owner / kWarps != a.rank) return;
    const int token = locate(a, (double)o.u * total, weight_drawn);
    if (tid == 0) {
        const float v = ardiff::to_float(reinterpret_cast<const T*>(s_piece)[token - a.first]);
        const double y = ((double)v - (double)a.m) * a.a;
        answer(args, row, token, (float)(y * 0.69314718055994530942 - log(total)));
    }
}

template <typename T>
int launch(Args a, int64_t n, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};
    const void* fn = reinterpret_cast<const void*>(&sample_kernel<T>);
    constexpr int kMostBytes = 160 * 1024;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return ARDIFF_ERR_CUDA;
    if (dev >= 64 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostBytes) != cudaSuccess) return ARDIFF_ERR_CUDA;
        if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    // parts of at most 64 KB where that is possible; more parts while there are SMs without one and parts of 16 KB
    const int64_t pieces = ((int64_t)a.V + 2 * ardiff::Piece<T>::N - 2) / ardiff::Piece<T>::N;
    int parts = 1;
    while (parts < kMaxParts && (pieces * 16 > (int64_t)parts * 65536 || (n * parts < 148 && pieces * 16 > (int64_t)parts * 16384)))
        parts *= 2;
    a.parts = parts;
    const int64_t bytes = (pieces + parts - 1) / parts * 16;
    if (bytes > kMostBytes) return ARDIFF_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = parts; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(n * parts)); cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)bytes; cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, sample_kernel<T>, (const Args)a);
    ardiff::set_launch_count(1);
    return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}

}  // namespace

extern "C" int ardiff_sample_tokens(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t ld, const float* u,
                                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                                    int32_t* token, float* logprob, void* stream) {
    const int size = ardiff::value_size(dtype);
    if (!size) return ARDIFF_ERR_UNSUPPORTED;
    if (n < 0 || n >= (int64_t)1 << 28 || V < 1 || V > ARDIFF_SAMPLE_MAX_V || ld < V) return ARDIFF_ERR_SHAPE;
    if (n == 0) {
        ardiff::set_launch_count(0);
        return ARDIFF_OK;
    }
    if (!logits || !u || !token || !logprob) return ARDIFF_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(logits) % size) return ARDIFF_ERR_ALIGN;
    Args a;
    memset(&a, 0, sizeof(a));
    a.x = logits; a.ld = ld; a.u = u; a.temperature = temperature; a.top_p = top_p; a.min_p = min_p; a.top_k = top_k;
    a.token = token; a.logprob = logprob; a.V = V;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == ARDIFF_F32) return launch<float>(a, n, st);
    if (dtype == ARDIFF_F16) return launch<__half>(a, n, st);
    return launch<__nv_bfloat16>(a, n, st);
}
