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
// A row belongs to a cluster of one to eight CTAs, a contiguous part each, a part to 32 segments, four a warp. A first pass reads the row
// from memory and keeps every thread's largest logit in every segment (a "group", 1024 a CTA); later passes, over rows that need
// them, find it in L2. What is done with it depends on its settings:
//   T = 0                  the largest logit's lowest index
//   no filter              the first pass sums the segments' weights, too, relative to a reference of the CTA's own, in fp64; then the
//                          one segment is walked in which the draw ends
//   top-k, small nuclei,   a list: at least k logits are not below the k-th of the groups' largest, and the mass down to one of those is
//   few with min-p         at least theirs; the groups with anything above that bound are read again, the first CTA sorts what
//                          it finds there and does the rest alone
//   large nuclei           a histogram of the weights says about where the nucleus ends, where a bin holds too many a second one
//                          more closely; an exact pass sums what lies above that range and lists what lies in it; the sums
//                          say whether the range was right, and on which side of it to look if it was not
//   large k                a histogram counts down to the bin of the k-th, which is listed
//   what none of these     (thousands of different logits closer together than 2^-14 octaves of the weight): a search by the logits
//   settles                as whole numbers
//
// Measured on B200 (one call after the other, inputs not in L2, us; floor: the row read once at the measured copy rate), 512 x 131072 bf16, floor
// 20.5: T = 0 28, top-k below 100 with top-p 47, no filter 106 (bound by 67 million fp64 weights of 15 instructions, 60 us at 64 a clock
// and SM), nuclei of rows that fall off steeply 420, of flat ones (tens of thousands) 610, min-p that keeps few 55, thousands 223.
// 1 x 32768 bf16 with top-k and top-p, two CTAs: 16, of which a dozen barriers and dependent loads are all.
// 64 registers a thread, for four CTAs an SM, cost sample_kernel 600 to 700 bytes of spills (up to 190 in the functions it calls); with
// 80 and three CTAs sums were 10 % faster and lists 30 % slower.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/ardiff.h"
#include "common.cuh"
#include "launch.cuh"
#include "nucleus.h"
#include "rows.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 4 * kThreads;      // of a histogram, four a thread
constexpr int kList = 4 * kThreads;      // logits that the first CTA sorts, four a thread
constexpr int kEach = 4;                 // list entries, bins a thread
constexpr int kGroups = 4;               // segments a warp; a thread's share of one is a group, whose largest logit is kept
constexpr int kSegments = kGroups * kWarps;  // of a CTA's part
constexpr int kMaxParts = 8;
constexpr float kLeastU = 0x1p-24f;      // below it, u asks how nothing adds up: every weight counts as what it is
constexpr float kLeastMin = 0x1p-60f;    // min_p from which every weight that has it is one that sums over many hold exactly
constexpr float kSane = 6e4f;            // logits up to which, at temperatures from 1e-3 to 1e3, a first pass can sum

struct Args {
    const void* x;
    int64_t ld;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* token;
    float* logprob;
    int32_t V, parts;
};

// A piece of the row, which the kernel before may have written and this one does not: behind begin_kernel()'s wait, both being volatile, but free
// to be moved over stores, all of which go elsewhere. (As ordinary loads: 256 x 131072 f32, flat nuclei, 306 us instead of 296.)
__device__ __forceinline__ uint4 load_logits(const uint4* p) {
    uint4 r;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// Kept: everything before this element in the order (descending, lowest index first), and it.
struct Cut {
    float value;
    int index;
    __device__ __forceinline__ bool keeps(float v, int i) const { return v > value || (v == value && i <= index); }
};
__device__ __forceinline__ Cut no_cut() { return Cut{-INFINITY, INT_MAX}; }

struct Shared {
    float top[kGroups][kThreads];        // the groups' largest logits
    float warp_max[kWarps];
    double seg[2][kSegments];            // sums of the segments; two, so that one may still be read by another CTA
    unsigned seg_ties[kSegments];
    double scan[kWarps];
    unsigned uscan[kWarps];
    double total, before;
    int owner;                           // segment in which a sum passes its target, of all CTAs'
    int found, last;
    float cta_max;
    float ref;                           // what the part's sums of the first pass are relative to
    int first;                           // lowest index of the part's largest logit
    unsigned groups;                     // entries of `group`
    unsigned count;                      // entries of `list` (of the first CTA)
    unsigned kmin, kmax;
    int pick_first, pick_last;
    unsigned pick_before, pick_after;
    int verdict;
    Cut cut;
    unsigned cut_ahead;
    double mass_above, mass_in;
    unsigned short group[kGroups * kThreads];
    alignas(16) unsigned long long list[kList];
    union alignas(16) {                  // (read in 16-byte pieces)
        unsigned hist[kBins];
        double w[kList];
    };
};

using ardiff::key_of;
using ardiff::value_of;

__device__ __forceinline__ float max_nan(float a, float b) {       // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 2^y of y = d a: y = k + r, |r| <= 1/2, 2^r = 1 + r P(r), P of degree 8 by interpolation at the Chebyshev nodes (3.7e-14 relative; exactly
// 1 at 0). |y| < 1000. The coefficients lie in constant memory, from where the multiply-adds take them as they are: as numbers in the
// code they were moved into registers for every value (34 instructions a value instead of 30).
__constant__ double kPow2[10] = {1.0203121063391729e-07, 1.3255224878668817e-06, 1.525268684626772e-05, 0.00015403455852453838,
                                 0.0013333558179043112, 0.009618129159402558, 0.055504108664760424, 0.2402265069581299,
                                 0.6931471805599453, 1.0};
__device__ __forceinline__ double pow2(double d, double a) {
    constexpr double kRound = 6755399441055744.0;                  // 1.5 2^52: adding it leaves the nearest integer
    const double t = fma(d, a, kRound);
    const double r = fma(d, a, kRound - t);
    double p = kPow2[0];
#pragma unroll
    for (int i = 1; i < 10; ++i) p = fma(p, r, kPow2[i]);
    return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
}

// The weights of a row. Sums over many use bulk(): logits below `lowest` count as 2^-100 each, which is nothing beside the largest
// one's 1 and to the least u (2^18 of them are 2^-82; at most 2^-77 where fp32 had to round `lowest`). One that may be drawn has its own()
// weight, down to fp64's smallest.
struct Weights {
    double m, a;                         // the largest logit, log2(e) / T
    float lowest;
    bool far;                            // bulk() will not do: a tiny u asks for the first tokens of any weight at all; temperatures
                                         // so high, or so low, that fp32 has no such `lowest`
    __device__ __forceinline__ double bulk(float v) const { return pow2((double)fmaxf(v, lowest) - m, a); }
    __device__ __noinline__ static double exact(double y) { return y >= -1100.0 ? exp2(y) : 0.0; }
    __device__ __forceinline__ double own(float v) const {
        const double d = (double)v - m, y = d * a;
        return y >= -100.0 ? pow2(d, a) : exact(y);                // (-inf: 0)
    }
};

template <typename T>
struct Part {                            // this CTA's part of its row
    static constexpr int N = ardiff::Piece<T>::N;
    const T* x;                          // the row
    int pieces, segment;                 // pieces (aligned, 16 bytes), and pieces a segment
    int first;                           // index of the part's first value in the row (negative in front of the row)
    int whole0, whole1;                  // pieces that lie in the row as a whole
    int rank, parts, V;
    Shared* s;

    __device__ __forceinline__ void sync() const {
        if (parts > 1) cg::this_cluster().sync(); else __syncthreads();
    }
    template <typename U> __device__ __forceinline__ U* at(U* p, int r) const {
        return parts > 1 ? cg::this_cluster().map_shared_rank(p, r) : p;
    }
    // the piece of the values e, e + 1, ... at either end of a row: -inf in the places outside it
    __device__ __noinline__ static uint4 edge(const T* x, int e, int V) {
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = e + i >= 0 && e + i < V ? ardiff::to_float(x[e + i]) : -INFINITY;
        return ardiff::pack(v, T());
    }
    // f(piece's bits, piece) for pieces begin, begin + step, ... below end; AHEAD loads at a time, issued while the ones before are used
    template <int AHEAD, typename F> __device__ __forceinline__ void scan(int begin, int end, int step, F&& f) const {
        const uint4* base = reinterpret_cast<const uint4*>(x + first);     // (aligned; pieces whole0 .. whole1 - 1 are read)
        const int most = whole1 - 1;
        if (begin >= end) return;
        // (a place outside the whole pieces gives the nearest of them, which is not used)
        auto load = [&](int p) { return whole0 <= most ? load_logits(base + max(whole0, min(p, most))) : uint4(); };
        uint4 q[AHEAD], next[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) q[i] = next[i] = load(begin + i * step);
#pragma unroll 1
        for (int p = begin; p < end; p += AHEAD * step) {
            if (p + AHEAD * step < end) {
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) next[i] = load(p + (AHEAD + i) * step);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int at = p + i * step;
                if (at >= end) break;
                if (at < whole0 || at >= whole1) q[i] = edge(x, first + at * N, V);
                f(q[i], at);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) q[i] = next[i];
        }
    }
    // f(value, index) for every value of the calling warp's segments (once in the code: not for what has to be fast)
    template <typename F> __device__ __forceinline__ void each(F&& f) const {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        scan<4>(warp * kGroups * segment + lane, min(pieces, (warp + 1) * kGroups * segment), 32, [&](const uint4& q, int p) {
            float v[N];
            ardiff::unpack(q, v, T());
#pragma unroll
            for (int i = 0; i < N; ++i) f(v[i], first + p * N + i);
        });
    }
};

// Which logits go on a list.
struct Listed {
    enum { ALL, REACH, WEIGHT, EQUAL } which;
    float m, bound, half, a32;           // REACH: nearer to m than bound; WEIGHT: half the exponent at least bound; EQUAL: bound
    __device__ __forceinline__ bool operator()(float v) const {
        if (which == REACH) return m - v < bound;
        if (which == WEIGHT) return (0.5f * v - half) * a32 >= bound;
        if (which == EQUAL) return v == bound;
        return v > -INFINITY;
    }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Exclusive sums over the CTA's threads; *total: of all.
__device__ __noinline__ double cta_scan(Shared& s, double v, double* total) {
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
__device__ __noinline__ unsigned cta_scan(Shared& s, unsigned v, unsigned* total) {
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

// Sums of f(value, index) over the segments; afterwards every CTA knows their sum (returned) and the first segment at whose end the
// running sum is above `share` of it (the last one with anything, if none is: s.owner), and the sum before that (s.before). Two
// calls in a row use different buffers: buf is turned, and says which one the last call used. (Not inlined: these loops get all
// registers that way, and f's values lie in them.)
template <typename T>
__device__ __noinline__ double add_segments(const Part<T> a, const int buf, const double share, const bool scaled, const Weights wt) {
    Shared& s = *a.s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    a.sync();
    if (scaled) {                                            // first-pass sums: from the part's own reference to the row's largest
        if (threadIdx.x < kSegments) s.seg[buf][threadIdx.x] *= wt.own(s.ref);
        a.sync();
    }
    if (warp == 0) {
        constexpr int kPer = kMaxParts * kSegments / 32;
        double v[kPer], own = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int g = lane * kPer + i;
            v[i] = g < a.parts * kSegments ? *a.at(&s.seg[buf][g % kSegments], g / kSegments) : 0.0;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) own += v[i];
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
template <typename T, typename F>
__device__ __noinline__ double sum_in(const Part<T> a, const int buf, const double share, const F f) {
    constexpr int N = Part<T>::N;
    Shared& s = *a.s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
    for (int g = warp * kGroups; g < (warp + 1) * kGroups; ++g) {
        double acc[2] = {0.0, 0.0};
        a.template scan<2>(g * a.segment + lane, min(a.pieces, (g + 1) * a.segment), 32, [&](const uint4& q, int p) {
            // (four weights side by side: with eight, registers run out)
#pragma unroll 1
            for (int h = 0; h < N; h += 4) {
                float v[4];
                ardiff::unpack4(q, h, v, T());
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i & 1] += f(v[i], a.first + p * N + h + i);
            }
        });
        const double mine = warp_sum(acc[0] + acc[1]);
        if (lane == 0) s.seg[buf][g] = mine;
    }
    return add_segments(a, buf, share, false, Weights());
}
template <typename T, typename F>
__device__ __forceinline__ double sum_segments(const Part<T>& a, int& buf, double share, const F& f) {
    buf ^= 1;
    return sum_in<T, F>(a, buf, share, f);
}

// In the CTA that owns segment g: the index of the first value at which the running sum of f, `carry` before the segment, passes
// `target` (the last value with anything, if none does). All threads of that CTA call it.
template <typename T, typename F>
__device__ __noinline__ int locate(const Part<T> a, const int g, double carry, const double target, const F f) {
    constexpr int N = Part<T>::N;
    Shared& s = *a.s;
    const int begin = g % kSegments * a.segment, end = min(a.pieces, begin + a.segment);
    __syncthreads();
    if (threadIdx.x == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    for (int p0 = begin; p0 < end; p0 += kThreads) {
        const int p = p0 + threadIdx.x, e = a.first + p * N;
        double w[N], own = 0.0;
        a.template scan<1>(p, min(end, p + 1), 1, [&](const uint4& q, int) {
            float v[N];
            ardiff::unpack(q, v, T());
#pragma unroll
            for (int i = 0; i < N; ++i) {
                w[i] = f(v[i], e + i);
                own += w[i];
            }
        });
        double total;
        double run = carry + cta_scan(s, own, &total);             // (its barriers put s.found's start before its use)
        if (own > 0.0) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
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

// Where the segment of a draw holds nothing (all of it masked, and the sums of the ones around it rounded differently on their two ways
// to the border): the index of the first value of any weight from `from` on, the last one before it if there is none. All threads.
template <typename T, typename F>
__device__ __noinline__ int nearest(const Part<T> a, const int from, const F f) {
    Shared& s = *a.s;
    __syncthreads();                                         // s.found and s.last have been read
    if (threadIdx.x == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.V; i += kThreads) {
        if (f(ardiff::to_float(a.x[i]), i) > 0.0) {
            if (i >= from) atomicMin(&s.found, i); else atomicMax(&s.last, i);
        }
    }
    __syncthreads();
    return s.found != INT_MAX ? s.found : s.last;
}

// Sorts s.list[0 .. n), ascending, n <= kList; all entries but those of ~0 are different. Up to kThreads of them each counts the smaller
// ones (64 take 0.3 us, where exchanging neighbours step by step took 2.7); beyond, each warp sorts 128 in its registers and
// every entry looks itself up in the other warps' runs.
__device__ __noinline__ void sort_list(Shared& s, const int n) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr unsigned long long kNone = ~0ull;
    __syncthreads();
    if (n <= kThreads) {
        const unsigned long long key = tid < n ? s.list[tid] : kNone;
        int rank = 0;
        if (warp * 32 < n) {
            int j = 0;
#pragma unroll 4
            for (; j + 1 < n; j += 2) {
                const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(&s.list[j]);
                rank += (q.x < key) + (q.y < key);
            }
            if (j < n) rank += s.list[j] < key;
        }
        const int valid = __syncthreads_count(key != kNone);
        if (key != kNone) s.list[rank] = key;
        if (tid >= valid && tid < n) s.list[tid] = kNone;
        __syncthreads();
        return;
    }
    unsigned long long key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = 4 * tid + i < n ? s.list[4 * tid + i] : kNone;
    auto order = [](unsigned long long& x, unsigned long long& y, bool up) {
        if ((x > y) == up) {
            const unsigned long long t = x;
            x = y;
            y = t;
        }
    };
    // 128 in a warp, places 4 lane .. 4 lane + 3: runs of ever longer size, upwards and downwards in turn
    order(key[0], key[1], true);
    order(key[2], key[3], false);
#pragma unroll
    for (int size = 4; size <= 128; size *= 2) {
        const bool up = (4 * lane & size) == 0;
#pragma unroll
        for (int step = size / 8; step > 0; step /= 2) {
            const bool low = ((lane & step) == 0) == up;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned long long other = __shfl_xor_sync(0xffffffffu, key[i], step);
                key[i] = (other < key[i]) == low ? other : key[i];
            }
        }
        order(key[0], key[2], up);
        order(key[1], key[3], up);
        order(key[0], key[1], up);
        order(key[2], key[3], up);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) s.list[4 * tid + i] = key[i];
    __syncthreads();
    int rank[4], valid = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) rank[i] = 4 * lane + i;
    for (int run = 0; run < kWarps; ++run) {
        if (run == warp || run * 128 >= n) continue;
        const unsigned long long* r = s.list + run * 128;
        int below[4] = {};
#pragma unroll
        for (int step = 64; step > 0; step /= 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (r[below[i] + step - 1] < key[i]) below[i] += step;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) rank[i] += below[i] + (r[below[i]] < key[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) valid += __syncthreads_count(key[i] != kNone);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (key[i] != kNone) s.list[rank[i]] = key[i];
        if (4 * tid + i >= valid) s.list[4 * tid + i] = kNone;
    }
    __syncthreads();
}

__device__ __forceinline__ unsigned long long entry(float x, int index) {
    return (unsigned long long)(~key_of(x)) << 32 | (unsigned)index;
}
__device__ __forceinline__ float entry_value(unsigned long long e) { return value_of(~(unsigned)(e >> 32)); }

// Takes every value that is to be listed out of the groups whose largest logit is: to the list of the first CTA (*count, list), or, of
// EQUAL ones, the lowest index to *lowest. All threads.
template <typename T>
__device__ __noinline__ void collect(const Part<T> a, const Listed listed, unsigned* count, unsigned long long* list, int* lowest) {
    constexpr int N = Part<T>::N;
    Shared& s = *a.s;
    if (threadIdx.x == 0) s.groups = 0u;
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
        if (listed(s.top[g][threadIdx.x])) s.group[atomicAdd(&s.groups, 1u)] = (unsigned short)(g * kThreads + threadIdx.x);
    __syncthreads();
    // every thread takes pieces of them in turn, four loads at a time
    const int turns = (a.segment + 31) / 32;
    int items = (int)s.groups * turns;
    const uint4* base = reinterpret_cast<const uint4*>(a.x + a.first);
    const int most = a.whole1 - 1;
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < items; i0 += 4 * kThreads) {
        uint4 q[4];
        int at[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned item = (unsigned)(i0 + j * kThreads);
            at[j] = a.pieces;
            if ((int)item < items) {
                const int id = s.group[item / turns], t = id & (kThreads - 1), in = (t & 31) + (int)(item % turns) * 32;
                if (in < a.segment) at[j] = min(a.pieces, ((t >> 5) * kGroups + id / kThreads) * a.segment + in);
            }
            q[j] = a.whole0 <= most && at[j] < a.pieces ? load_logits(base + max(a.whole0, min(at[j], most))) : uint4();
        }
        // (one copy of what follows: the pieces move down)
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {
            if (at[0] < a.pieces) {
                if (at[0] < a.whole0 || at[0] >= a.whole1) q[0] = Part<T>::edge(a.x, a.first + at[0] * N, a.V);
                float v[N];
                ardiff::unpack(q[0], v, T());
                unsigned hit = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) hit |= listed(v[i]) && v[i] > -INFINITY ? 1u << i : 0u;
#pragma unroll 1
                while (hit) {
                    const int i = __ffs(hit) - 1, index = a.first + at[0] * N + i;
                    hit &= hit - 1;
                    if (lowest) {
                        atomicMin(lowest, index);
                    } else {
                        const unsigned place = atomicAdd(count, 1u);
                        if (place < (unsigned)kList) {
                            list[place] = entry(ardiff::to_float(a.x[index]), index);
                        } else {                             // there is more than the list holds, and the count says so
                            items = hit = 0;
                            at[1] = at[2] = at[3] = a.pieces;
                        }
                    }
                }
            }
            q[0] = q[1], q[1] = q[2], q[2] = q[3];
            at[0] = at[1], at[1] = at[2], at[2] = at[3];
        }
    }
}

struct Settings {
    float T, p, mp, u;
    int k;
    bool use_k, use_p, use_m;
};

__device__ __forceinline__ void answer(const Args& a, int64_t row, int token, float logprob) {
    a.token[row] = token;
    a.logprob[row] = logprob;
}

// The first CTA alone: s.list[0 .. n) holds every logit that may be kept. `whole`: the mass that top-p is a share of, where it is not
// the list's own (negative).
__device__ __forceinline__ void finish_list(const Args& args, int64_t row, Shared& s, const Weights& wt, const Settings& o, int n,
                                            double whole) {
    sort_list(s, n);
    const int j0 = kEach * threadIdx.x;
    const int limit = o.use_k ? min(o.k, n) : n;
    unsigned long long e[kEach];
    double w[kEach], own = 0.0, total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        e[i] = ~0ull;
        w[i] = 0.0;
        if (j0 + i < limit) e[i] = s.list[j0 + i], w[i] = wt.own(entry_value(e[i]));
        own += w[i];
    }
    double before = cta_scan(s, own, &total);
    const double enough = (double)o.p * (whole >= 0.0 ? whole : total);
    bool keep[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        keep[i] = j0 + i < limit && (!o.use_p || j0 + i == 0 || before < enough) && (!o.use_m || w[i] >= (double)o.mp);
        before += w[i];
    }
    if (threadIdx.x == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    __syncthreads();                                         // the list has been read
    // what is kept, in order of index
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        s.list[j0 + i] = keep[i] ? (e[i] & 0xffffffffull) << 32 | (unsigned)(j0 + i) : ~0ull;
        s.w[j0 + i] = keep[i] ? w[i] : 0.0;
    }
    __syncthreads();
    sort_list(s, limit);
    own = 0.0;
    unsigned at[kEach];
    double v[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        at[i] = j0 + i < limit ? (unsigned)s.list[j0 + i] : ~0u;
        v[i] = at[i] != ~0u ? s.w[at[i]] : 0.0;
        own += v[i];
    }
    double run = cta_scan(s, own, &total);
    const double target = (double)o.u * total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        run += v[i];
        if (v[i] > 0.0) {
            atomicMax(&s.last, j0 + i);
            if (run > target) atomicMin(&s.found, j0 + i);
        }
    }
    __syncthreads();
    const unsigned long long drawn = s.list[s.found != INT_MAX ? s.found : s.last];
    const int j = (int)(unsigned)drawn;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (j == j0 + i) {
            const double y = ((double)entry_value(e[i]) - wt.m) * wt.a;
            answer(args, row, (int)(drawn >> 32), (float)(y * 0.69314718055994530942 - log(total)));
        }
    }
}

// Bins of logits by their distance d below the largest. By the bits of d: 32 bins an octave, from 2^-16 to 2^16, the last bin beyond.
__device__ __forceinline__ int distance_bin(float d) {
    const int b = (int)(__float_as_uint(d) >> 18) - (int)(111u << 5);
    return min(max(b, 0), kBins - 1);
}
__device__ __forceinline__ float distance_edge(int b) { return __uint_as_float((unsigned)(b + (111 << 5)) << 18); }
// By the weight: a code of 2^14 steps an octave, up to 64 octaves (to the nearest whole number: adding 2^23 leaves it in the last
// bits), of which a histogram takes the upper ten bits, and one over a single bin of it the lower ten.
constexpr int kFine = 10, kCodes = kBins << kFine;
__device__ __forceinline__ int weight_code(float d, float a32) {
    return __float_as_int(fminf(d * a32 * 16384.0f, (float)(kCodes - 1)) + 8388608.0f) - __float_as_int(8388608.0f);
}
// Weights in the middle of bins: of codes first + b step .. first + (b + 1) step - 1; of keys from top - (b << shift) down to the
// next bin's.
struct CodeBins {
    int first, step;
    __device__ __forceinline__ double operator()(int b) const {
        return (double)ardiff::ex2(-((float)(first + b * step) + 0.5f * (float)(step - 1)) * 0.00006103515625f);
    }
};
struct KeyBins {
    unsigned top, bottom;
    int shift;
    float m, a32;
    __device__ __forceinline__ double operator()(int b) const {
        const unsigned down = ((unsigned)b << shift) + (shift ? 1u << (shift - 1) : 0u);
        return (double)ardiff::ex2((value_of(top - min(down, top - bottom)) - m) * a32);
    }
};

__device__ __forceinline__ void clear_bins(Shared& s) { reinterpret_cast<uint4*>(s.hist)[threadIdx.x] = uint4(); }
__device__ __forceinline__ void count_bin(Shared& s, int b) { atomicAdd(&s.hist[b], 1u); }
// The calling thread's bins of all CTAs' histograms, kEach * threadIdx.x and the ones behind it.
template <typename T>
__device__ __forceinline__ void gather_bins(const Part<T>& a, unsigned (&c)[kEach]) {
    uint4 q[kMaxParts];
#pragma unroll
    for (int p = 0; p < kMaxParts; ++p) {                    // (all loads before the first sum: another CTA's bins are far away)
        q[p] = uint4();
        if (p < a.parts) q[p] = reinterpret_cast<const uint4*>(a.at(a.s->hist, p))[threadIdx.x];
    }
#pragma unroll
    for (int p = 0; p < kMaxParts; ++p) c[0] += q[p].x, c[1] += q[p].y, c[2] += q[p].z, c[3] += q[p].w;
}

// What a histogram says about where a prefix ends: the bins, first to last (larger logits first), that hold its last element, the
// elements before them and in them, and the mass before them by the bins' middles.
struct Range {
    int first, last;
    unsigned before, in;
    double mass;
};

// Adds up the CTAs' histograms and picks the bin in which the count passes k (count), the estimated mass `enough`, or the count half of
// all (half: where estimates did not help). A bin that was found by an estimate comes with its neighbours, as far as the list
// has room; if it has none, with `spread` of them on either side. before, mass: in front of the histogram; whole: the exact mass of all
// that was counted, if it is known (then the estimates come from behind, where bins hold many elements each and their middles err
// little), else negative. middle(b): a weight of bin b. False: there is nothing.
template <typename T, typename F>
__device__ __noinline__ bool pick(const Part<T> a, const bool count, unsigned k, double enough, bool half, int spread, unsigned before,
                                  double mass, double whole, const F middle, Range& r) {
    Shared& s = *a.s;
    const int b0 = kEach * threadIdx.x;
    unsigned c[kEach] = {}, own = 0, total;
    gather_bins(a, c);
#pragma unroll
    for (int i = 0; i < kEach; ++i) own += c[i];
    if (threadIdx.x == 0) {
        s.found = s.pick_first = INT_MAX;
        s.last = s.pick_last = -1;
    }
    unsigned n[kEach + 1];
    double m[kEach + 1];
    n[0] = before + cta_scan(s, own, &total);
#pragma unroll
    for (int i = 0; i < kEach; ++i) n[i + 1] = n[i] + c[i];
    m[0] = mass;
    if (total == 0u) return false;
    if (count && before + total < k) {                       // not as many
        r = Range{0, 0, before, total, 0.0};
        return true;
    }
    if (count || half) {
        const unsigned goal = count ? k : before + (total + 1) / 2;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (n[i] < goal && n[i + 1] >= goal) s.found = b0 + i;
            m[i + 1] = mass;
        }
    } else {
        double w[kEach], sum = 0.0, all;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            w[i] = c[i] ? c[i] * middle(b0 + i) : 0.0;
            sum += w[i];
        }
        m[0] = cta_scan(s, sum, &all);
        m[0] += whole >= 0.0 ? whole - all : mass;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            m[i + 1] = m[i] + w[i];
            if (c[i]) {
                atomicMax(&s.last, b0 + i);
                if (m[i + 1] >= enough) atomicMin(&s.found, b0 + i);
            }
        }
    }
    __syncthreads();
    const int found = s.found != INT_MAX ? s.found : s.last;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (found == b0 + i) s.pick_before = n[i], s.pick_after = n[i + 1];
    __syncthreads();
    const unsigned lo = s.pick_before, hi = s.pick_after, in = hi - lo;
    const unsigned more = count || in > (unsigned)kList ? 0u : min(((unsigned)kList - in) / 2, 64u);
    if (more == 0u) {
        if (threadIdx.x == 0) {
            s.pick_first = max(found - spread, 0);
            s.pick_last = min(found + spread, kBins - 1);
        }
    } else {                                                 // (empty bins at either end come along)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (b0 + i <= found && n[i] + more >= lo) atomicMin(&s.pick_first, b0 + i);
            if (b0 + i >= found && n[i + 1] <= hi + more) atomicMax(&s.pick_last, b0 + i);
        }
    }
    __syncthreads();
    r.first = s.pick_first;
    r.last = s.pick_last;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (r.first == b0 + i) s.pick_before = n[i], s.mass_above = m[i];
        if (r.last == b0 + i) s.pick_after = n[i + 1];
    }
    __syncthreads();
    r.before = s.pick_before;
    r.in = s.pick_after - r.before;
    r.mass = s.mass_above;
    return true;
}

// w where `in`, 0 elsewhere: as a product, so that the weights of neighbouring values are formed side by side and none in a branch of its
// own (which the compiler makes of a selection: 2.5 times as slow).
__device__ __forceinline__ double masked(double w, bool in) { return w * __hiloint2double(in ? 0x3ff00000 : 0, 0); }

// What the sums over segments add up, value by value.
struct Bulk {                            // all weights
    Weights wt;
    __device__ __forceinline__ double operator()(float v, int) const { return wt.bulk(v); }
};
struct Drawn {                           // the weights of what is kept, exactly; floor: below it none has min_p (all halved)
    Weights wt;
    Cut cut;
    float half, a32, floor;
    double mp;
    __device__ __forceinline__ double operator()(float v, int i) const {
        if (!cut.keeps(v, i) || !((0.5f * v - half) * a32 >= floor)) return 0.0;
        const double w = wt.own(v);
        return w >= mp ? w : 0.0;
    }
};
struct Kept {                            // the weights of what the cut keeps
    Weights wt;
    Cut cut;
    __device__ __forceinline__ double operator()(float v, int i) const {
        return masked(wt.bulk(v), cut.keeps(v, i));
    }
};
struct KeptMin {                         // the same of those that have min_p, where min_p is a weight that bulk() gives exactly
    Weights wt;
    Cut cut;
    double mp;
    __device__ __forceinline__ double operator()(float v, int i) const {
        const double w = wt.bulk(v);
        return masked(w, cut.keeps(v, i) && w >= mp);
    }
};
template <bool FAR>
struct Counted {                         // the same, with a histogram of the weights (all but the last bin)
    Weights wt;
    Cut cut;
    float m, a32;
    unsigned* hist;
    __device__ __forceinline__ double operator()(float v, int i) const {
        const double w = FAR ? wt.own(v) : wt.bulk(v);
        const bool in = cut.keeps(v, i);
        const int b = weight_code(m - v, a32) >> kFine;
        if (in && b < kBins - 1) atomicAdd(&hist[b], 1u);
        return masked(w, in);
    }
};
struct AboveValue {                      // the weights above a value
    Weights wt;
    Cut cut;
    float top;
    __device__ __forceinline__ double operator()(float v, int i) const { return v > top && cut.keeps(v, i) ? wt.own(v) : 0.0; }
};
struct Equal {                           // the number of elements of a value
    Cut cut;
    float value;
    __device__ __forceinline__ double operator()(float v, int i) const { return v == value && cut.keeps(v, i) ? 1.0 : 0.0; }
};

enum Verdict { kFound, kAbove, kBelow, kUnknown, kNotNeeded };

// The first CTA alone: where in the sorted list (n entries, the elements next to `sure` in mass, or the nth in number) the prefix ends.
// s.verdict: kFound, and s.cut its last element (count = false: also s.found, its place in the list); or it lies above the list, or below.
__device__ __noinline__ void end_in_list(Shared& s, const Weights wt, const bool count, int n, unsigned nth, double sure, double enough) {
    sort_list(s, n);
    if (count) {
        if (threadIdx.x == 0) {
            const unsigned long long e = s.list[nth];
            s.cut = Cut{entry_value(e), (int)(unsigned)e};
            s.verdict = kFound;
        }
        return;
    }
    if (threadIdx.x == 0) s.found = INT_MAX;
    const int j0 = kEach * threadIdx.x;
    double w[kEach], own = 0.0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        w[i] = j0 + i < n ? wt.own(entry_value(s.list[j0 + i])) : 0.0;
        own += w[i];
    }
    double run = sure + cta_scan(s, own, &all);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        run += w[i];
        if (j0 + i < n && run >= enough) atomicMin(&s.found, j0 + i);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s.mass_in = sure + all;
        s.verdict = sure >= enough ? kAbove : s.found == INT_MAX ? kBelow : kFound;
        if (s.verdict == kFound) {
            const unsigned long long e = s.list[s.found];
            s.cut = Cut{entry_value(e), (int)(unsigned)e};
        }
    }
    __syncthreads();
}

// The search for a prefix's last element among what `cut` keeps, by the logits as whole numbers: the k-th (count), or the first at which
// the mass reaches `enough`. Histograms narrow the range of numbers until few elements are in it or all are equal; an exact pass
// sums what lies above, and a range that an estimate got wrong is done with, together with everything on its far side.
template <typename T>
__device__ __noinline__ Cut search(const Part<T> a, const Weights wt, float a32, const Cut cut, const bool count, unsigned k, double enough,
                                   int& buf) {
    Shared& s = *a.s;
    const float m = (float)wt.m;
    unsigned lo_key = key_of(-INFINITY) + 1, hi_key = key_of(m);         // where the element can be; masked logits are none
    double hi_mass = 0.0;                                                // above hi_key
    // The range shrinks to one bin of the histogram before it, or fits the list, at every step of the inner loop; of the outer one
    // half of the elements or more are done with, from the third time on.
    for (int turn = 0; turn < 64; ++turn) {
        unsigned kmin = lo_key, kmax = hi_key;
        Range r{0, 0, 0u, UINT_MAX, hi_mass};
        while (r.in == UINT_MAX || (r.in > (unsigned)kList && kmin < kmax)) {
            int shift = 0;
            while (((kmax - kmin) >> shift) >= (unsigned)kBins) ++shift;
            a.sync();                                        // the last histograms have been read
            clear_bins(s);
            __syncthreads();
            a.each([&](float x, int i) {
                const unsigned q = key_of(x);
                if (q >= kmin && q <= kmax && cut.keeps(x, i)) count_bin(s, (int)((kmax - q) >> shift));   // largest first
            });
            a.sync();
            const bool any = pick(a, count, k, enough, turn > 1, 0, r.before, r.mass, -1.0, KeyBins{kmax, kmin, shift, m, a32}, r);
            if (!any || (count && r.before + r.in < k)) {    // nothing there: all above it is kept; or all of fewer than k
                a.sync();
                return count ? cut : Cut{value_of(hi_key + 1), INT_MAX};
            }
            const unsigned top = kmax - ((unsigned)r.first << shift);
            const unsigned long long below = (unsigned long long)(r.last + 1) << shift;      // (up to 2^32)
            if (kmax - kmin >= below) kmin = kmax - (unsigned)below + 1;
            kmax = top;
        }
        // the exact sum above the range; the range's elements to the first CTA
        const float top = value_of(kmax), bottom = value_of(kmin);
        const bool ties = r.in > (unsigned)kList;
        a.sync();
        if (threadIdx.x == 0) s.count = 0u;
        a.sync();
        double sure = 0.0;
        if (!count) sure = sum_segments(a, buf, 2.0, AboveValue{wt, cut, top});
        if (!ties) {
            a.each([&](float x, int i) {
                if (x >= bottom && x <= top && cut.keeps(x, i)) {
                    const unsigned at = atomicAdd(a.at(&s.count, 0), 1u);
                    if (at < (unsigned)kList) *a.at(&s.list[at], 0) = entry(x, i);
                }
            });
            a.sync();
            if (a.rank == 0) end_in_list(s, wt, count, (int)min(s.count, (unsigned)kList), k - r.before - 1, sure, enough);
        } else {
            // one value, more often than the list is long: as many of it as are needed, lowest indices first
            const double w = count ? 1.0 : wt.own(top);
            const double need = count ? (double)(k - r.before) : ardiff::needed(enough, sure, w, r.in);
            const int verdict = count ? kFound : sure >= enough ? kAbove : need > (double)r.in ? kBelow : kFound;
            // (the sum over all is r.in: the share of it is a whole number less a half, up to rounding)
            sum_segments(a, buf, (need - 0.5) / (double)r.in, Equal{cut, top});
            const int owner = s.owner / kSegments;
            if (verdict == kFound && owner == a.rank) {
                const int at = locate(a, s.owner, s.before, need - 0.5, Equal{cut, top});
                if (threadIdx.x == 0) s.cut = Cut{top, at};
            }
            a.sync();
            if (a.rank == 0 && threadIdx.x == 0) {
                if (verdict == kFound) s.cut = Cut{top, a.at(&s.cut, owner)->index};
                s.verdict = verdict;
                s.mass_in = sure + r.in * w;
            }
        }
        a.sync();
        const int verdict = *a.at(&s.verdict, 0);
        const Cut found{a.at(&s.cut, 0)->value, a.at(&s.cut, 0)->index};
        const double with = *a.at(&s.mass_in, 0);
        a.sync();
        if (verdict == kFound) return found;
        if (verdict == kAbove) {
            lo_key = kmax + 1;
        } else {
            hi_key = kmin - 1;
            hi_mass = with;
        }
        if (lo_key > hi_key) break;                          // sums that differ in their last bit
    }
    return Cut{value_of(hi_key + 1), INT_MAX};
}

// The first pass: the groups' largest logits and, with SUMS, the sums of the segments, relative to the largest of the first few (s.ref: the
// part's own, so that the row is read only once; a weight may be above 1 then).
template <typename T, bool SUMS>
__device__ __forceinline__ void first_pass(const Part<T>& a, const double scale) {
    constexpr int N = Part<T>::N;
    Shared& s = *a.s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    Weights wt{};
    if (SUMS) {
        float ref = -INFINITY;
        a.template scan<1>(warp * kGroups * a.segment + lane, min(a.pieces, warp * kGroups * a.segment + min(32, a.segment)), 32,
                           [&](const uint4& q, int) { ref = fmaxf(ref, ardiff::piece_max(q, T())); });
#pragma unroll
        for (int q = 16; q > 0; q >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, q));
        if (lane == 0) s.warp_max[warp] = ref;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) ref = fmaxf(ref, s.warp_max[w]);
        ref = fminf(fmaxf(ref, -kSane), kSane);
        if (tid == 0) s.ref = ref;
        wt.m = ref;
        wt.a = scale;
        wt.lowest = (float)(wt.m - 100.0 / scale);
    }
#pragma unroll 1
    for (int g = 0; g < kGroups; ++g) {
        const int at = warp * kGroups + g;
        float top = -INFINITY;
        double acc[2] = {0.0, 0.0};
        a.template scan<SUMS ? 2 : 4>(at * a.segment + lane, min(a.pieces, (at + 1) * a.segment), 32, [&](const uint4& q, int) {
            top = max_nan(top, ardiff::piece_max(q, T()));
            if (SUMS) {
                float v[N];
                ardiff::unpack(q, v, T());
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i & 1] += wt.bulk(v[i]);
            }
        });
        s.top[g][tid] = top;
        if (SUMS) {
            const double mine = warp_sum(acc[0] + acc[1]);
            if (lane == 0) s.seg[0][at] = mine;
        }
    }
}

// The sums of the weights above a range of codes, over the segments; what is in the range goes to the list of the first CTA (*count, list;
// NULL: it does not).
template <typename T>
__device__ __noinline__ double sum_above(const Part<T> a, const int buf, const Weights wt, const Cut cut, const float m, const float a32,
                                         const int first, const int last, unsigned* count, unsigned long long* list) {
    constexpr int N = Part<T>::N;
    Shared& s = *a.s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
    for (int g = warp * kGroups; g < (warp + 1) * kGroups; ++g) {
        double acc[2] = {0.0, 0.0};
        a.template scan<2>(g * a.segment + lane, min(a.pieces, (g + 1) * a.segment), 32, [&](const uint4& q, int p) {
            unsigned hit = 0;
#pragma unroll 1
            for (int h = 0; h < N; h += 4) {                 // (as above)
                float v[4];
                ardiff::unpack4(q, h, v, T());
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int code = weight_code(m - v[i], a32);
                    const bool in = cut.keeps(v[i], a.first + p * N + h + i);
                    acc[i & 1] += masked(wt.bulk(v[i]), in && code < first);
                    hit |= in && code >= first && code <= last ? 1u << (h + i) : 0u;
                }
            }
            if (hit && count) {
#pragma unroll 1
                for (; hit; hit &= hit - 1) {
                    const int index = a.first + p * N + __ffs(hit) - 1;
                    const unsigned place = atomicAdd(count, 1u);
                    if (place < (unsigned)kList) list[place] = entry(ardiff::to_float(a.x[index]), index);
                }
            }
        });
        const double mine = warp_sum(acc[0] + acc[1]);
        if (lane == 0) s.seg[buf][g] = mine;
    }
    return add_segments(a, buf, 2.0, false, Weights());
}

// The first CTA: the draw's segment, where the sum over segment g (of all CTAs') is in_segment(g); a thread a segment.
template <typename T, typename F>
__device__ __forceinline__ void draw_segment(const Part<T>& a, double u, F&& in_segment) {
    static_assert(kMaxParts * kSegments <= kThreads, "a thread a segment");
    Shared& s = *a.s;
    const int g = threadIdx.x;
    const double own = g < a.parts * kSegments ? in_segment(g) : 0.0;
    double total;
    const double before = cta_scan(s, own, &total);
    if (g == 0) {
        s.found = INT_MAX;
        s.last = -1;
    }
    __syncthreads();
    if (own > 0.0) {
        atomicMax(&s.last, g);
        if (before + own > u * total) atomicMin(&s.found, g);
    }
    __syncthreads();
    if (g == (s.found != INT_MAX ? s.found : s.last)) {
        s.owner = g;
        s.before = before;
        s.total = total;
    }
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) sample_kernel(const Args args) {
    constexpr int N = ardiff::Piece<T>::N;
    __shared__ Shared s;
    ardiff::begin_kernel();
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
    // the aligned pieces that cover the row; `shift` places in front of it belong to none of them
    a.x = static_cast<const T*>(args.x) + row * args.ld;
    const int shift = (int)((reinterpret_cast<uintptr_t>(a.x) & 15u) / sizeof(T));
    const int pieces = (shift + args.V + N - 1) / N;
    const int per = (pieces + a.parts - 1) / a.parts;
    const int p0 = min(pieces, a.rank * per);
    a.pieces = min(pieces, p0 + per) - p0;
    a.segment = (a.pieces + kSegments - 1) / kSegments;
    a.first = p0 * N - shift;
    a.whole0 = a.first < 0 ? 1 : 0;
    a.whole1 = max(a.whole0, min(a.pieces, (args.V - a.first) / N));
    // the first pass sums, too, where all weights count and the temperature is one for which fp32 tells which logits are far below
    const bool greedy = o.T == 0.f;
    const double scale = 1.4426950408889634074 / (double)o.T;
    const bool sums = valid && o.u >= kLeastU && o.T >= 1e-3f && o.T <= 1e3f && !o.use_k && (o.use_p ? args.V > kList : !o.use_m);
    if (sums) first_pass<T, true>(a, scale);
    else first_pass<T, false>(a, scale);
    float own = s.top[0][tid];
#pragma unroll
    for (int g = 1; g < kGroups; ++g) own = max_nan(own, s.top[g][tid]);
    __syncthreads();
#pragma unroll
    for (int q = 16; q > 0; q >>= 1) own = max_nan(own, __shfl_xor_sync(0xffffffffu, own, q));
    if (lane == 0) s.warp_max[warp] = own;
    if (tid == 0) {
        s.count = 0u;
        s.first = INT_MAX;
    }
    __syncthreads();
    own = s.warp_max[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) own = max_nan(own, s.warp_max[w]);
    if (greedy)                                              // the lowest index of this part's largest
        collect(a, Listed{Listed::EQUAL, 0.f, own, 0.f, 0.f}, (unsigned*)nullptr, (unsigned long long*)nullptr, &s.first);
    if (tid == 0) s.cta_max = own;
    a.sync();
    float m = own, ref = sums ? s.ref : 0.f;                  // of all parts; the lowest reference
#pragma unroll
    for (int r = 0; r < kMaxParts; ++r) {
        if (r < a.parts) {
            m = max_nan(m, *a.at(&s.cta_max, r));
            if (sums) ref = fminf(ref, *a.at(&s.ref, r));
        }
    }
    if (!valid || !(fabsf(m) < INFINITY) || greedy) {
        if (a.rank == 0 && tid == 0) {
            int token = -1;
            if (valid && fabsf(m) < INFINITY) {
                token = INT_MAX;
                for (int r = 0; r < a.parts; ++r)
                    if (*a.at(&s.cta_max, r) == m) token = min(token, *a.at(&s.first, r));
            }
            answer(args, row, token, token >= 0 ? 0.f : NAN);
        }
        a.sync();
        return;
    }
    Weights wt;
    wt.m = m;
    wt.a = scale;
    wt.lowest = (float)fmax(wt.m - 100.0 / wt.a, -3e38);
    const double octaves = ((double)wt.lowest - wt.m) * wt.a;
    wt.far = o.u < kLeastU || octaves > -95.0 || octaves < -900.0;
    const float a32 = (float)fmin(wt.a, 3e38);
    const float half = 0.5f * m;                             // (halves: a difference of two logits can pass fp32's range)
    const float floor_ = o.use_m ? 0.5f * (log2f(o.mp) - 0.01f) : -INFINITY;
    // (what is too far above a part's reference has overflowed)
    const bool summed = sums && fabsf(m) <= kSane && ((double)m - (double)ref) * scale <= 900.0;
    int buf = 0;
    Drawn drawn{wt, no_cut(), half, a32, floor_, o.use_m ? (double)o.mp : 0.0};
    Cut& cut = drawn.cut;
    int owner = -1;                                          // the draw's segment, where the search for the cut finds it
    double before = 0.0, total = 0.0;
    if (o.use_k || o.use_p || o.use_m) {
        // which logits a list of all that may be kept has to hold, if there is a list
        Listed listed{Listed::ALL, m, 0.f, half, a32};
        bool list = true;
        Range r;
        int last_code = 0;                                   // of a nucleus' end
        double whole = -1.0;
        if (args.V > kList) {
            list = false;
            if (o.use_p && !o.use_k) {
                if (summed) whole = add_segments(a, buf, 2.0, true, wt);
                else if (wt.far) whole = sum_segments(a, buf, 2.0, AboveValue{wt, cut, -INFINITY});
                else whole = sum_segments(a, buf, 2.0, Bulk{wt});
            }
            // by the groups' largest logits: at least k logits are not below the k-th of them, and the mass down to one of them is at
            // least theirs (in whole steps of 2^-18, rounded down)
            clear_bins(s);
            if (tid == 0) s.found = INT_MAX;
            __syncthreads();
            unsigned groups = 0;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const float v = s.top[g][tid];
                if (o.use_k || o.use_p) {
                    const int b = distance_bin(m - v);
                    if (b < kBins - 1)
                        atomicAdd(&s.hist[b], o.use_k ? 1u : (unsigned)(0.9999f * 262144.0f * ardiff::ex2((v - m) * a32)));
                } else {
                    groups += __syncthreads_count((0.5f * v - half) * a32 >= floor_);
                }
            }
            if (tid == 0) s.groups = groups;
            a.sync();
            if (o.use_k || o.use_p) {
                unsigned c[kEach] = {}, all;
                gather_bins(a, c);
                unsigned n = cta_scan(s, (c[0] + c[1]) + (c[2] + c[3]), &all);
                const double goal = o.use_k ? (double)o.k : fmax((double)o.p * whole * 262144.0, 1.0);
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    if ((double)n < goal && (double)(n + c[i]) >= goal) s.found = kEach * tid + i;
                    n += c[i];
                }
                __syncthreads();
                if (s.found != INT_MAX) {
                    list = true;
                    listed.which = Listed::REACH;
                    listed.bound = distance_edge(s.found + 1);
                }
            } else {                                         // a list has no room for more groups than it has entries
                for (int p = 0; p < a.parts; ++p) groups = p == 0 ? *a.at(&s.groups, 0) : groups + *a.at(&s.groups, p);
                list = groups <= (unsigned)kList;
                listed.which = Listed::WEIGHT;
                listed.bound = floor_;
            }
            a.sync();                                        // the others' bins have been read
        }
        if (list) {
            const unsigned* count = a.at(&s.count, 0);
            collect(a, listed, a.at(&s.count, 0), a.at(s.list, 0), (int*)nullptr);
            a.sync();
            const unsigned n = *count;
            a.sync();
            if (n <= (unsigned)kList) {
                if (a.rank == 0) finish_list(args, row, s, wt, o, (int)n, whole);
                return;
            }
        }
        if (o.use_k) {
            // the k-th by a histogram over all logits, and a list of its bin
            __syncthreads();
            clear_bins(s);
            if (tid == 0) s.count = 0u;
            __syncthreads();
            a.each([&](float v, int) { if (v > -INFINITY) count_bin(s, distance_bin(m - v)); });
            a.sync();
            pick(a, true, (unsigned)o.k, 0.0, false, 0, 0u, 0.0, -1.0, CodeBins{0, 1}, r);
            if (r.before + r.in >= (unsigned)o.k) {          // (else there are fewer than k)
                if (r.in <= (unsigned)kList) {
                    unsigned* count = a.at(&s.count, 0);
                    unsigned long long* list = a.at(s.list, 0);
                    a.each([&](float v, int i) {
                        if (v > -INFINITY && distance_bin(m - v) == r.first) list[atomicAdd(count, 1u)] = entry(v, i);
                    });
                    a.sync();
                    if (a.rank == 0) end_in_list(s, wt, true, (int)r.in, (unsigned)o.k - r.before - 1, 0.0, 0.0);
                    a.sync();
                    cut = Cut{a.at(&s.cut, 0)->value, a.at(&s.cut, 0)->index};
                } else {
                    cut = search(a, wt, a32, cut, true, (unsigned)o.k, 0.0, buf);
                }
            }
            a.sync();
        }
        if (o.use_p) {
            // a histogram that says about where the nucleus ends
            clear_bins(s);
            __syncthreads();
            if (o.use_k) {
                if (wt.far) whole = sum_segments(a, buf, 2.0, Counted<true>{wt, cut, m, a32, s.hist});
                else whole = sum_segments(a, buf, 2.0, Counted<false>{wt, cut, m, a32, s.hist});
            } else {
                a.each([&](float v, int) {
                    const int b = weight_code(m - v, a32) >> kFine;
                    if (b < kBins - 1) count_bin(s, b);
                });
                a.sync();
            }
            pick(a, false, 0u, (double)o.p * whole, false, 1, 0u, 0.0, whole, CodeBins{0, 1 << kFine}, r);
            r.last = min(r.last, kBins - 2);                 // (the last bin was not counted)
            last_code = (r.last << kFine) + (1 << kFine) - 1;
            const double enough = fmax((double)o.p * whole, 1e-300);                  // at least one
            int first_code = r.first << kFine;
            bool window = r.in > 2 * kThreads;               // first_code .. last_code want a histogram of their own
            int verdict = kAbove;
            for (int turn = 0; (verdict == kAbove || verdict == kBelow) && turn < 6; ++turn) {
                if (window) {
                    int shift = 0;
                    while ((last_code - first_code) >> shift >= kBins) ++shift;
                    a.sync();                                    // the last histogram has been read
                    clear_bins(s);
                    __syncthreads();
                    // with it the mass in front of them, in fp32: bins' middles then err by what lies in the window alone (where many logits
                    // are equal, middles in front of it put many rows' ends beside the right bin, and those go round again: 512 x 131072
                    // bf16, flat nuclei, 606 -> 488 us)
                    float sum = 0.f;
                    a.each([&](float v, int i) {
                        const int code = weight_code(m - v, a32);
                        const bool in = cut.keeps(v, i);
                        if (in && code >= first_code && code <= last_code) count_bin(s, (code - first_code) >> shift);
                        const float w = ardiff::ex2((v - m) * a32);
                        sum += in && code < first_code ? w : 0.f;
                    });
                    const double mine = warp_sum(sum);
                    buf ^= 1;
                    if (lane < kGroups) s.seg[buf][warp * kGroups + lane] = lane == 0 ? mine : 0.0;
                    const double base = add_segments(a, buf, 2.0, false, Weights());
                    if (!pick(a, false, 0u, enough, false, 0, 0u, base, -1.0, CodeBins{first_code, 1 << shift}, r)) break;
                    last_code = min(last_code, first_code + ((r.last + 1) << shift) - 1);
                    first_code += r.first << shift;
                }
                // the sum of what lies above the range; a list of what lies in it, or, where that is more than a list holds, whether it is
                // one value, and how often in which segment
                const bool listed = r.in <= (unsigned)kList;
                a.sync();
                if (tid == 0) {
                    s.count = 0u;
                    s.kmin = UINT_MAX;
                    s.kmax = 0u;
                    s.verdict = kUnknown;
                }
                a.sync();
                double sure = 0.0;
                if (!wt.far) {
                    buf ^= 1;
                    sure = sum_above(a, buf, wt, cut, m, a32, first_code, last_code, listed ? a.at(&s.count, 0) : nullptr, a.at(s.list, 0));
                }
                if (listed && !wt.far && a.rank == 0) {
                    const int n = (int)min(s.count, (unsigned)kList);
                    end_in_list(s, wt, false, n, 0u, sure, enough);
                    if (s.verdict == kFound) {
                        const int kept = s.found + 1;
                        const bool above = o.use_m && wt.own(entry_value(s.list[0])) < (double)o.mp;
                        __syncthreads();                         // s.verdict and s.found have been read
                        // what is kept of the list, in order of index
                        unsigned long long e[kEach];
#pragma unroll
                        for (int i = 0; i < kEach; ++i) e[i] = s.list[kEach * tid + i];
                        __syncthreads();
#pragma unroll
                        for (int i = 0; i < kEach; ++i) {
                            const int j = kEach * tid + i;
                            if (j < kept) {
                                const double w = wt.own(entry_value(e[i]));
                                s.list[j] = (e[i] & 0xffffffffull) << 32 | (unsigned)j;
                                s.w[j] = o.use_m && w < (double)o.mp ? 0.0 : w;
                            }
                        }
                        __syncthreads();
                        sort_list(s, kept);
                        draw_segment(a, (double)o.u, [&](int g) {
                            // the entries from the segment's first index on, up to the next one's
                            const int q0 = min(pieces, g / kSegments * per), mine = min(pieces, q0 + per) - q0;
                            const int len = (mine + kSegments - 1) / kSegments, at = g % kSegments * len;
                            const int begin = (q0 + min(mine, at)) * N - shift, end = (q0 + min(mine, at + len)) * N - shift;
                            int lo = 0, hi = kept;
                            while (lo < hi) {
                                const int mid = (lo + hi) >> 1;
                                if ((int)(s.list[mid] >> 32) < begin) lo = mid + 1; else hi = mid;
                            }
                            double sum = *a.at(&s.seg[buf][g % kSegments], g / kSegments);
                            for (; lo < kept && (int)(s.list[lo] >> 32) < end; ++lo) sum += s.w[(unsigned)s.list[lo]];
                            return sum;
                        });
                        if (tid == 0) s.verdict = above ? kNotNeeded : kFound;
                    }
                }
                double need = 0.0;
                float value = 0.f;
                if (!listed && !wt.far) {
                    unsigned lo = UINT_MAX, hi = 0u;
                    for (int g = warp * kGroups; g < (warp + 1) * kGroups; ++g) {
                        unsigned n = 0;
                        a.template scan<1>(g * a.segment + lane, min(a.pieces, (g + 1) * a.segment), 32, [&](const uint4& q, int p) {
                            float v[N];
                            ardiff::unpack(q, v, T());
#pragma unroll
                            for (int i = 0; i < N; ++i) {
                                const int code = weight_code(m - v[i], a32);
                                if (code >= first_code && code <= last_code && cut.keeps(v[i], a.first + p * N + i)) {
                                    ++n;
                                    lo = min(lo, key_of(v[i]));
                                    hi = max(hi, key_of(v[i]));
                                }
                            }
                        });
                        n = __reduce_add_sync(0xffffffffu, n);
                        if (lane == 0) s.seg_ties[g] = n;
                    }
                    lo = __reduce_min_sync(0xffffffffu, lo);
                    hi = __reduce_max_sync(0xffffffffu, hi);
                    if (lane == 0) {
                        atomicMin(&s.kmin, lo);
                        atomicMax(&s.kmax, hi);
                    }
                    a.sync();
                    lo = UINT_MAX, hi = 0u;
                    for (int p = 0; p < a.parts; ++p) {
                        lo = min(lo, *a.at(&s.kmin, p));
                        hi = max(hi, *a.at(&s.kmax, p));
                    }
                    value = value_of(lo);
                    const double w = wt.own(value);
                    need = ardiff::needed(enough, sure, w, r.in);
                    if (lo == hi && a.rank == 0 && tid == 0) {
                        s.verdict = sure >= enough ? kAbove : need > (double)r.in ? kBelow : kFound;
                        s.mass_in = sure + r.in * w;
                    }
                    if (lo == hi && sure < enough && need <= (double)r.in && a.rank == 0) {
                        const unsigned ties = tid < a.parts * kSegments ? *a.at(&s.seg_ties[tid % kSegments], tid / kSegments) : 0u;
                        unsigned all;
                        const unsigned ahead = cta_scan(s, ties, &all);
                        draw_segment(a, (double)o.u, [&](int g) {
                            const double kept = fmin(fmax(need - (double)ahead, 0.0), (double)ties);
                            return *a.at(&s.seg[buf][g % kSegments], g / kSegments) + w * kept;
                        });
                        if (tid == s.owner) s.cut_ahead = ahead;
                        if (tid == 0 && o.use_m && w < (double)o.mp) s.verdict = kNotNeeded;
                    }
                }
                a.sync();
                verdict = *a.at(&s.verdict, 0);
                if (verdict == kFound) {
                    owner = *a.at(&s.owner, 0);
                    before = *a.at(&s.before, 0);
                    total = *a.at(&s.total, 0);
                    if (listed) {
                        cut = Cut{a.at(&s.cut, 0)->value, a.at(&s.cut, 0)->index};
                    } else {
                        need -= (double)*a.at(&s.cut_ahead, 0);  // of this value in the draw's segment, lowest indices first
                    }
                }
                a.sync();
                if (verdict == kFound && owner / kSegments != a.rank) return;
                if (verdict == kFound && !listed) {
                    const unsigned ties = s.seg_ties[owner % kSegments];
                    int index = need <= 0.0 ? -1 : INT_MAX;
                    if (need > 0.0 && need < (double)ties) index = locate(a, owner, 0.0, need - 0.5, Equal{cut, value});
                    // (a cut before this one keeps all of the range or is its end)
                    cut = Cut{value, cut.value == value ? min(index, cut.index) : index};
                }
                // the estimate was wrong: the same with a window beside it
                window = true;
                if (verdict == kAbove) {
                    last_code = first_code - 1;
                    first_code = max(0, last_code - 4095);
                } else {
                    first_code = last_code + 1;
                    last_code = min(first_code + 4095, ((kBins - 1) << kFine) - 1);
                }
            }
            if (verdict != kFound && verdict != kNotNeeded) cut = search(a, wt, a32, cut, false, 0u, enough, buf);
        }
    }
    // the draw among what the cut keeps
    if (owner < 0) {
        if (wt.far || (o.use_m && o.mp < kLeastMin)) total = sum_segments(a, buf, (double)o.u, drawn);
        else if (o.use_m) total = sum_segments(a, buf, (double)o.u, KeptMin{wt, cut, (double)o.mp});
        else if (o.use_k || o.use_p) total = sum_segments(a, buf, (double)o.u, Kept{wt, cut});
        else if (summed) total = add_segments(a, buf, (double)o.u, true, wt);
        else total = sum_segments(a, buf, (double)o.u, Bulk{wt});
        owner = s.owner;
        before = s.before;
        a.sync();                                            // every CTA has read the others' sums
        if (owner / kSegments != a.rank) return;
    }
    int token = locate(a, owner, before, (double)o.u * total, drawn);
    if (token < 0) token = nearest(a, a.first + owner % kSegments * a.segment * N, drawn);
    if (tid == 0) {
        const double y = ((double)ardiff::to_float(a.x[token]) - wt.m) * wt.a;
        answer(args, row, token, (float)(y * 0.69314718055994530942 - log(total)));
    }
}

template <typename T>
int launch(Args a, int64_t n, cudaStream_t st) {
    // More CTAs a row while there is room for them and each keeps so many pieces that it gains: a list is one CTA's work, and the others
    // cost it meetings. us with 1 / 2 / 4 / 8 CTAs, 8 rows of bf16: top-k with top-p 16384 14.6 / 15.9 / 16.7 / 18.6, 32768 15.7 / 17.1 /
    // 16.2 / 17.5, 65536 19.0 / 17.7 / 17.4 / 17.1, 131072 25.6 / 20.2 / 17.8 / 18.1; no filter 8192 12.0 / 13.5 / 14.1 / 13.7, 16384 14.0 /
    // 13.9 / 13.6 / 14.5, 32768 17.3 / 16.0 / 14.1 / 14.0; nuclei alone 16384 51.6 / 47.0 / 45.7 / 47.2, 32768 75 / 60 / 51 / 50. The lists alone
    // would have twice as many pieces a CTA; but calls with top_k have rows without it, which lose more (64 x 65536, nuclei: 80 us
    // with four CTAs, 100 with two). Room: 64 rows of 131072 with no filter 23.9 with four CTAs, 26.5 with eight.
    const int64_t least = a.top_k ? 2048 : 1024;
    const int64_t pieces = ((int64_t)a.V + ardiff::Piece<T>::N - 1) / ardiff::Piece<T>::N;
    int parts = 1;
    while (parts < kMaxParts && n * parts < 148 * 2 && pieces >= 2 * parts * least) parts *= 2;
    a.parts = parts;
    const bool ok = ardiff::launch_early(sample_kernel<T>, (unsigned)(n * parts), kThreads, (unsigned)parts, 0, st, a);
    ardiff::set_launch_count(1);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
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
