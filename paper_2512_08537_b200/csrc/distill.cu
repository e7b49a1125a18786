// Distillation of a draft model from the largest logits that its target kept: for every row, with q the softmax of the
// teacher's entries over the temperature and p the softmax of the student's whole row over it,
//   loss = sum_j q_j (ln q_j - ln p[id_j]),      d loss / d x_i = (p_i [row has entries] - sum_{j: id_j = i} q_j) / T.
// Statistics kept for a backward pass are the row's largest value m and ln Z, Z = sum_i exp((x_i - m) / T): p_i is formed from
// x_i - m and not from x_i / T minus one rounded number, so that large logits cost no accuracy.
//
// A row belongs to a cluster of one to eight CTAs, a contiguous part each; their (m, Z) meet through distributed shared memory.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>

#include "../../include/ardiff.h"
#include "common.cuh"
#include "launch.cuh"
#include "rows.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int kCache = 60 * 1024;        // bytes of a part that are kept for the gradient: three CTAs an SM
enum Mode { FORWARD, STEP, BACKWARD };
template <int MODE> constexpr int kThreadsOf = MODE == STEP ? 512 : 256;
template <int MODE> constexpr int kAheadOf = MODE == FORWARD ? 8 : 4;        // pieces a thread has under way

struct Args {
    const void* x;
    const void* teacher;
    const int32_t* ids;
    const float* weight;         // STEP, BACKWARD
    float* loss;                 // FORWARD, STEP
    float* stats;                // out, or in for BACKWARD
    void* grad;                  // STEP, BACKWARD
    int64_t ld, ld_grad;
    int32_t teacher_type, V, k, parts;
    int32_t cached;              // STEP: pieces of a part that shared memory holds
    int32_t seen;                // STEP, BACKWARD: places of the ids' table, a power of two, at least twice k
    float inv_t;                 // 1 / T
};

__device__ __forceinline__ float load_teacher(const Args& a, int64_t i) {
    if (a.teacher_type == ARDIFF_F32) return static_cast<const float*>(a.teacher)[i];
    if (a.teacher_type == ARDIFF_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(a.teacher)[i]);
    return __half2float(static_cast<const __half*>(a.teacher)[i]);
}

struct MaxSum { float m, z; };   // largest value, sum of exp((x - m) / T)

// c = log2(e) / T. -inf is the largest value of nothing: its sum is 0 and it counts for nothing beside another.
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b, float c) {
    const float m = fmaxf(a.m, b.m);
    const float at = m == -INFINITY ? 0.f : m;
    return MaxSum{m, a.z * ardiff::ex2((a.m - at) * c) + b.z * ardiff::ex2((b.m - at) * c)};
}

// A thread's running largest value m and sum of exponentials above `ref`, which follows m a few octaves late. The sum is a compensated one
// (`lost`: what its last addition rounded off) of the pieces' sums: plain additions one after the other round the same way where
// many logits are equal, and 8192 of them are off by 4e-5 to 8e-5. And it is scaled only where a value is kLate octaves above `ref`:
// a row that rises slowly would else be scaled, and rounded, at every step.
struct Running {
    float m, ref, z, lost;
};
constexpr float kLate = 4.f;
template <typename T, int kAhead>
__device__ __forceinline__ void take(Running& s, const uint4 (&q)[kAhead], int n, float c) {
    constexpr int N = ardiff::Piece<T>::N;
    float top = ardiff::piece_max(q[0], T());
#pragma unroll
    for (int j = 1; j < kAhead; ++j)
        if (j < n) top = fmaxf(top, ardiff::piece_max(q[j], T()));
    s.m = fmaxf(s.m, top);
    if ((top - s.ref) * c > kLate) {
        const float down = ardiff::ex2((s.ref - top) * c);   // from -inf: 0
        s.z *= down;
        s.lost *= down;
        s.ref = top;
    }
    const float at = s.ref == -INFINITY ? 0.f : s.ref;
    const ardiff::Two minus = ardiff::two(-at, -at), c2 = ardiff::two(c, c);
    ardiff::Two sum = ardiff::two(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        if (j < n) {
            float v[N];
            ardiff::unpack(q[j], v, T());
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const float2 y = ardiff::apart((ardiff::two(v[i], v[i + 1]) + minus) * c2);
                sum = sum + ardiff::two(ardiff::ex2(y.x), ardiff::ex2(y.y));
            }
        }
    }
    const float2 sums = ardiff::apart(sum);
    const float more = sums.x + sums.y - s.lost, z = s.z + more;
    s.lost = z - s.z - more;
    s.z = z;
}

template <typename T, int MODE>
__global__ void __launch_bounds__(kThreadsOf<MODE>, MODE == FORWARD ? 4 : MODE == STEP ? 3 : 6) distill_kernel(const Args a) {
    constexpr int kThreads = kThreadsOf<MODE>, kWarps = kThreads / 32, kAhead = kAheadOf<MODE>;
    ardiff::begin_kernel();
    using ardiff::Row;
    constexpr int N = ardiff::Piece<T>::N;
    extern __shared__ __align__(16) unsigned char smem[];
    uint4* s_cache = reinterpret_cast<uint4*>(smem);         // [cached] pieces of this part
    float* s_q = reinterpret_cast<float*>(s_cache + a.cached);   // [k] teacher's logits, then probabilities
    float* s_x = s_q + a.k;                                  // [k] the student's logits there
    int32_t* s_id = reinterpret_cast<int32_t*>(s_x + a.k);   // [k] -1: no entry
    int32_t* s_seen = s_id + a.k;                            // [a.seen] ids, each at or behind the place that its bits point to
    __shared__ int s_again;                                  // whether an id occurs more than once
    __shared__ MaxSum s_part[kWarps], s_entries[kWarps];
    __shared__ MaxSum s_own;
    __shared__ float s_loss[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    const float c = a.inv_t * 1.4426950408889634f;
    const Row<T> x(static_cast<const T*>(a.x) + row * a.ld, a.V);
    const int per = (x.pieces + a.parts - 1) / a.parts;
    const int p0 = min(x.pieces, part * per), p1 = min(x.pieces, p0 + per);
    // the values of this part, as a range: what is before the first piece goes with the first part, what is behind with the last
    const int v0 = part == 0 ? 0 : x.lead + p0 * N, v1 = part == a.parts - 1 ? a.V : x.lead + p1 * N;
    T* grad = MODE == FORWARD ? nullptr : static_cast<T*>(a.grad) + row * a.ld_grad;

    // the first pieces are under way before anything is waited for
    const uint4* body = x.body();
    uint4 q[kAhead];
    int n_q = 0;
    auto load = [&](int p) {
        n_q = p < p1 ? min(kAhead, (p1 - p + kThreads - 1) / kThreads) : 0;
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (j < n_q) q[j] = ardiff::load_piece(body + p + j * kThreads);
    };
    if (MODE != BACKWARD) load(p0 + tid);
    if (MODE != FORWARD) {
        for (int j = tid; j < a.seen; j += kThreads) s_seen[j] = -1;
        if (tid == 0) s_again = 0;
    }
    bool some = false;
    for (int j = tid; j < a.k; j += kThreads) {
        int id = a.ids[row * a.k + j];
        const float t = load_teacher(a, row * a.k + j);
        if (id < 0 || id >= a.V || t == -INFINITY) id = -1;
        s_id[j] = id;
        s_q[j] = t;
        s_x[j] = id >= 0 && (MODE != BACKWARD || (id >= v0 && id < v1)) ? ardiff::to_float(x.x[id]) : 0.f;
        some |= id >= 0;
    }
    some = __syncthreads_or(some);
    if (!some) {                                             // nothing to learn from this row: its logits do not matter
        if (MODE != FORWARD)
            for (int i = v0 + tid; i < v1; i += kThreads) grad[i] = ardiff::from_float<T>(0.f);
        if (MODE != BACKWARD && part == 0 && tid == 0) {
            a.loss[row] = 0.f;
            a.stats[2 * row] = 0.f;
            a.stats[2 * row + 1] = 0.f;
        }
        return;                                              // every CTA of the cluster alike
    }
    // this thread's entries: their largest and the sum of their exponentials above it
    MaxSum t{-INFINITY, 0.f};
    const bool entries = warp * 32 < a.k;                    // this warp has some
    for (int j = tid; j < a.k; j += kThreads) {
        const int id = s_id[j];
        if (id < 0) continue;
        t = merge(t, MaxSum{s_q[j], 1.f}, c);
        if (MODE != FORWARD) {
            unsigned h = (unsigned)id * 2654435761u;
            for (;;) {                                       // (more places than ids)
                h &= (unsigned)(a.seen - 1);
                const int there = atomicCAS(&s_seen[h], -1, id);
                if (there == id) s_again = 1;
                if (there == id || there == -1) break;
                ++h;
            }
        }
    }
    auto reduce_entries = [&]() {
        if (!entries) return;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            t = merge(t, MaxSum{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.z, o)}, c);
        if (lane == 0) s_entries[warp] = t;
    };
    auto add_warps = [&](const MaxSum* w, int n) {           // every warp for itself, one value a lane
        MaxSum v = lane < n ? w[lane] : MaxSum{-INFINITY, 0.f};
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1)
            v = merge(v, MaxSum{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.z, o)}, c);
        return MaxSum{__shfl_sync(0xffffffffu, v.m, 0), __shfl_sync(0xffffffffu, v.z, 0)};
    };
    float m, ln_z, scale;
    if (MODE != BACKWARD) {
        Running run{-INFINITY, -INFINITY, 0.f, 0.f};
#pragma unroll 1
        for (int p = p0 + tid; n_q > 0; p += kAhead * kThreads) {
            if (MODE == STEP) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (j < n_q && p - p0 + j * kThreads < a.cached) s_cache[p - p0 + j * kThreads] = q[j];
            }
            take<T, kAhead>(run, q, n_q, c);
            load(p + kAhead * kThreads);
        }
        MaxSum s = merge(MaxSum{run.m, 0.f}, MaxSum{run.ref, run.z}, c);
        const int edge = part == 0 && tid < x.lead ? tid : part == a.parts - 1 && x.tail() + tid < a.V ? x.tail() + tid : -1;
        const int both = part == 0 && tid < x.lead && part == a.parts - 1 && x.tail() + tid < a.V ? x.tail() + tid : -1;
        if (edge >= 0) {
            const float v = ardiff::to_float(x.x[edge]);
            s = merge(s, MaxSum{v, 1.f}, c);
        }
        if (both >= 0) {
            const float v = ardiff::to_float(x.x[both]);
            s = merge(s, MaxSum{v, 1.f}, c);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            s = merge(s, MaxSum{__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.z, o)}, c);
        if (lane == 0) s_part[warp] = s;
        reduce_entries();
        __syncthreads();
        s = add_warps(s_part, kWarps);
        if (a.parts > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (tid == 0) s_own = s;
            cl.sync();
            s = *cl.map_shared_rank(&s_own, 0);
            for (int r = 1; r < a.parts; ++r) s = merge(s, *cl.map_shared_rank(&s_own, r), c);
        }
        m = s.m;
        if (m == -INFINITY || s.z != s.z) m = s.z = NAN;     // a row of nothing, or with NaN or +inf, has no softmax
        ln_z = logf(s.z);
        if (MODE == STEP) scale = a.weight[row] * a.inv_t / s.z;
    } else {
        m = a.stats[2 * row];
        ln_z = a.stats[2 * row + 1];
        scale = a.weight[row] * a.inv_t;
        reduce_entries();
        __syncthreads();
    }
    if (entries) t = add_warps(s_entries, min(kWarps, (a.k + 31) / 32));
    const float top = t.m, ln = logf(t.z);
    // the teacher's probabilities; this row's loss
    float loss = 0.f;
    for (int j = tid; j < a.k; j += kThreads) {
        const float t = (s_q[j] - top) * a.inv_t - ln;
        const float q = s_id[j] >= 0 ? expf(t) : 0.f;
        if (MODE != BACKWARD && (q > 0.f || q != q)) loss += q * (t - ((s_x[j] - m) * a.inv_t - ln_z));
        s_q[j] = q;
    }
    if (MODE != BACKWARD) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
        if (lane == 0) s_loss[warp] = loss;
    }
    __syncthreads();
    if (MODE != BACKWARD && part == 0 && tid == 0) {
        float all = s_loss[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) all += s_loss[w];
        a.loss[row] = all;
        a.stats[2 * row] = m;
        a.stats[2 * row + 1] = ln_z;
    }
    if (MODE != FORWARD) {
        const float l2 = MODE == BACKWARD ? ln_z * 1.4426950408889634f : 0.f;
        auto prob = [&](float v) { return ardiff::ex2((v - m) * c - l2); };
        const ardiff::Two minus = ardiff::two(-m, -m), c2 = ardiff::two(c, c), scale2 = ardiff::two(scale, scale);
        T* out = grad + x.lead;
        const bool wide = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
#pragma unroll 1
        for (int p = p0 + tid; p < p1; p += 4 * kThreads) {
            uint4 r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = p + j * kThreads;
                if (i >= p1) continue;
                if (MODE == STEP && i - p0 < a.cached) r[j] = s_cache[i - p0];       // (each thread's own)
                else r[j] = ardiff::load_piece(body + i);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = p + j * kThreads;
                if (i >= p1) continue;
                float v[N];
                ardiff::unpack(r[j], v, T());
#pragma unroll
                for (int l = 0; l < N; l += 2) {
                    const float2 y = ardiff::apart((ardiff::two(v[l], v[l + 1]) + minus) * c2);
                    const float2 e = ardiff::apart(ardiff::two(ardiff::ex2(y.x - l2), ardiff::ex2(y.y - l2)) * scale2);
                    v[l] = e.x;
                    v[l + 1] = e.y;
                }
                if (wide) {
                    __stcs(reinterpret_cast<uint4*>(out) + i, ardiff::pack(v, T()));
                } else {
#pragma unroll
                    for (int l = 0; l < N; ++l) out[i * N + l] = ardiff::from_float<T>(v[l]);
                }
            }
        }
        if (part == 0 && tid < x.lead) grad[tid] = ardiff::from_float<T>(prob(ardiff::to_float(x.x[tid])) * scale);
        if (part == a.parts - 1 && x.tail() + tid < a.V) {
            const int i = x.tail() + tid;
            grad[i] = ardiff::from_float<T>(prob(ardiff::to_float(x.x[i])) * scale);
        }
        __syncthreads();
        // the entries' places once more, with the teacher's share in the sum before it is rounded; an id that occurs again has
        // the sum of its shares, and every one of them writes the same
        const float share = a.weight[row] * a.inv_t;
        if (!s_again) {
            for (int j = tid; j < a.k; j += kThreads) {
                const int id = s_id[j];
                if (id >= v0 && id < v1) grad[id] = ardiff::from_float<T>(prob(s_x[j]) * scale - s_q[j] * share);
            }
        } else {
            for (int j = warp; j < a.k; j += kWarps) {
                const int id = s_id[j];
                if (id < v0 || id >= v1) continue;
                float q_sum = 0.f;
                for (int i = lane; i < a.k; i += 32) q_sum += s_id[i] == id ? s_q[i] : 0.f;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) q_sum += __shfl_xor_sync(0xffffffffu, q_sum, o);
                if (lane == 0) grad[id] = ardiff::from_float<T>(prob(s_x[j]) * scale - q_sum * share);
            }
        }
    }
    if (MODE != BACKWARD && a.parts > 1) cg::this_cluster().sync();      // a CTA leaves when its part has been read
}

template <typename T, int MODE>
int launch(const Args& a, int64_t n, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};         // devices on which the kernel may have its shared memory
    if (MODE == STEP) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess) return ARDIFF_ERR_CUDA;
        if (dev >= 64 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
            if (cudaFuncSetAttribute(distill_kernel<T, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     kCache + ARDIFF_DISTILL_MAX_K * 20) != cudaSuccess)
                return ARDIFF_ERR_CUDA;
            if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
        }
    }
    const size_t shared = (size_t)a.k * 12 + (size_t)a.seen * 4 + (size_t)a.cached * 16;
    const bool ok = ardiff::launch_early(distill_kernel<T, MODE>, (unsigned)(n * a.parts), kThreadsOf<MODE>, MODE == BACKWARD ? 1u : (unsigned)a.parts,
                                         shared, st, a);
    ardiff::set_launch_count(1);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}

template <int MODE>
int dispatch(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t ld, const void* teacher, int32_t teacher_type,
             const int32_t* ids, int32_t k, float temperature, const float* weight, float* loss, float* stats, void* grad,
             int64_t ld_grad, void* stream) {
    const int size = ardiff::value_size(dtype);
    if (!size || !ardiff::value_size(teacher_type)) return ARDIFF_ERR_UNSUPPORTED;
    if (n < 0 || n >= (int64_t)1 << 28 || V < 1 || V > ARDIFF_DISTILL_MAX_V || k < 1 || k > ARDIFF_DISTILL_MAX_K || ld < V)
        return ARDIFF_ERR_SHAPE;
    if (MODE != FORWARD && ld_grad < V) return ARDIFF_ERR_SHAPE;
    const float inv_t = 1.0f / temperature;                   // (and its octaves a unit, which the kernel forms, too)
    if (!(temperature > 0.f) || !isfinite(inv_t * 1.4426950408889634f) || !(inv_t > 0.f)) return ARDIFF_ERR_SHAPE;
    if (n == 0) {
        ardiff::set_launch_count(0);
        return ARDIFF_OK;
    }
    if (!logits || !teacher || !ids || !stats) return ARDIFF_ERR_NULL;
    if (MODE != BACKWARD && !loss) return ARDIFF_ERR_NULL;
    if (MODE != FORWARD && (!weight || !grad)) return ARDIFF_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(grad)) % size ||
        reinterpret_cast<uintptr_t>(teacher) % ardiff::value_size(teacher_type))
        return ARDIFF_ERR_ALIGN;
    Args a;
    memset(&a, 0, sizeof(a));
    a.x = logits; a.teacher = teacher; a.ids = ids; a.weight = weight; a.loss = loss; a.stats = stats; a.grad = grad;
    a.ld = ld; a.ld_grad = ld_grad; a.teacher_type = teacher_type; a.V = V; a.k = k; a.inv_t = inv_t;
    const int64_t pieces = (int64_t)V * size / 16;
    a.parts = 1;
    // A gradient's parts are strangers to each other: of 4096 pieces, so that they end one by one and not in a few waves (4096 x 131072
    // bf16: 364 us with a CTA a row, 348 with two, 330 with four, 369 with eight).
    if (MODE == BACKWARD) a.parts = (int)std::min<int64_t>(std::max<int64_t>(1, (pieces + 4095) / 4096), (((int64_t)1 << 31) - 1) / n);
    // More CTAs a row while there is room for them and each keeps several pieces a thread; otherwise meeting costs more than a part of a
    // row saves (us with 1 / 2 / 4 CTAs, bf16: loss 2048 x 32768 35 / 52 / 96, 296 x 32768 9.6 / 11.0 / 18.4, 64 x 32768 7.4 / 6.7 / 6.9,
    // 16 x 8191 4.7 / 5.3 / 5.4; step 2048 x 32768 77 / 111 / 206, 64 x 131072 34 / 23 / 22, with eight 26).
    while (a.parts < 8 && n * a.parts < 148 * 2 && pieces >= (int64_t)8 * kThreadsOf<MODE> * a.parts) a.parts *= 2;
    if (MODE != FORWARD)
        for (a.seen = 2; a.seen < 2 * k; a.seen *= 2) {}
    if (MODE == STEP) a.cached = (int)std::min<int64_t>((pieces + a.parts - 1) / a.parts, kCache / 16);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == ARDIFF_F32) return launch<float, MODE>(a, n, st);
    if (dtype == ARDIFF_F16) return launch<__half, MODE>(a, n, st);
    return launch<__nv_bfloat16, MODE>(a, n, st);
}

}  // namespace

extern "C" int ardiff_distill_topk(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t ld, const void* teacher,
                                   int32_t teacher_dtype, const int32_t* ids, int32_t k, float temperature, float* loss,
                                   float* stats, void* stream) {
    return dispatch<FORWARD>(logits, dtype, n, V, ld, teacher, teacher_dtype, ids, k, temperature, nullptr, loss, stats,
                             nullptr, 0, stream);
}

extern "C" int ardiff_distill_topk_backward(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t ld,
                                            const void* teacher, int32_t teacher_dtype, const int32_t* ids, int32_t k,
                                            float temperature, const float* stats, const float* weight, void* grad,
                                            int64_t ld_grad, void* stream) {
    return dispatch<BACKWARD>(logits, dtype, n, V, ld, teacher, teacher_dtype, ids, k, temperature, weight, nullptr,
                              const_cast<float*>(stats), grad, ld_grad, stream);
}

extern "C" int ardiff_distill_topk_step(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t ld,
                                        const void* teacher, int32_t teacher_dtype, const int32_t* ids, int32_t k,
                                        float temperature, const float* weight, float* loss, float* stats, void* grad,
                                        int64_t ld_grad, void* stream) {
    return dispatch<STEP>(logits, dtype, n, V, ld, teacher, teacher_dtype, ids, k, temperature, weight, loss, stats, grad,
                          ld_grad, stream);
}
