// ardiff_pages_evict: the tokens that have got least attention leave the cache.
//
// Of a request's `length` tokens `keep` stay: the ones in front of `first`, and of the others those of largest weight, lowest place first
// where equal, with recent ones counted as infinitely heavy. Attention does not ask in which order keys lie (their positions are in their
// rotations), so a token that stays keeps its place unless it lies at or behind the new end; those move, in order, into the places below it that
// became free. So as many rows move as leave a place free below the new end, not the whole cache, and sources (>= keep) and
// destinations (< keep) are apart: all moves run at once, in place.
//
// Two kernels. The first finds, by CTA a request (or a cluster of eight, where there are few requests of many tokens), the keep-th largest weight by three
// counts of 11, 11 and 10 bits over whole numbers that order as the weights do, then walks the places once more with a running count of heavier and
// equal ones: the number kept in front of a place p is heavier(p) + min(equal(p), equal ones needed), which gives every hole and every token
// behind the end its rank. CTAs of a cluster have a stretch of places each and read one another's counts. The second kernel copies the rows.
// Bound by the latency of those passes where few rows move (128 requests of 2056 tokens: 11 us and 4), by memory where many do.
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/ardiff.h"
#include "common.cuh"
#include "launch.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 2048;
constexpr int kPer = 4;                          // places of a thread, consecutive, in the last walk
constexpr int kKept = 40960;                     // keys that a CTA's shared memory holds; more are worked out again in every pass
constexpr int kCluster = 8;

struct Evict {
    const int32_t* length;
    const int32_t* budget;
    const int32_t* first;                        // or NULL: 0
    const float* score;
    const int32_t* position;                     // or NULL: the place
    const int32_t* seen;                         // or NULL: the length
    const int32_t* table;
    char* k;
    char* v;
    int32_t* new_length;
    float* new_score;
    int32_t* new_position;
    int32_t* source;
    int32_t* status;
    int2* move;                                  // [requests][capacity]: hole, token
    int32_t* moves;                              // [requests]
    long long ld, new_ld, limit;                 // limit: the longest request
    long long k_page, k_token, k_head, v_page, v_token, v_head;   // bytes
    int requests, recent, page, width, pages, heads, row, capacity;   // row: bytes of a head's row
};

// Whole numbers in the order of the weights: NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t ordered(float x) {
    if (!(x == x)) x = -INFINITY;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kInfinite = 0xff800000u;      // +inf

// Exclusive sums of two 32-bit counts over the CTA, and the totals. `s` holds 32 values.
__device__ __forceinline__ uint2 cta_scan(uint2 v, uint2* s, uint2* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint2 inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, inc.x, o), y = __shfl_up_sync(0xffffffffu, inc.y, o);
        if (lane >= o) { inc.x += x; inc.y += y; }
    }
    __syncthreads();
    if (lane == 31) s[warp] = inc;
    __syncthreads();
    uint2 w = s[lane];
    const uint2 own = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, w.x, o), y = __shfl_up_sync(0xffffffffu, w.y, o);
        if (lane >= o) { w.x += x; w.y += y; }
    }
    total->x = __shfl_sync(0xffffffffu, w.x, 31);
    total->y = __shfl_sync(0xffffffffu, w.y, 31);
    w.x -= own.x; w.y -= own.y;
    return make_uint2(inc.x - v.x + __shfl_sync(0xffffffffu, w.x, warp), inc.y - v.y + __shfl_sync(0xffffffffu, w.y, warp));
}

__device__ __forceinline__ uint32_t peer(const uint32_t* p, int cta) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(ptx::map_peer(ptx::smem_u32(p), cta)) : "memory");
    return v;
}

__device__ __forceinline__ void add_to_peer(const uint32_t* p, int cta, uint32_t v) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(ptx::map_peer(ptx::smem_u32(p), cta)), "r"(v) : "memory");
}

// kParts CTAs (a cluster) a request.
template <int kParts>
__global__ void __launch_bounds__(kThreads) select_kernel(const Evict a) {
    extern __shared__ uint32_t s_key[];
    __shared__ uint32_t s_bin[kBins], s_all[kParts > 1 ? 2 : 1][kParts > 1 ? kBins : 1], s_counts[4];      // heavier, equal: of the stretch, and of its part in front of the new end
    __shared__ uint2 s_scan[32];
    __shared__ uint32_t s_prefix, s_rest;
    ardiff::begin_kernel();
    const int tid = threadIdx.x, r = blockIdx.x / kParts, rank = blockIdx.x % kParts;
    auto meet = [&]() {
        if (kParts > 1) ptx::cluster_sync_all();
        else __syncthreads();
    };
    auto sum_of = [&](const uint32_t* p, int parts) {
        uint32_t v = 0;
        if constexpr (kParts == 1) {
            v = parts ? *p : 0u;
        } else {
            for (int i = 0; i < parts; ++i) v += peer(p, i);
        }
        return v;
    };
    if (kParts > 1)
        for (int b = tid; b < kBins; b += kThreads) s_all[0][b] = 0;
    if (blockIdx.x == 0) {
        bool bad = false;
        for (int i = tid; i < a.requests; i += kThreads) bad |= a.length[i] < 0 || (long long)a.length[i] > a.limit;
        bad = __syncthreads_or(bad);
        if (tid == 0) *a.status = bad ? ARDIFF_ERR_SHAPE : ARDIFF_OK;
    }
    const int length = a.length[r];
    meet();                                      // new_length may be the length itself
    if (length < 0 || (long long)length > a.limit) {         // left as it is
        if (tid == 0 && rank == 0) { a.new_length[r] = length; a.moves[r] = 0; }
        return;
    }
    const int first = a.first ? min(max(a.first[r], 0), length) : 0;
    const int keep = min(length, max(max(a.budget[r], 0), first));
    const float* score = a.score + r * a.ld;
    const int32_t* position = a.position ? a.position + r * a.ld : nullptr;
    const long long recent_from = (long long)(a.seen ? a.seen[r] : length) - a.recent;
    float* new_score = a.new_score + r * a.new_ld;
    int32_t* new_position = a.new_position ? a.new_position + r * a.new_ld : nullptr;
    int32_t* source = a.source ? a.source + r * a.new_ld : nullptr;
    meet();                                      // (seen, first or budget may be the same array, too)
    if (tid == 0 && rank == 0) a.new_length[r] = keep;
    auto stay = [&](int p) {
        new_score[p] = score[p];
        if (new_position) new_position[p] = position ? position[p] : p;
        if (source) source[p] = p;
    };
    if (keep == length) {
        if (tid == 0 && rank == 0) a.moves[r] = 0;
        for (int p = rank * kThreads + tid; p < length; p += kParts * kThreads) stay(p);
        return;
    }

    auto work_out = [&](int p) -> uint32_t {
        const long long pos = position ? position[p] : p;
        return pos >= recent_from ? kInfinite : ordered(score[p]);
    };
    const int n = length - first, stretch = ((n + kParts - 1) / kParts + kPer - 1) / kPer * kPer;
    const int lo = min(n, rank * stretch), hi = min(n, lo + stretch), end = keep - first;     // of this CTA; the new end
    auto key = [&](int i) -> uint32_t { return i - lo < kKept ? s_key[i - lo] : work_out(first + i); };
    for (int i = lo + tid; i < min(hi, lo + kKept); i += kThreads) s_key[i - lo] = work_out(first + i);

    // the need-th largest key, by its highest 11 bits, the next 11, the last 10
    uint32_t prefix = 0, need = end;
    constexpr int shift[3] = {21, 10, 0}, above[3] = {32, 21, 10};
    if (need > 0) {
#pragma unroll
        for (int round = 0; round < 3; ++round) {
            // (two lots of sums: the next round's is cleared while this one's is not yet complete)
            for (int b = tid; b < kBins; b += kThreads) {
                s_bin[b] = 0;
                if (kParts > 1) s_all[kParts > 1 ? (round + 1) & 1 : 0][b] = 0;
            }
            __syncthreads();
            const uint32_t mask = round == 2 ? 1023u : 2047u;
            for (int i = lo + tid; i < hi; i += kThreads) {
                const uint32_t k = key(i);
                if (round == 0 || (k >> above[round]) == (prefix >> above[round])) atomicAdd(&s_bin[(k >> shift[round]) & mask], 1u);
            }
            __syncthreads();
            const uint32_t* bin = s_bin;
            if (kParts > 1) {
                // every CTA adds its few bins that are not empty to everyone's sums
                uint32_t* sums = s_all[kParts > 1 ? round & 1 : 0];
                for (int b = tid; b < kBins; b += kThreads)
                    if (s_bin[b])
                        for (int i = 0; i < kParts; ++i) add_to_peer(sums + b, i, s_bin[b]);
                meet();
                bin = sums;
            }
            // bins from the top: thread t has the two from kBins - 1 - 2 t down
            const int top = kBins - 1 - 2 * tid;
            const uint32_t upper = bin[top], lower = bin[top - 1];
            uint2 total;
            const uint32_t before = cta_scan(make_uint2(upper + lower, 0u), s_scan, &total).x;
            if (before < need && need <= before + upper + lower) {
                const bool second = need > before + upper;
                s_prefix = prefix | ((uint32_t)(second ? top - 1 : top) << shift[round]);
                s_rest = need - before - (second ? upper : 0u);
            }
            __syncthreads();
            prefix = s_prefix;
            need = s_rest;                       // of those that begin like this
            __syncthreads();
        }
    } else {
        prefix = 0xffffffffu;                    // nothing is heavier or as heavy
        __syncthreads();
    }
    const uint32_t border = prefix, equal = need;

    // heavier and equal ones in front of this CTA's places, and of all in front of the new end
    uint2 carry = make_uint2(0u, 0u);
    uint32_t inside;
    {
        uint2 all = make_uint2(0u, 0u), front = make_uint2(0u, 0u);
        for (int i = lo + tid; i < hi; i += kThreads) {
            const uint32_t k = key(i);
            all.x += k > border; all.y += k == border;
            if (i < end) { front.x += k > border; front.y += k == border; }
        }
        uint2 sum_all, sum_front;
        cta_scan(all, s_scan, &sum_all);
        cta_scan(front, s_scan, &sum_front);
        if (tid == 0) { s_counts[0] = sum_all.x; s_counts[1] = sum_all.y; s_counts[2] = sum_front.x; s_counts[3] = sum_front.y; }
        meet();
        if (kParts > 1) carry = make_uint2(sum_of(&s_counts[0], rank), sum_of(&s_counts[1], rank));
        inside = sum_of(&s_counts[2], kParts) + min(sum_of(&s_counts[3], kParts), equal);
    }

    // places in order: what is kept, its rank; holes in front of the new end, tokens behind it
    int2* move = a.move + (long long)r * a.capacity;
    for (int base = lo; base < hi; base += kThreads * kPer) {
        uint32_t k[kPer];
        uint2 mine = make_uint2(0u, 0u);
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int i = base + tid * kPer + u;
            k[u] = i < hi ? key(i) : 0u;
            if (i < hi) { mine.x += k[u] > border; mine.y += k[u] == border; }
        }
        uint2 total;
        uint2 at = cta_scan(mine, s_scan, &total);
        at.x += carry.x; at.y += carry.y;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int i = base + tid * kPer + u, p = first + i;
            if (i < hi) {
                const uint32_t before = at.x + min(at.y, equal);
                const bool stays = k[u] > border || (k[u] == border && at.y < equal);
                if (p < keep) {
                    if (stays) stay(p);
                    else move[i - before].x = p;
                } else if (stays) {
                    move[before - inside].y = p;
                }
            }
            at.x += k[u] > border; at.y += k[u] == border;
        }
        carry.x += total.x; carry.y += total.y;
    }
    for (int p = rank * kThreads + tid; p < first; p += kParts * kThreads) stay(p);
    const int moves = end - (int)inside;
    if (tid == 0 && rank == 0) a.moves[r] = moves;
    meet();
    for (int j = rank * kThreads + tid; j < moves; j += kParts * kThreads) {
        const int2 m = move[j];
        new_score[m.x] = score[m.y];
        if (new_position) new_position[m.x] = position ? position[m.y] : m.y;
        if (source) source[m.x] = m.y;
    }
}

// A warp a move: the rows of all heads, keys and values, four pieces a lane under way. The lanes look up 32 moves at once, so that between one
// move and the next nothing is waited for but the rows (8 requests, 14 thousand moves of 4 KB: 117 MB in 20 us, 5.9 TB/s).
__global__ void __launch_bounds__(256) move_kernel(const Evict a, int split) {
    ardiff::begin_kernel();
    const int r = blockIdx.x / split, lane = threadIdx.x & 31, warps = split * 8;
    const int2* move = a.move + (long long)r * a.capacity;
    const int32_t* table = a.table + (long long)r * a.width;
    const int moves = a.moves[r];
    const int pieces = a.row / 16, all = a.heads * pieces;
    for (int j0 = (blockIdx.x - r * split) * 8 + (threadIdx.x >> 5); j0 < moves; j0 += warps * 32) {
        const int j = j0 + lane * warps;         // (moves are at most 2^30, and 32 warps' worth 151552)
        long long k_from = -1, v_from = 0, k_to = 0, v_to = 0;
        if (j < moves) {
            const int2 m = move[j];
            const int to_page = m.x / a.page, from_page = m.y / a.page;
            const int to = table[to_page], from = table[from_page];
            if (to < 0 || to >= a.pages || from < 0 || from >= a.pages) {
                *a.status = ARDIFF_ERR_SHAPE;
            } else {
                const long long to_in = m.x - to_page * a.page, from_in = m.y - from_page * a.page;
                k_from = from * a.k_page + from_in * a.k_token;
                v_from = from * a.v_page + from_in * a.v_token;
                k_to = to * a.k_page + to_in * a.k_token;
                v_to = to * a.v_page + to_in * a.v_token;
            }
        }
        const int here = min(32, (moves - j0 + warps - 1) / warps);
        for (int t = 0; t < here; ++t) {
            const long long kf = __shfl_sync(0xffffffffu, k_from, t), vf = __shfl_sync(0xffffffffu, v_from, t);
            const long long kt = __shfl_sync(0xffffffffu, k_to, t), vt = __shfl_sync(0xffffffffu, v_to, t);
            if (kf < 0) continue;
            for (int c0 = lane; c0 < all; c0 += 128) {
                uint4 x[4], y[4];
                long long k_off[4], v_off[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int c = c0 + 32 * u;
                    if (c >= all) continue;
                    const int h = c / pieces, in = (c - h * pieces) * 16;
                    k_off[u] = h * a.k_head + in;
                    v_off[u] = h * a.v_head + in;
                    x[u] = *reinterpret_cast<const uint4*>(a.k + kf + k_off[u]);
                    y[u] = *reinterpret_cast<const uint4*>(a.v + vf + v_off[u]);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (c0 + 32 * u >= all) continue;
                    *reinterpret_cast<uint4*>(a.k + kt + k_off[u]) = x[u];
                    *reinterpret_cast<uint4*>(a.v + vt + v_off[u]) = y[u];
                }
            }
        }
    }
}

// moves of a request: as many as there are holes below the new end and tokens behind it
int64_t move_capacity(int64_t limit) { return limit / 2 + 1; }

}  // namespace

extern "C" int64_t ardiff_pages_evict_workspace(int32_t requests, int32_t page, int32_t width) {
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS || page < 1 || width < 0 || (int64_t)page * width > ARDIFF_CACHE_MAX_PLACES)
        return ARDIFF_ERR_SHAPE;
    return (int64_t)requests * (8 * move_capacity((int64_t)page * width) + 4) + 16;
}

extern "C" int ardiff_pages_evict(const ardiff_pages_evict_call* call, void* stream) {
    if (!call) return ARDIFF_ERR_NULL;
    const ardiff_pages_evict_call& c = *call;
    if (!ardiff::in_32_bits({c.requests, c.recent, c.width, c.dtype, c.pages, c.page, c.heads, c.head_width})) return ARDIFF_ERR_SHAPE;
    const int requests = (int)c.requests, page = (int)c.page, width = (int)c.width, size = ardiff::value_size((int32_t)c.dtype);
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS || page < 1 || width < 0 || c.pages < 0 || c.heads < 1 || c.heads > 65535 ||
        c.head_width < 1 || c.head_width > ARDIFF_ROTARY_MAX_WIDTH || c.recent < 0 || c.ld < 0 || c.new_ld < 0 || (int64_t)page * width > ARDIFF_CACHE_MAX_PLACES)
        return ARDIFF_ERR_SHAPE;
    if (!size || c.head_width * size % 16) return ARDIFF_ERR_UNSUPPORTED;
    if (!c.status) return ARDIFF_ERR_NULL;
    if (requests > 0 && (!c.length || !c.budget || !c.score || !c.new_length || !c.new_score || !c.workspace || (width > 0 && !c.table) || !c.k_cache || !c.v_cache))
        return ARDIFF_ERR_NULL;
    if (((reinterpret_cast<uintptr_t>(c.k_cache) | reinterpret_cast<uintptr_t>(c.v_cache)) & 15u) ||
        ((c.k_page | c.k_token | c.k_head | c.v_page | c.v_token | c.v_head) * size & 15) || (reinterpret_cast<uintptr_t>(c.workspace) & 15u))
        return ARDIFF_ERR_ALIGN;
    const int64_t limit = (int64_t)page * width;
    if (c.workspace_bytes < ardiff_pages_evict_workspace(requests, page, width) && requests > 0) return ARDIFF_ERR_SHAPE;
    if (requests > 1 && c.ld != c.new_ld && (c.score == c.new_score || (c.position && c.position == c.new_position))) return ARDIFF_ERR_SHAPE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Evict a;
    memset(&a, 0, sizeof(a));
    a.length = c.length; a.budget = c.budget; a.first = c.first; a.score = c.score; a.position = c.position; a.seen = c.seen; a.table = c.table;
    a.k = static_cast<char*>(c.k_cache); a.v = static_cast<char*>(c.v_cache);
    a.new_length = c.new_length; a.new_score = c.new_score; a.new_position = c.new_position; a.source = c.source; a.status = c.status;
    a.capacity = (int)move_capacity(limit);
    a.move = static_cast<int2*>(c.workspace);
    a.moves = reinterpret_cast<int32_t*>(a.move + (int64_t)requests * a.capacity);
    a.ld = c.ld; a.new_ld = c.new_ld;
    a.limit = limit < c.ld ? limit : c.ld;
    a.limit = a.limit < c.new_ld ? a.limit : c.new_ld;
    a.k_page = c.k_page * size; a.k_token = c.k_token * size; a.k_head = c.k_head * size;
    a.v_page = c.v_page * size; a.v_token = c.v_token * size; a.v_head = c.v_head * size;
    a.requests = requests; a.recent = c.recent; a.page = page; a.width = width; a.pages = c.pages; a.heads = c.heads; a.row = c.head_width * size;
    if (requests == 0) {
        const bool ok = cudaMemsetAsync(c.status, 0, 4, st) == cudaSuccess;
        ardiff::set_launch_count(0);
        return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
    }
    const int sms = ardiff::device_sms();
    if (sms < 1) return ARDIFF_ERR_CUDA;
    // A cluster a request where that fills no more than two rounds of the SMs and a CTA has 512 places or more of the longest one (8 requests of 16384:
    // 38 us with a CTA each, 18 with eight).
    const bool clusters = requests * kCluster <= 2 * sms && limit >= kCluster * 512;
    const int64_t places = clusters ? (limit + kCluster - 1) / kCluster + kPer : limit, keys = places < kKept ? places : kKept;
    const int split = requests >= 592 ? 1 : (592 + requests - 1) / requests;
    static std::atomic<uint64_t> ready[2] = {};
    const bool ok = (clusters ? ardiff::shared_memory(select_kernel<kCluster>, kKept * 4, ready[1]) &&
                                    ardiff::launch_early(select_kernel<kCluster>, (unsigned)requests * kCluster, kThreads, kCluster, (size_t)keys * 4, st, a)
                              : ardiff::shared_memory(select_kernel<1>, kKept * 4, ready[0]) &&
                                    ardiff::launch_early(select_kernel<1>, (unsigned)requests, kThreads, 1, (size_t)keys * 4, st, a)) &&
                    ardiff::launch_early(move_kernel, (unsigned)(requests * split), 256, 1, 0, st, a, split);
    ardiff::set_launch_count(2);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}
