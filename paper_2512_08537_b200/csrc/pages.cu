// Paged-cache bookkeeping on the device, around a round of speculation:
//   ardiff_pages_extend    places new tokens: takes pages from the free list, lengthens the block tables, writes the slot,
//                          position and request of every new token;
//   ardiff_pages_truncate  takes rejected tokens back: pages that no token needs go back to the free list.
//
// Everything follows from two prefix sums over the requests, tokens and pages: with held_r = ceil(length_r / page) and
// new_r = ceil((length_r + add_r) / page) - held_r, request r's j-th new page is the free list's entry
// count - 1 - (sum_{r' < r} new_r' + j), and its token at position p lies in page number p / page of its table. Every number is
// whole, so no order of threads changes a result.
//
// Bound by latency: one CTA sums, checks and, where the buffers hold few tokens, writes everything in one launch. Where they
// hold many, a second kernel over all SMs writes tokens and tables; it finds all it needs in the first one's outputs
// (offset and new_length), so no scratch is needed and inputs may be updated in place.
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/ardiff.h"
#include "common.cuh"
#include "launch.cuh"

namespace {

constexpr int kThreads = 1024;
constexpr int kPer = 4;                          // requests a thread, consecutive
constexpr int kTile = kThreads * kPer;           // requests whose sums lie in shared memory together

struct Sums { long long tokens, pages; };

__device__ __forceinline__ Sums operator+(Sums a, Sums b) { return Sums{a.tokens + b.tokens, a.pages + b.pages}; }

__device__ __forceinline__ Sums shfl_up(Sums v, int o) {
    return Sums{__shfl_up_sync(0xffffffffu, v.tokens, o), __shfl_up_sync(0xffffffffu, v.pages, o)};
}

// Exclusive sums over the CTA's threads, and their total. All threads call it; `s` holds a value a warp.
__device__ __forceinline__ Sums cta_scan(Sums v, Sums* s, Sums* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sums inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums up = shfl_up(inc, o);
        if (lane >= o) inc = inc + up;
    }
    __syncthreads();                             // the last call's values have been read
    if (lane == 31) s[warp] = inc;
    __syncthreads();
    Sums w = s[lane];                            // 32 warps
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums up = shfl_up(w, o);
        if (lane >= o) w = w + up;
    }
    *total = Sums{__shfl_sync(0xffffffffu, w.tokens, 31), __shfl_sync(0xffffffffu, w.pages, 31)};
    const Sums before = Sums{__shfl_sync(0xffffffffu, w.tokens, (warp + 31) & 31),
                             __shfl_sync(0xffffffffu, w.pages, (warp + 31) & 31)};
    Sums ex{inc.tokens - v.tokens, inc.pages - v.pages};
    return warp ? ex + before : ex;
}

// tokens in 0 .. 2^31 - 1, so that the sum fits 32 bits without a sign
__device__ __forceinline__ int pages_of(int tokens, int page) {
    return (int)(((unsigned)tokens + (unsigned)(page - 1)) / (unsigned)page);
}

struct Extend {
    const int32_t* length;
    const int32_t* add;
    int32_t* table;
    const int32_t* free_pages;
    const int32_t* free_count;
    int64_t* slot;
    int32_t* position;
    int32_t* request;
    int32_t* offset;
    int32_t* new_length;
    int32_t* new_free_count;
    int32_t* status;
    long long free_capacity, max_tokens;
    int requests, page, width;
    bool wide;                                   // slot, position and request start on 16-byte boundaries
};

// What the token writer keeps of a tile of requests: the first token and the first new page of each, its pages held before.
struct Tile {
    int off[kTile + 1];
    int first[kTile];
    int start[kTile];                            // position of the request's first new token
};

// Writes the tokens [lo, hi) of a tile of `m` requests from `r0` on: a thread takes four consecutive ones, looks up the
// request of the first and walks on. `free_top`: the free list's entries before the call.
__device__ void write_tokens(const Extend& a, const Tile& t, int r0, int m, int lo, int hi, int free_top) {
    const int q_end = (int)(((unsigned)hi + 3u) / 4u);       // (hi may be the last number of 32 bits)
    for (int q = lo / 4 + (int)threadIdx.x; q < q_end; q += kThreads) {
        const int t0 = max(lo, 4 * q), t1 = (int)min((unsigned)hi, 4u * (unsigned)q + 4u);
        int below = 0, above = m;                // the last request whose first token is not behind t0
        while (above - below > 1) {
            const int mid = (below + above) >> 1;
            if (t.off[mid] <= t0) below = mid; else above = mid;
        }
        int r = below;
        int64_t slot[4];
        int pos4[4], req4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int tok = 4 * q + i;
            if (tok < t0 || tok >= t1) continue;
            while (tok >= t.off[r + 1]) ++r;     // requests without new tokens are passed over; tok < off[m]
            const int pos = t.start[r] + (tok - t.off[r]);
            const int pg = (int)((unsigned)pos / (unsigned)a.page), in_page = pos - pg * a.page;
            const int held = pages_of(t.start[r], a.page);
            int32_t* entry = a.table + (int64_t)(r0 + r) * a.width + pg;
            int id;
            if (pg < held) {
                id = *entry;
            } else {
                id = a.free_pages[free_top - 1 - (t.first[r] + pg - held)];
                if (in_page == 0) *entry = id;   // the first token of every new page is a new token
            }
            slot[i] = (int64_t)id * a.page + in_page;
            pos4[i] = pos;
            req4[i] = r0 + r;
        }
        if (a.wide && t1 - t0 == 4) {
            reinterpret_cast<longlong2*>(a.slot)[2 * q] = make_longlong2(slot[0], slot[1]);
            reinterpret_cast<longlong2*>(a.slot)[2 * q + 1] = make_longlong2(slot[2], slot[3]);
            if (a.position) reinterpret_cast<int4*>(a.position)[q] = make_int4(pos4[0], pos4[1], pos4[2], pos4[3]);
            if (a.request) reinterpret_cast<int4*>(a.request)[q] = make_int4(req4[0], req4[1], req4[2], req4[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tok = 4 * q + i;
                if (tok < t0 || tok >= t1) continue;
                a.slot[tok] = slot[i];
                if (a.position) a.position[tok] = pos4[i];
                if (a.request) a.request[tok] = req4[i];
            }
        }
    }
}

// One CTA: sums and checks, then offset, new_length, new_free_count and status; with WRITE tokens and tables too.
template <bool WRITE>
__global__ void __launch_bounds__(kThreads) extend_kernel(const Extend a) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Sums s_scan[32];
    ardiff::begin_kernel();
    Tile& t = *reinterpret_cast<Tile*>(smem);
    const int tid = threadIdx.x;
    const bool one = a.requests <= kTile;
    int len[kPer], add[kPer];
    bool bad = false;
    Sums mine{0, 0};
    const int free_top = *a.free_count;
    for (int r0 = 0; r0 < a.requests; r0 += kTile) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + tid * kPer + i;
            len[i] = r < a.requests ? a.length[r] : 0;
            add[i] = r < a.requests ? a.add[r] : 0;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const long long after = (long long)len[i] + add[i];
            if (len[i] < 0 || add[i] < 0 || after > (long long)a.width * a.page || after > 0x7fffffffll) bad = true;
            else mine = mine + Sums{add[i], pages_of((int)after, a.page) - pages_of(len[i], a.page)};
        }
    }
    Sums total;
    const Sums before = cta_scan(mine, s_scan, &total);
    bad = __syncthreads_or(bad || free_top < 0 || free_top > a.free_capacity || total.tokens > a.max_tokens);
    const bool short_ = total.pages > free_top;
    const bool ok = !bad && !short_;
    if (tid == 0) {
        *a.status = bad ? ARDIFF_ERR_SHAPE : short_ ? ARDIFF_ERR_NOMEM : ARDIFF_OK;
        *a.new_free_count = ok ? free_top - (int)total.pages : free_top;
        a.offset[a.requests] = ok ? (int)total.tokens : 0;
    }
    Sums carry{0, 0};
    for (int r0 = 0; r0 < a.requests; r0 += kTile) {
        Sums at = before;
        if (!one) {                              // several tiles: the first pass has read them all, its registers hold the last
            Sums v{0, 0}, tile;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = r0 + tid * kPer + i;
                len[i] = r < a.requests ? a.length[r] : 0;
                add[i] = r < a.requests ? a.add[r] : 0;
                if (ok) v = v + Sums{add[i], pages_of(len[i] + add[i], a.page) - pages_of(len[i], a.page)};
            }
            at = carry + cta_scan(v, s_scan, &tile);
            carry = carry + tile;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + tid * kPer + i;
            if (r < a.requests) {
                a.offset[r] = ok ? (int)at.tokens : 0;
                a.new_length[r] = ok ? len[i] + add[i] : len[i];
            }
            if (WRITE && ok) {
                t.off[tid * kPer + i] = (int)at.tokens;
                t.first[tid * kPer + i] = (int)at.pages;
                t.start[tid * kPer + i] = len[i];
                at = at + Sums{add[i], pages_of(len[i] + add[i], a.page) - pages_of(len[i], a.page)};
            } else if (ok) {
                at.tokens += add[i];
            }
        }
        if (WRITE && ok) {
            if (tid == kThreads - 1) t.off[kTile] = (int)at.tokens;
            __syncthreads();
            write_tokens(a, t, r0, kTile, t.off[0], t.off[kTile], free_top);
            __syncthreads();
        }
    }
}

// Tokens and tables of a call whose sums extend_kernel<false> has written, over all SMs: every CTA forms the sums of each tile
// again (they are few) and writes its share of the tokens.
__global__ void __launch_bounds__(kThreads) extend_write_kernel(const Extend a) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Sums s_scan[32];
    Tile& t = *reinterpret_cast<Tile*>(smem);
    const int tid = threadIdx.x;
    ardiff::begin_kernel();
    const int total = a.offset[a.requests];
    const int quads = (int)(((unsigned)total + 3u) / 4u);
    const int per = (quads + gridDim.x - 1) / gridDim.x;
    const int lo = (int)min((long long)total, 4ll * per * blockIdx.x), hi = (int)min((long long)total, 4ll * per * (blockIdx.x + 1));
    if (lo >= hi) return;
    // pages taken by the whole call: where the free list ended before it
    long long pages = 0;
    for (int r0 = 0; r0 < a.requests; r0 += kTile) {
        Sums v{0, 0}, tile;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + i * kThreads + tid;
            if (r < a.requests) {
                const int after = a.new_length[r], more = a.offset[r + 1] - a.offset[r];
                v.pages += pages_of(after, a.page) - pages_of(after - more, a.page);
            }
        }
        cta_scan(v, s_scan, &tile);
        pages += tile.pages;
    }
    const int free_top = *a.new_free_count + (int)pages;
    Sums carry{0, 0};
    for (int r0 = 0; r0 < a.requests; r0 += kTile) {
        Sums v{0, 0}, tile;
        int after[kPer], off[kPer + 1];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + tid * kPer + i;
            off[i] = a.offset[min(r, a.requests)];
            after[i] = r < a.requests ? a.new_length[r] : 0;
        }
        off[kPer] = a.offset[min(r0 + tid * kPer + kPer, a.requests)];
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            v.pages += pages_of(after[i], a.page) - pages_of(after[i] - (off[i + 1] - off[i]), a.page);
        Sums at = carry + cta_scan(v, s_scan, &tile);
        carry = carry + tile;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int more = off[i + 1] - off[i];
            t.off[tid * kPer + i] = off[i];
            t.first[tid * kPer + i] = (int)at.pages;
            t.start[tid * kPer + i] = after[i] - more;
            at.pages += pages_of(after[i], a.page) - pages_of(after[i] - more, a.page);
        }
        if (tid == kThreads - 1) t.off[kTile] = off[kPer];
        __syncthreads();
        write_tokens(a, t, r0, kTile, max(lo, t.off[0]), min(hi, t.off[kTile]), free_top);
        __syncthreads();
    }
}

struct Truncate {
    const int32_t* length;
    const int32_t* target;
    const int32_t* table;
    int32_t* free_pages;
    const int32_t* free_count;
    int32_t* new_free_count;
    int32_t* status;
    long long free_capacity;
    int requests, page, width;
};

// One CTA. Request r gives back the pages stay_r .. held_r - 1 of its table; they go on the free list in the order that makes a
// later extend hand them out as an earlier one did (the last request's last page lowest).
__global__ void __launch_bounds__(kThreads) truncate_kernel(const Truncate a) {
    __shared__ Sums s_scan[32];
    __shared__ int s_first[kTile + 1], s_stay[kTile];
    ardiff::begin_kernel();
    const int tid = threadIdx.x;
    const bool one = a.requests <= kTile;
    int stay[kPer], back[kPer];
    bool bad = false;
    Sums mine{0, 0};
    const int free_top = *a.free_count;
    for (int r0 = 0; r0 < a.requests; r0 += kTile) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + tid * kPer + i;
            const int len = r < a.requests ? a.length[r] : 0, to = r < a.requests ? a.target[r] : 0;
            if (to < 0 || to > len || (long long)len > (long long)a.width * a.page) {
                bad = true;
                stay[i] = back[i] = 0;
            } else {
                stay[i] = pages_of(to, a.page);
                back[i] = pages_of(len, a.page) - stay[i];
            }
            mine.pages += back[i];
        }
    }
    Sums total;
    const Sums before = cta_scan(mine, s_scan, &total);
    bad = __syncthreads_or(bad || free_top < 0 || free_top + total.pages > a.free_capacity);
    if (tid == 0) {
        *a.status = bad ? ARDIFF_ERR_SHAPE : ARDIFF_OK;
        *a.new_free_count = bad ? free_top : free_top + (int)total.pages;
    }
    if (bad) return;
    const int last = free_top + (int)total.pages - 1;
    Sums carry{0, 0};
    for (int r0 = 0; r0 < a.requests; r0 += kTile) {
        Sums at = before;
        if (!one) {
            Sums v{0, 0}, tile;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = r0 + tid * kPer + i;
                stay[i] = r < a.requests ? pages_of(a.target[r], a.page) : 0;
                back[i] = r < a.requests ? pages_of(a.length[r], a.page) - stay[i] : 0;
                v.pages += back[i];
            }
            at = carry + cta_scan(v, s_scan, &tile);
            carry = carry + tile;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            s_first[tid * kPer + i] = (int)at.pages;
            s_stay[tid * kPer + i] = stay[i];
            at.pages += back[i];
        }
        if (tid == kThreads - 1) s_first[kTile] = (int)at.pages;
        __syncthreads();
        // (without a sign: the last step may pass 2^31)
        for (unsigned next = (unsigned)s_first[0] + tid; next < (unsigned)s_first[kTile]; next += kThreads) {
            const int g = (int)next;
            int below = 0, above = kTile;        // the last request whose first page given back is not behind g
            while (above - below > 1) {
                const int mid = (below + above) >> 1;
                if (s_first[mid] <= g) below = mid; else above = mid;
            }
            a.free_pages[last - g] = a.table[(int64_t)(r0 + below) * a.width + s_stay[below] + (g - s_first[below])];
        }
        __syncthreads();
    }
}

// Buffers of at most this many tokens: one CTA writes them in the launch that sums. (The host knows the buffer's size, not how much of it
// the call fills. us with one / two launches: 256 requests with 256 tokens 7.4 / 10.4, with 8000 12.9 / 10.6; 2048 requests with 8000
// 14.9 / 12.5; 64 with 16000 16.8 / 9.9. So a full buffer of this size loses some 5 us, a nearly empty one gains 3.)
constexpr int64_t kOneLaunchTokens = 16384;

// The current device's SM count, its kernels' shared memory granted; 0 where that fails. Asked once a device.
int prepare_device() {
    static std::atomic<int> known[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < 64 && known[dev].load(std::memory_order_relaxed)) return known[dev].load(std::memory_order_relaxed);
    int sms = 0;
    const int bytes = (int)sizeof(Tile);
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1 || cudaFuncSetAttribute(extend_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess ||
        cudaFuncSetAttribute(extend_write_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess)
        return 0;
    if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

}  // namespace

extern "C" int ardiff_pages_extend(int32_t requests, int32_t page, int32_t width, const int32_t* length, const int32_t* add,
                                   int32_t* table, const int32_t* free_pages, int64_t free_capacity,
                                   const int32_t* free_count, int64_t max_tokens, int64_t* slot, int32_t* position,
                                   int32_t* request, int32_t* offset, int32_t* new_length, int32_t* new_free_count,
                                   int32_t* status, void* stream) {
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS || page < 1 || width < 0 || free_capacity < 0 ||
        free_capacity >= (int64_t)1 << 31 || max_tokens < 0 || max_tokens >= (int64_t)1 << 31)
        return ARDIFF_ERR_SHAPE;
    if (!free_count || !offset || !new_free_count || !status) return ARDIFF_ERR_NULL;
    if (requests > 0 && (!length || !add || !new_length || (width > 0 && !table))) return ARDIFF_ERR_NULL;
    if ((free_capacity > 0 && !free_pages) || (max_tokens > 0 && !slot)) return ARDIFF_ERR_NULL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Extend a;
    memset(&a, 0, sizeof(a));
    a.length = length; a.add = add; a.table = table; a.free_pages = free_pages; a.free_count = free_count;
    a.slot = slot; a.position = position; a.request = request; a.offset = offset; a.new_length = new_length;
    a.new_free_count = new_free_count; a.status = status;
    a.free_capacity = free_capacity; a.max_tokens = max_tokens;
    a.requests = requests; a.page = page; a.width = width;
    a.wide = ((reinterpret_cast<uintptr_t>(slot) | reinterpret_cast<uintptr_t>(position) |
               reinterpret_cast<uintptr_t>(request)) & 15u) == 0;
    const int sms = prepare_device();
    if (sms < 1) return ARDIFF_ERR_CUDA;
    if (max_tokens <= kOneLaunchTokens) {
        const bool ok = ardiff::launch_early(extend_kernel<true>, 1, kThreads, 1, sizeof(Tile), st, a);
        ardiff::set_launch_count(1);
        return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
    }
    const bool ok = ardiff::launch_early(extend_kernel<false>, 1, kThreads, 1, 0, st, a) &&
                    ardiff::launch_early(extend_write_kernel, (unsigned)sms, kThreads, 1, sizeof(Tile), st, a);
    ardiff::set_launch_count(2);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}

extern "C" int ardiff_pages_truncate(int32_t requests, int32_t page, int32_t width, const int32_t* length,
                                     const int32_t* target, const int32_t* table, int32_t* free_pages,
                                     int64_t free_capacity, const int32_t* free_count, int32_t* new_free_count,
                                     int32_t* status, void* stream) {
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS || page < 1 || width < 0 || free_capacity < 0 ||
        free_capacity >= (int64_t)1 << 31)
        return ARDIFF_ERR_SHAPE;
    if (!free_count || !new_free_count || !status) return ARDIFF_ERR_NULL;
    if (requests > 0 && (!length || !target || (width > 0 && !table))) return ARDIFF_ERR_NULL;
    if (free_capacity > 0 && !free_pages) return ARDIFF_ERR_NULL;
    Truncate a;
    memset(&a, 0, sizeof(a));
    a.length = length; a.target = target; a.table = table; a.free_pages = free_pages; a.free_count = free_count;
    a.new_free_count = new_free_count; a.status = status; a.free_capacity = free_capacity;
    a.requests = requests; a.page = page; a.width = width;
    const bool ok = ardiff::launch_early(truncate_kernel, 1, kThreads, 1, 0, static_cast<cudaStream_t>(stream), a);
    ardiff::set_launch_count(1);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}
