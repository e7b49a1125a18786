// ardiff_attend_weights: the attention weight that every token of a cache gets from the call's queries, added to what it had:
//
//   new_score[r][p] = decay score[r][p] + sum over the request's new tokens i and query heads h of exp(scale q_ih.k_p - lse_ih)
//
// lse comes from the attention itself, so no maximum and no second pass is needed, and every key's sum stands alone: a CTA takes 64
// keys of a request, goes through all kv heads (whose keys lie side by side in the cache), and writes each sum once. No atomics: equal calls
// give equal bits. Keys are the left operand (a warp 16 of them) and query rows the columns, so that a sum over rows stays in a
// thread's registers and four lanes.
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

constexpr int kPlanThreads = 1024;
constexpr int kTileKeys = 64;
constexpr int kThreads = 128;
constexpr int kStages = 4;

struct Weights {
    Pages cache;
    Queries x;
    const int32_t* length;
    const int32_t* offset;
    const int32_t* first;
    const float* score;
    float* new_score;
    int32_t* status;
    long long* tiles;                            // [requests + 1]: tiles of the requests before
    long long ld, new_ld, limit;
    float scale, decay;                          // scale: times log2 e
    int requests, causal;
};

__global__ void __launch_bounds__(kPlanThreads) tiles_kernel(const Weights c) {
    __shared__ long long s_scan[32];
    ardiff::begin_kernel();
    const int tid = threadIdx.x, R = c.requests;
    bool bad = false;
    long long tiles = 0;
    for (int r0 = 0; r0 < R; r0 += kPlanThreads) {
        const int r = r0 + tid;
        int n = 0;
        if (r < R) {
            const int a = c.offset[r], b = c.offset[r + 1], len = c.length[r];
            bad |= a < 0 || b < a || b > c.x.tokens || len < 0 || len > c.limit;
            const int first = c.first ? max(0, c.first[r]) : 0;
            n = len > first ? (len - first + kTileKeys - 1) / kTileKeys : 0;
        }
        long long total;
        const long long at = tiles + cta_scan(n, s_scan, &total);
        if (r < R) c.tiles[r] = at;
        tiles += total;
    }
    bad = __syncthreads_or(bad);
    if (tid == 0) {
        *c.status = bad ? ARDIFF_ERR_SHAPE : ARDIFF_OK;
        c.tiles[R] = bad ? 0 : tiles;
    }
}

template <int D> constexpr int kTileBytes = kTileKeys * kPitch<D>;
template <int D> constexpr int kShared = kStages * (kTileBytes<D> + kTileKeys * 8);

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) weights_kernel(const Weights c) {
    extern __shared__ __align__(128) char smem[];
    long long* place = reinterpret_cast<long long*>(smem + kStages * kTileBytes<D>);     // [stages][keys]
    ardiff::begin_kernel();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane & 3, row8 = lane >> 2;
    const int R = c.requests, H = c.cache.heads, G = c.x.G;
    const long long tiles = c.tiles[R];
    const uint32_t at = ptx::smem_u32(smem);
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int r = find_last(c.tiles, R, tile);
        const int token0 = c.offset[r], n = c.offset[r + 1] - token0, len = c.length[r];
        const int key0 = (c.first ? max(0, c.first[r]) : 0) + (int)(tile - c.tiles[r]) * kTileKeys;
        const int keys = min(kTileKeys, len - key0);
        const int rows = n * G, limit = c.causal ? len - n + 1 : len;
        __syncthreads();                         // the last tile's places have been read
        if (tid < kTileKeys) {
            long long p = -1;
            if (tid < keys) {
                const unsigned key = key0 + tid, pg = key / (unsigned)c.cache.page, in = key - pg * c.cache.page;
                const int id = c.cache.table[(long long)r * c.cache.width + pg];
                if (id >= 0 && id < c.cache.pages) p = id * c.cache.k_page + in * c.cache.k_token;
                else *c.status = ARDIFF_ERR_SHAPE;
            }
            place[tid] = p;
        }
        __syncthreads();
        auto fetch = [&](int h) {
            if (h < H && rows > 0) {
                const uint32_t to = at + (h % kStages) * kTileBytes<D>;
                constexpr int kChunks = D / 8;
                for (int i = tid; i < kTileKeys * kChunks; i += kThreads) {
                    const int row = i / kChunks, ch = i - row * kChunks;
                    const long long p = place[row];
                    cp_async16(to + chunk_at<D>(row, ch), c.cache.k + (p < 0 ? 0 : p + h * c.cache.k_head + ch * 16), p < 0 ? 0 : 16);
                }
            }
            cp_async_commit();
        };
        for (int h = 0; h < kStages - 1; ++h) fetch(h);
        float sum[2] = {0.f, 0.f};
        for (int h = 0; h < H && rows > 0; ++h) {
            cp_async_wait<kStages - 2>();
            __syncthreads();
            fetch(h + kStages - 1);
            const uint32_t tile_at = at + (h % kStages) * kTileBytes<D>;
            const int k_row = warp * 16 + (lane & 15), k_ch = lane >> 4;
            uint32_t k[D / 16][4];
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) ldmatrix_x4(k[ks], tile_at + chunk_at<D>(k_row, ks * 2 + k_ch));
            for (int row0 = 0; row0 < rows; row0 += 8) {
                // column lane / 4 of the right operand; the result's columns are 2 quad and 2 quad + 1
                const int row = row0 + row8, tok = row / G;
                const T* from = static_cast<const T*>(c.x.q) + (token0 + (long long)tok) * c.x.q_token + (h * G + row - tok * G) * c.x.q_head;
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t b0 = row < rows ? *reinterpret_cast<const uint32_t*>(from + ks * 16 + quad * 2) : 0u;
                    const uint32_t b1 = row < rows ? *reinterpret_cast<const uint32_t*>(from + ks * 16 + quad * 2 + 8) : 0u;
                    mma_16816(s, k[ks], b0, b1, T());
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = row0 + quad * 2 + e, t = col / G;
                    if (col >= rows) continue;
                    const float lse = c.x.lse[(token0 + (long long)t) * c.x.lse_token + h * G + col - t * G];
                    const float base = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;      // a row without keys
                    const int lim = limit + (c.causal ? t : 0), key = key0 + warp * 16 + row8;
                    if (key < lim) sum[0] += ex2(s[e] * c.scale - base);
                    if (key + 8 < lim) sum[1] += ex2(s[2 + e] * c.scale - base);
                }
            }
        }
        cp_async_wait<0>();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 1);
            sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 2);
            const int in = warp * 16 + row8 + 8 * u;
            if (quad == 0 && in < keys) {
                const int p = key0 + in;
                c.new_score[r * c.new_ld + p] = (p < len - n ? c.decay * c.score[r * c.ld + p] : 0.f) + sum[u];
            }
        }
    }
}

template <typename T, int D> bool launch(const Weights& c, int sms, cudaStream_t st) {
    if (cudaFuncSetAttribute(weights_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared<D>) != cudaSuccess) return false;
    return launch_early(tiles_kernel, 1, kPlanThreads, 1, 0, st, c) && launch_early(weights_kernel<T, D>, 3 * sms, kThreads, 1, kShared<D>, st, c);
}
template <typename T> bool launch_width(const Weights& c, int width, int sms, cudaStream_t st) {
    switch (width) {
        case 64: return launch<T, 64>(c, sms, st);
        case 80: return launch<T, 80>(c, sms, st);
        case 96: return launch<T, 96>(c, sms, st);
        default: return launch<T, 128>(c, sms, st);
    }
}

}  // namespace

extern "C" int64_t ardiff_attend_weights_workspace(int32_t requests) {
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS) return ARDIFF_ERR_SHAPE;
    return ((int64_t)requests + 1) * 8;
}

extern "C" int ardiff_attend_weights(const void* q, int64_t q_token, int64_t q_head, int32_t q_heads, int64_t tokens, int32_t dtype,
                                     const void* k_cache, int64_t k_page, int64_t k_token, int64_t k_head, int32_t pages, int32_t page,
                                     int32_t heads, int32_t head_width, const int32_t* table, int32_t width, int32_t requests,
                                     const int32_t* length, const int32_t* offset, const int32_t* first, const float* lse,
                                     int64_t lse_token, const float* score, int64_t ld, int32_t most, float scale, float decay, int32_t causal,
                                     float* new_score, int64_t new_ld, int32_t* status, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
    if (requests < 0 || requests > ARDIFF_PAGES_MAX_REQUESTS || tokens < 0 || heads < 1 || q_heads < heads || q_heads % heads ||
        q_heads > ARDIFF_ROTARY_MAX_HEADS || tokens * q_heads >= (int64_t)1 << 31 || pages < 0 || page < 1 || width < 0 ||
        (int64_t)page * width >= (int64_t)1 << 31 || most < 0 || ld < 0 || new_ld < 0 || !isfinite(scale) || !isfinite(decay))
        return ARDIFF_ERR_SHAPE;
    if ((dtype != ARDIFF_BF16 && dtype != ARDIFF_F16) || (head_width != 64 && head_width != 80 && head_width != 96 && head_width != 128))
        return ARDIFF_ERR_UNSUPPORTED;
    if (!status || !offset || !workspace) return ARDIFF_ERR_NULL;
    if (requests > 0 && (!length || (width > 0 && !table) || !k_cache || !score || !new_score)) return ARDIFF_ERR_NULL;
    if (tokens > 0 && (!q || !lse)) return ARDIFF_ERR_NULL;
    auto low = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if (((low(q) | low(k_cache)) & 15u) || (low(workspace) & 15u) || ((q_token | q_head | k_page | k_token | k_head) & 7)) return ARDIFF_ERR_ALIGN;
    if (workspace_bytes < ardiff_attend_weights_workspace(requests)) return ARDIFF_ERR_SHAPE;
    const int sms = device_sms();
    if (sms < 1) return ARDIFF_ERR_CUDA;
    Weights c;
    memset(&c, 0, sizeof(c));
    c.cache.k = static_cast<const char*>(k_cache); c.cache.k_page = k_page * 2; c.cache.k_token = k_token * 2; c.cache.k_head = k_head * 2;
    c.cache.table = table; c.cache.width = width; c.cache.page = page; c.cache.pages = pages; c.cache.heads = heads;
    c.x.q = q; c.x.lse = const_cast<float*>(lse); c.x.q_token = q_token; c.x.q_head = q_head; c.x.lse_token = lse_token;
    c.x.heads = q_heads; c.x.G = q_heads / heads; c.x.tokens = tokens;
    c.length = length; c.offset = offset; c.first = first; c.score = score; c.new_score = new_score; c.status = status;
    c.tiles = static_cast<long long*>(workspace);
    c.ld = ld; c.new_ld = new_ld;
    const int64_t cap = (int64_t)page * width, rows = ld < new_ld ? ld : new_ld;
    c.limit = cap < rows ? cap : rows;
    c.scale = scale * 1.4426950408889634f; c.decay = decay;
    c.requests = requests; c.causal = causal != 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool ok = dtype == ARDIFF_F16 ? launch_width<__half>(c, head_width, sms, st) : launch_width<__nv_bfloat16>(c, head_width, sms, st);
    ardiff::set_launch_count(2);
    return ok ? ARDIFF_OK : ARDIFF_ERR_CUDA;
}
