// What the kernels of attention over pages share: the cache, the plan of a call's work, the pieces of results that are joined.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ardiff.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace ardiff {

// n / d for n < 2^31
struct Divide {
    uint32_t d, m, s;
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return d == 1 ? n : __umulhi(n, m) >> s; }
};
// m = 2^(32 + s) / d rounded up with 2^s < d <= 2^(s + 1): exact for n < 2^31, since m d - 2^(32 + s) < d <= 2^(s + 1)
inline Divide divide_by(uint32_t d) {
    uint32_t s = 0;
    while (d > 1 && (2u << s) < d) ++s;
    return Divide{d, d > 1 ? (uint32_t)((((uint64_t)1 << (32 + s)) + d - 1) / d) : 0u, s};
}

struct Pages {                                   // strides in 16 bytes
    const char* k;
    const char* v;
    uint32_t k_page, k_token, k_head, v_page, v_token, v_head;
    const int32_t* table;
    int width, page, pages, heads;
    Divide by_page;
};

// A byte offset in a cache.
__device__ __forceinline__ long long offset_of(uint32_t page_stride, uint32_t token_stride, uint32_t head_stride, int id, uint32_t row, int h) {
    return (long long)(((unsigned long long)(uint32_t)id * page_stride + (unsigned long long)row * token_stride + (unsigned long long)(uint32_t)h * head_stride) << 4);
}

// Query rows that look at the same keys together. A segment is the new tokens of one request, or of a group of requests that share
// their first tokens; row j of it is token token0 + j / G, query head h G + j % G (G: query heads a kv head). A block is some rows of a segment, up to 16 or
// 32 in the list of narrow blocks (a whole segment), 256 in that of wide ones, and the keys that they see, key0 .. key0 + keys - 1. Its row j sees those from `low` on (wide
// blocks begin at a multiple of their tiles) and below limit + step * (j / G). The first `split` pages are found through row `front` of the table, the
// others through row `request`.
struct alignas(16) Block {
    int token0, row0, rows, request, key0, keys, low, limit, step, split, front, pad;
    long long first_step, first_row;             // steps and rows of the list's blocks before
};

struct PlanHead {
    long long steps;                             // of all blocks: key tiles times kv heads (narrow: times teams of heads)
    long long rows_before;                       // of the other list, in front of this one's among the pieces
    int blocks, own;                             // blocks [0, own): shared tokens; [own, blocks): the requests' own
    int all_rows, pad;                           // whether there are rows to join beside those of units that are cut
};

// Of a request: the first block of its group's shared tokens (-1: none), in which list, and its first row there; how many shared tokens it does not read
// itself; how many pages it finds through another row of the table.
struct Share {
    int prefix, wide, row0, shared, split, front, pad0, pad1;
};

constexpr int kNarrowRows = 32, kNarrowKeys = 16, kWideRows = 256, kWideKeys = 128;
template <bool kWide> struct Sizes {
    static constexpr int rows = kWide ? kWideRows : kNarrowRows, keys = kWide ? kWideKeys : kNarrowKeys;
};

struct List {
    PlanHead* head;
    Block* block;
    long long* steps;                            // [blocks + 1]: steps of the blocks before
    int workers;                                 // that share its steps: CTAs of the wide kernel, teams of the narrow one
};

struct Plan {
    List narrow, wide;
    Share* share;                                // [requests]
    int narrow_rows;                             // of a segment, at most, for it to be narrow: 16 or 32
    int team;                                    // warps of the narrow kernel, a kv head each, that go through the same keys: 1, 2, 4 or 8
};

struct Queries {                                 // strides in values
    const void* q;
    void* out;
    float* lse;
    long long q_token, q_head, out_token, out_head, lse_token;
    int heads, G;
    long long tokens;
    Divide by_G;
};

// Results of a unit (a block and a kv head) in pieces: one of every worker that went on with it, in that worker's place, and in front of all those the piece of
// the worker that began it: in its rows' own place (narrow blocks' rows, then wide ones'), or, where no units are joined with others' and there are more rows
// than that takes, in a second place of the worker, which leaves at most one unit unfinished. Values are relative to the piece's base, in powers of two (its maximum, or somewhat less), and lie
// four of a row together, the rows of the block behind one another, so that threads with a row each write side by side.
struct Pieces {
    float* o;                                    // a piece: [width / 4][rows of the block][4]
    float2* ml;                                  // [rows]: base, sum
    long long narrow_rows, wide_rows;            // where the workers' places begin
    int narrow_cap, wide_cap;                    // rows of a place: of a block, at most
    int begun;                                   // whether workers have a second place, as many rows in front
};

struct Call {
    Pages cache;
    Queries x;
    Plan plan;
    Pieces pieces;
    const int32_t* length;
    const int32_t* offset;
    const int32_t* group;
    const int32_t* shared;
    int32_t* status;
    float scale;                                 // times log2 e
    int requests, groups, causal, most;          // most: new tokens of a request, 0: not known
};

template <bool kWide> __device__ __forceinline__ const List& list_of(const Call& c) { return kWide ? c.plan.wide : c.plan.narrow; }

// The steps of a worker: the same number for all but the last ones. A narrow one (16 keys) has at least 4, so that joining the
// pieces (a row of fp32 values each) does not take longer than reading the keys.
template <bool kWide> __device__ __forceinline__ long long steps_each(long long steps, int workers) {
    return max(kWide ? 1ll : 4ll, (steps + workers - 1) / workers);
}
// a / b for numbers that hardly ever need 64 bits
__device__ __forceinline__ int quotient_of(long long a, long long b) {
    return (a | b) >> 32 ? (int)(a / b) : (int)((uint32_t)a / (uint32_t)b);
}

// A worker's place for kv head h (a team of narrow workers has as many).
template <bool kWide> __device__ __forceinline__ long long place_row(const Call& c, int h, int worker) {
    return kWide ? c.pieces.wide_rows + (long long)worker * c.pieces.wide_cap
                 : c.pieces.narrow_rows + ((long long)worker * c.plan.team + h % c.plan.team) * c.pieces.narrow_cap;
}
// Where the piece of the worker that began a unit lies.
template <bool kWide> __device__ __forceinline__ long long first_row(const Call& c, long long rows_before, const Block& k, int h, int worker) {
    return c.pieces.begun ? place_row<kWide>(c, h, worker) - c.pieces.narrow_rows : (rows_before + k.first_row) * c.cache.heads + (long long)h * k.rows;
}
template <bool kWide> __device__ __forceinline__ long long piece_row(const Call& c, long long rows_before, const Block& k, int h, int worker, int first) {
    return worker != first ? place_row<kWide>(c, h, worker) : first_row<kWide>(c, rows_before, k, h, worker);
}

__device__ __forceinline__ float* piece_values(const Call& c, long long piece, int width, int rows, int row, int value) {
    return c.pieces.o + piece * width + ((long long)(value >> 2) * rows + row) * 4 + (value & 3);
}

// Where a wide worker is in the line of steps: block, head, tile of keys.
struct Cursor {
    int b, h, tile, tiles;
    Block at;
    __device__ __forceinline__ void enter(const Call& c) {
        at = c.plan.wide.block[b];
        tiles = (at.keys + kWideKeys - 1) / kWideKeys;
    }
    __device__ __forceinline__ void start(const Call& c, int block, long long step) {
        b = block;
        enter(c);
        const int in = (int)(step - at.first_step);          // heads times tiles of a block: below 2^31
        h = in / tiles;
        tile = in - h * tiles;
    }
    // (only called while there is a next step)
    __device__ __forceinline__ void next(const Call& c) {
        if (++tile < tiles) return;
        tile = 0;
        if (++h < c.cache.heads) return;
        h = 0;
        do {
            ++b;
            enter(c);
        } while (tiles == 0);
    }
};

// The offsets of key `j` of the tile at `load` in the caches of keys and values, -1 for none.
__device__ __forceinline__ longlong2 place_of(const Call& c, const Cursor& load, int j) {
    const int in = load.tile * kWideKeys + j;
    if (in >= load.at.keys) return make_longlong2(-1, -1);
    const unsigned key = load.at.key0 + in, pg = c.cache.by_page.quotient(key), row = key - pg * c.cache.page;
    const int id = c.cache.table[(long long)((int)pg < load.at.split ? load.at.front : load.at.request) * c.cache.width + pg];
    if (id < 0 || id >= c.cache.pages) {
        *c.status = ARDIFF_ERR_SHAPE;
        return make_longlong2(-1, -1);
    }
    return make_longlong2(offset_of(c.cache.k_page, c.cache.k_token, c.cache.k_head, id, row, load.h),
                          offset_of(c.cache.v_page, c.cache.v_token, c.cache.v_head, id, row, load.h));
}

// The wide blocks (attend_wide.cu).
bool launch_wide(const Call& c, int32_t dtype, int width, cudaStream_t st);

// The last of n + 1 ascending numbers x[0] = 0 .. x[n] that is not above s < x[n]. All lanes of a warp call it with the same arguments.
__device__ __forceinline__ int find_last(const long long* x, int n, long long s) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n;                          // x[lo] <= s < x[hi]
    while (hi - lo > 1) {
        const int step = (hi - lo + 32) / 33;
        const int at = lo + (lane + 1) * step;
        const bool below = at < hi && x[at] <= s;
        const int k = __popc(__ballot_sync(0xffffffffu, below));   // probes ascend, so these are the first k
        const int up = lo + (k + 1) * step;
        lo += k * step;
        hi = up < hi ? up : hi;
    }
    return lo;
}

// Pairs of 16-bit values. Weights are relative to 2^kLift below the highest score so far, which may be passed by 2^kSlack in all before it moves: in f16, whose
// largest number is 2^16, weights of 2^7 for the highest score and up to 2^15, so that keys 2^21 lighter than the heaviest still have all their bits as operands
// (with weights of 1 for the highest those of 2^-14 and less, which can be many behind one heavy key, lost theirs). bf16 has the range of fp32.
template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    static constexpr bool kBf16 = true;
    static constexpr float kLift = 0.f, kSlack = 8.f;
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ float rounded(float a) { return __bfloat162float(__float2bfloat16_rn(a)); }
    static __device__ __forceinline__ bool not_finite(uint32_t p) { return (p & 0x7f800000u) == 0x7f800000u || (p & 0x7f80u) == 0x7f80u; }
};
template <> struct Pair<__half> {
    static constexpr bool kBf16 = false;
    static constexpr float kLift = 7.f, kSlack = 15.f;
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ float rounded(float a) { return __half2float(__float2half_rn(a)); }
    static __device__ __forceinline__ bool not_finite(uint32_t p) { return (p & 0x7c000000u) == 0x7c000000u || (p & 0x7c00u) == 0x7c00u; }
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

constexpr unsigned long long kWaitLimit = 4000000000ull;   // ns

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

// Copies that a warp which gave up has sent for: they land before shared memory is given back. Copy i is step i's, into stage i % stages; `sent`
// have been sent. Bounded, as all waits.
__device__ __forceinline__ void wait_for_copies(uint32_t bars, int full, uint32_t sent, uint32_t stages) {
    for (uint32_t i = sent > stages ? sent - stages : 0; i < sent; ++i)
        for (int j = 0; j < 1 << 20 && !ptx::mbar_try_wait(bars + (full + i % stages) * 8, (i / stages) & 1); ++j) {}
}

// 16-byte chunk c of row `row` of a tile of rows of D values: chunks change places with the row, or rows are a chunk longer than their values, so
// that the eight rows of a matrix lie in different banks.
template <int D> constexpr int kPitch = D % 64 ? 2 * D + 16 : 2 * D;
template <int D> __device__ __forceinline__ uint32_t chunk_at(int row, int c) {
    return row * kPitch<D> + ((D % 64 ? c : c ^ (row & 7)) << 4);
}

__device__ __forceinline__ long long warp_inclusive(long long v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += up;
    }
    return v;
}
// Exclusive sum over a CTA's 1024 threads, and the total; `s` holds 32 values.
__device__ __forceinline__ long long cta_scan(long long v, long long* s, long long* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long inc = warp_inclusive(v);
    __syncthreads();
    if (lane == 31) s[warp] = inc;
    __syncthreads();
    const long long w = warp_inclusive(s[lane]);
    *total = __shfl_sync(0xffffffffu, w, 31);
    const long long before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return inc - v + (warp ? before : 0);
}

// an arrival on the barrier once this thread's copies so far have landed
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
}

// a b + c
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// byte of 16-byte chunk c of a row of D values, in tiles of blocks of 64 values
__device__ __forceinline__ uint32_t swizzled(int row, int c) {
    return (uint32_t)((c >> 3) * 16384 + row * 128 + (((c & 7) ^ (row & 7)) << 4));
}

// The strides of a cache of 16-bit values in 16 bytes; false where one is negative or too large (those of what there is one of may be anything).
inline bool strides_of(int64_t page, int64_t token, int64_t head, const Pages& p, uint32_t& to_page, uint32_t& to_token, uint32_t& to_head) {
    if (p.pages <= 1) page = 0;
    if (p.page == 1) token = 0;
    if (p.heads == 1) head = 0;
    if (page < 0 || token < 0 || head < 0 || (page | token | head) >> 35) return false;
    to_page = (uint32_t)(page / 8); to_token = (uint32_t)(token / 8); to_head = (uint32_t)(head / 8);
    return true;
}

// A cache as an array of four dimensions for TMA (tokens of a page, heads, pages), in boxes of `tokens` tokens and 64 values of a head, swizzled by
// 128 bytes. False where it cannot be described so (strides of 2^40 bytes or 0, no page): it is copied by 16 bytes then.
bool describe(CUtensorMap* map, const char* base, bool bf16, int width, int tokens, const Pages& p, uint32_t token, uint32_t head, uint32_t page);
// Queries as an array of three dimensions (heads, tokens), in boxes of the G heads of a kv head, of `rows` / G tokens and of 64 values: `rows` rows in the
// order of the blocks. False where G does not divide `rows` or the strides do not fit.
bool describe_queries(CUtensorMap* map, const Queries& x, bool bf16, int width, int rows);
// The largest power of two of tokens, up to 128, that divides a page; 0 where it is below the 8 rows of a swizzled block.
int box_tokens(int page);

}  // namespace ardiff
