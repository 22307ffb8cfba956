// The gradient of an embedding, added to its fp32 accumulator: acc[tok_i, :] += s * g[i, :] (include/solo.h).
//
// Two launches for up to 65,536 tokens.  The first puts the tokens and their positions in order, equal tokens in the order they came in: up
// to RANK_MOST of them by counting, for every token, those that come before it; more in the shared memory of a cluster of up to sixteen
// CTAs, least significant digit first.  Then a CTA takes 128 entries of the sorted
// order and 256 or 128 columns, a warp 16 of these entries.  A warp sums the rows of each run of equal tokens in registers; runs that
// lie in one warp's entries are added to the accumulator at once, the pieces of others are put together in shared memory, and those of
// runs that reach into other CTAs in the workspace, by the CTA that finishes last, in their order.  So every row of the
// accumulator is read and written once, without atomics and in an order that the tokens alone decide, and a CTA has the
// same number of rows whatever the tokens are: frequent ones cost no more than rare ones.
//
// A few tokens take one launch: a CTA per token and 256 columns looks for the same token in the whole list and, if its
// own is the first, sums the rows.
#include "solo.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "solo_device.cuh"
#include "solo_host.h"

namespace solo {
namespace {

namespace cg = cooperative_groups;

constexpr int SORT_CTA = 256;
constexpr int SORT_WARPS = SORT_CTA / 32;
constexpr int SORT_CLUSTER = 16;                       // most CTAs of the sort
constexpr int SORT_PER_CTA = 4096;                     // most tokens of one of them
constexpr int SORT_AIM = 1024;                         // tokens per CTA that the cluster's size aims at
constexpr int CHUNK = SORT_CLUSTER * SORT_PER_CTA;     // tokens per pair of launches
constexpr int DIGIT_MAX = 9, DIGITS = 1 << DIGIT_MAX;

constexpr int ROWS_WARPS = 8, ROWS_CTA = ROWS_WARPS * 32;   // of the summing kernel
constexpr int WARP_ROWS = 16, CTA_ROWS = ROWS_WARPS * WARP_ROWS;
constexpr int REACH = 8;                               // entries of the next CTA that a run's end may take up and stay whole
constexpr double AHEAD = 48e6;                         // bytes brought to L2 while the sort runs, at most
constexpr int WIDE = 8, NARROW = 4;                    // columns of a lane; a CTA has 32 times as many

struct SortArgs {
    const void* tokens;
    int32_t token_bytes, num_tokens, num_rows;
    int32_t log_per_cta;        // each CTA holds 2^log_per_cta places of the order
    int32_t digit_bits, passes;
    uint32_t* tok;              // [num_tokens] sorted; num_rows: outside the table
    uint16_t* pos;              // [num_tokens] position of each in the chunk
    uint32_t* counters;         // zeroed for the kernel after
    int32_t num_counters;
};

struct SortShared {
    uint2 item[2][SORT_PER_CTA];                // token, position
    uint16_t hist[SORT_WARPS][DIGITS];          // of each warp, then how many of a digit lie in the warps before
    uint32_t total[SORT_CLUSTER][DIGITS];       // of each CTA
    uint32_t base[DIGITS];                      // first place of a digit's tokens of this CTA
    uint32_t scan[SORT_WARPS];
};

// The time goes into latencies (16,384 tokens, two passes: 1024 threads in eight CTAs 12.5 us, 256 threads in sixteen 9.6 us).
// ROUNDS: tokens per thread, at most; BITS: of a digit, at most.
template <int ROUNDS, int BITS> __global__ __launch_bounds__(SORT_CTA) void rows_sort_kernel(const __grid_constant__ SortArgs a) {
    constexpr uint32_t ALL = 0xFFFFFFFFu, NONE = 0xFFFFFFFFu;
    extern __shared__ __align__(16) unsigned char smem[];
    SortShared& s = *reinterpret_cast<SortShared*>(smem);
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int me = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    pdl_wait();
    pdl_release();
    cluster.barrier_arrive();                   // every CTA has started before its memory is written
    const int per_cta = 1 << a.log_per_cta;
    const int first = me * per_cta;
    const int count = min(max(a.num_tokens - first, 0), per_cta);
    const int rounds = (per_cta + SORT_CTA - 1) / SORT_CTA;
    const uint32_t digits = 1u << a.digit_bits;
    // A warp's tokens follow one another; first from global memory, then from this CTA's places.  (Without conditions, so that the
    // loads are under way together: places without a token read the last one.)
    uint2 item[ROUNDS];
    uint32_t rank[ROUNDS];
    int64_t token[ROUNDS];
    const auto from = [&](int r) { return min(first + (warp * rounds + min(r, rounds - 1)) * 32 + lane, a.num_tokens - 1); };
    if (a.token_bytes == 8) {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) token[r] = ((const int64_t*)a.tokens)[from(r)];
    } else {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) token[r] = ((const int32_t*)a.tokens)[from(r)];
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        item[r] = make_uint2(token[r] >= 0 && token[r] < a.num_rows ? (uint32_t)token[r] : (uint32_t)a.num_rows, (uint32_t)(first + (warp * rounds + r) * 32 + lane));
    for (int i = me * SORT_CTA + tid; i < a.num_counters; i += ctas * SORT_CTA) a.counters[i] = 0;
    cluster.barrier_wait();
    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * a.digit_bits, to_buf = p & 1;
        for (uint32_t i = lane; i < digits / 2; i += 32) reinterpret_cast<uint32_t*>(s.hist[warp])[i] = 0;
        if (digits < 2 && lane == 0) s.hist[warp][0] = 0;
        __syncwarp();
        // Place of every token among those of its digit in its warp.  Lanes with the same digit: a vote for each of its bits (a
        // match over the warp takes a step for each distinct digit).
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if (r < rounds) {
                const bool have = (warp * rounds + r) * 32 + lane < count;
                const uint32_t d = (item[r].x >> shift) & (digits - 1);
                uint32_t peers = __ballot_sync(ALL, have);
#pragma unroll
                for (int b = 0; b < BITS; ++b) {
                    const bool bit = (d >> b) & 1;
                    const uint32_t vote = __ballot_sync(ALL, bit);
                    peers &= bit ? vote : ~vote;
                }
                rank[r] = have ? peers : 0;
            }
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if (r < rounds) {
                const uint32_t peers = rank[r], before = peers & ((1u << lane) - 1u);
                uint16_t* const h = &s.hist[warp][(item[r].x >> shift) & (digits - 1)];
                const uint32_t seen = peers ? *h : 0;
                __syncwarp();
                if (peers && before == 0) *h = (uint16_t)(seen + __popc(peers));
                __syncwarp();
                rank[r] = peers ? seen + __popc(before) : NONE;
            }
        }
        __syncthreads();
        // Over the warps, then over the CTAs; a thread has one or two digits, next to each other.
        const int own = digits > SORT_CTA ? 2 : 1;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t d = tid * own + k;
            if (k < own && d < digits) {
                uint32_t h[SORT_WARPS], sum = 0;
#pragma unroll
                for (int w = 0; w < SORT_WARPS; ++w) h[w] = s.hist[w][d];
#pragma unroll
                for (int w = 0; w < SORT_WARPS; ++w) {
                    s.hist[w][d] = (uint16_t)sum;
                    sum += h[w];
                }
                for (int r = 0; r < ctas; ++r) cluster.map_shared_rank(&s, r)->total[me][d] = sum;
            }
        }
        cluster.sync();
        uint32_t all[2] = {0, 0}, mine[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t d = tid * own + k;
            if (k < own && d < digits)
                for (int r = 0; r < ctas; ++r) {
                    if (r == me) mine[k] = all[k];
                    all[k] += s.total[r][d];
                }
        }
        uint32_t upto = all[0] + all[1];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(ALL, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) s.scan[warp] = upto;
        __syncthreads();
        uint32_t start = upto - all[0] - all[1];
#pragma unroll
        for (int w = 0; w < SORT_WARPS; ++w) start += w < warp ? s.scan[w] : 0;
        if ((uint32_t)(tid * own) < digits) {
            s.base[tid * own] = start + mine[0];
            if (own == 2) s.base[tid * 2 + 1] = start + all[0] + mine[1];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if (r < rounds && rank[r] != NONE) {
                const uint32_t d = (item[r].x >> shift) & (digits - 1);
                const uint32_t to = s.base[d] + s.hist[warp][d] + rank[r];
                cluster.map_shared_rank(&s, to >> a.log_per_cta)->item[to_buf][to & (uint32_t)(per_cta - 1)] = item[r];
            }
        }
        cluster.sync();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            item[r] = s.item[to_buf][min((warp * rounds + r) * 32 + lane, SORT_PER_CTA - 1)];
        }
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int j = (warp * rounds + r) * 32 + lane;
        if (r < rounds && j < count) {
            a.tok[first + j] = item[r].x;
            a.pos[first + j] = (uint16_t)item[r].y;
        }
    }
}

// Two sums in one instruction.
__device__ __forceinline__ void add_pair(float& a, float& b, float x, float y) {
    asm("{ .reg .b64 s, t; mov.b64 s, {%0, %1}; mov.b64 t, {%2, %3}; add.rn.f32x2 s, s, t; mov.b64 {%0, %1}, s; }" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}

// The place of every token is the number of tokens that are smaller, or equal and before it: a lane per token, an eighth of the tokens
// per warp.  n^2 comparisons, but no step that waits for another CTA (rank_first() has the times of both).  A comparison is the
// saturation of a difference of whole numbers, exactly 0 or 1, on the pipe for fp32, which takes a warp every cycle where integer
// comparisons take one every other.
constexpr int RANK_MOST = 4096, RANK_ROWS = (1 << 24) - 2;

__global__ __launch_bounds__(SORT_CTA) void rows_rank_kernel(const __grid_constant__ SortArgs a) {
    __shared__ __align__(16) float key[RANK_MOST];
    __shared__ float part[SORT_WARPS][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.num_tokens;
    pdl_wait();
    pdl_release();
    const int quads = (n + 3) / 4;
    const auto load = [&](auto tokens) {
#pragma unroll 8
        for (int j = tid; j < 4 * quads; j += SORT_CTA) {
            const int64_t t = tokens[min(j, n - 1)];
            key[j] = j >= n ? __int_as_float(0x7F800000) : (float)(t >= 0 && t < a.num_rows ? (int)t : a.num_rows);
        }
    };
    if (a.token_bytes == 8) load((const int64_t*)a.tokens);
    else load((const int32_t*)a.tokens);
    for (int i = blockIdx.x * SORT_CTA + tid; i < a.num_counters; i += gridDim.x * SORT_CTA) a.counters[i] = 0;
    __syncthreads();
    const int i0 = blockIdx.x * 32, i = i0 + lane;
    const float t = key[min(i, n - 1)];
    const int lo = quads * warp / SORT_WARPS, hi = quads * (warp + 1) / SORT_WARPS;         // in quads, as this CTA's own tokens: q0 to q0 + 7
    const int q0 = i0 / 4;
    const float4* const quad = reinterpret_cast<const float4*>(key);
    float before[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const auto count = [&](int from, int to, float limit) {
#pragma unroll 8
        for (int q = from; q < to; ++q) {
            const float4 k = quad[q];
            add_pair(before[0], before[1], __saturatef(limit - k.x), __saturatef(limit - k.y));
            add_pair(before[2], before[3], __saturatef(limit - k.z), __saturatef(limit - k.w));
        }
    };
    count(lo, min(hi, q0), t + 1.0f);
    for (int j = 4 * max(lo, q0); j < 4 * min(hi, q0 + 8); ++j) before[0] += __saturatef(t + (j < i ? 1.0f : 0.0f) - key[j]);
    count(max(lo, q0 + 8), hi, t);
    part[warp][lane] = (before[0] + before[1]) + (before[2] + before[3]);
    __syncthreads();
    if (warp == 0 && i < n) {
        float place = 0.0f;
#pragma unroll
        for (int w = 0; w < SORT_WARPS; ++w) place += part[w][lane];
        a.tok[(int)place] = (uint32_t)t;
        a.pos[(int)place] = (uint16_t)i;
    }
}

struct RowsArgs {
    float* acc;
    const void* grad;
    const uint32_t* tok;
    const uint16_t* pos;
    float* partial;             // [2 CTAs, width]: pieces that continue a run, then runs' first pieces
    uint32_t* counters;         // [CTAs, slabs] pieces done, at a run's first CTA
    int64_t width, grad_stride;
    int32_t num_tokens, num_rows, slabs;
    float scale;
    // what is brought to L2 while the sort runs: rows of gradients, and with `tokens` (the unsorted ones) of the accumulator
    const void* tokens;
    int32_t token_bytes, ahead_ctas, ahead_rows;
};

// Loads that are issued where they are written, so that those of several rows are under way together: a compiler may move a
// plain one down to where it is used.  With `on` false nothing is loaded and the result is what it was.
__device__ __forceinline__ void load16_once(uint4& v, const void* p) {
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
}
__device__ __forceinline__ void load8_once(uint2& v, const void* p) {
    asm volatile("ld.global.cs.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
}
__device__ __forceinline__ void load16_acc(float (&v)[4], const float* p, bool on) {
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %5, 0; @q ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4]; }"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]) : "l"(p), "r"((uint32_t)on) : "memory");
}
__device__ __forceinline__ void load4_acc(float& v, const float* p, bool on) {
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q ld.global.cg.f32 %0, [%1]; }" : "+f"(v) : "l"(p), "r"((uint32_t)on) : "memory");
}
// (what is not loaded here is of no use)
__device__ __forceinline__ void load16_once(uint4& v, const void* p, bool on) {
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %5, 0; @q ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4]; }"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p), "r"((uint32_t)on) : "memory");
}
template <int DT> __device__ __forceinline__ float row_elem(const char* g, int64_t i, bool on) {
    if constexpr (DT == SOLO_DT_F32) {
        float v = 0.0f;
        load4_acc(v, (const float*)g + i, on);
        return v;
    } else {
        uint16_t h = 0;
        asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q ld.global.cs.u16 %0, [%1]; }" : "+h"(h) : "l"(g + 2 * i), "r"((uint32_t)on) : "memory");
        if constexpr (DT == SOLO_DT_BF16) return __uint_as_float((uint32_t)h << 16);
        else return __half2float(__ushort_as_half(h));
    }
}

// RV columns of a thread: consecutive ones and wide accesses (VEC), or one in every 32.  A thread without columns of its own reads
// the last ones again and stores nothing.
template <int DT, bool VEC, int RV> struct Cols {
    static constexpr int WORDS = VEC && DT != SOLO_DT_F32 ? RV / 2 : RV;
    int64_t c0, width;
    bool some;
    __device__ __forceinline__ Cols(int64_t slab, int64_t width_) : width(width_) {
        const int lane = threadIdx.x & 31;
        c0 = slab * (32 * RV) + (VEC ? lane * RV : lane);
        some = c0 < width;
        if (VEC && !some) c0 = width - RV;
    }
    __device__ __forceinline__ int64_t at(int k) const { return VEC ? c0 + k : c0 + k * 32; }
    __device__ __forceinline__ bool in(int k) const { return VEC || at(k) < width; }
    struct Raw { uint32_t w[WORDS]; };
    // of the row that starts at g
    template <class... On> __device__ __forceinline__ Raw load(const char* g, On... on) const {
        Raw r;
        if constexpr (VEC) {
            const char* const p = g + c0 * (DT == SOLO_DT_F32 ? 4 : 2);
            if constexpr (WORDS % 4 == 0) {
#pragma unroll
                for (int q = 0; q < WORDS / 4; ++q) {
                    uint4 v;
                    load16_once(v, p + 16 * q, on...);
                    r.w[4 * q] = v.x; r.w[4 * q + 1] = v.y; r.w[4 * q + 2] = v.z; r.w[4 * q + 3] = v.w;
                }
            } else {
                uint2 v;
                load8_once(v, p);
                r.w[0] = v.x; r.w[1] = v.y;
            }
        } else {
#pragma unroll
            for (int k = 0; k < RV; ++k) r.w[k] = __float_as_uint(row_elem<DT>(g, at(k), (in(k) && ... && on)));
        }
        return r;
    }
    __device__ __forceinline__ static void add(const Raw& r, float (&s)[RV]) {
#pragma unroll
        for (int k = 0; k < RV / 2; ++k) {
            float2 f;
            if constexpr (!VEC || DT == SOLO_DT_F32) f = make_float2(__uint_as_float(r.w[2 * k]), __uint_as_float(r.w[2 * k + 1]));
            else if constexpr (DT == SOLO_DT_BF16) f = make_float2(__uint_as_float(r.w[k] << 16), __uint_as_float(r.w[k] & 0xFFFF0000u));
            else f = __half22float2(*reinterpret_cast<const __half2*>(&r.w[k]));
            add_pair(s[2 * k], s[2 * k + 1], f.x, f.y);
        }
    }
    // v is left as it is unless `on`
    __device__ __forceinline__ void load_f32(const float* p, float (&v)[RV], bool on = true) const {
        if constexpr (VEC) {
#pragma unroll
            for (int q = 0; q < RV / 4; ++q) {
                float f[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                load16_acc(f, p + c0 + 4 * q, on);
                v[4 * q] = f[0]; v[4 * q + 1] = f[1]; v[4 * q + 2] = f[2]; v[4 * q + 3] = f[3];
            }
        } else {
#pragma unroll
            for (int k = 0; k < RV; ++k) load4_acc(v[k], p + at(k), on && in(k));
        }
    }
    __device__ __forceinline__ void store_f32(float* p, const float (&v)[RV]) const {
        if constexpr (VEC) {
            if (some) {
#pragma unroll
                for (int q = 0; q < RV / 4; ++q)
                    reinterpret_cast<float4*>(p + c0)[q] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < RV; ++k) if (in(k)) p[at(k)] = v[k];
        }
    }
};

// How many CTAs a run of token t reaches back into from CTA c, or on into by more than REACH entries: from the tokens next to the CTAs'
// borders, one border a lane.  The first 32 of them are read by the caller ahead of time.
__device__ __forceinline__ uint32_t border_before(const uint32_t* tok, int c, int k) {
    const int e = (c - k - (int)(threadIdx.x & 31)) * CTA_ROWS - 1;
    return e >= 0 ? tok[e] : 0xFFFFFFFFu;
}
__device__ __forceinline__ uint32_t border_after(const uint32_t* tok, int n, int c, int k) {
    const int e = (c + 1 + k + (int)(threadIdx.x & 31)) * CTA_ROWS + REACH;
    return e < n ? tok[e] : 0xFFFFFFFFu;
}
template <class Border> __device__ __forceinline__ int ctas_reached(uint32_t first, uint32_t t, Border border) {
    for (int k = 0;; k += 32) {
        const uint32_t same = __ballot_sync(0xFFFFFFFFu, (k ? border(k) : first) == t);
        if (same != 0xFFFFFFFFu) return k + __ffs(~same) - 1;
    }
}

// The CTAs of the sum that are resident while the sort runs have nothing else to do: they bring rows to L2 (16,384 tokens of 768 columns 34.8 ->
// 32.8 us with nothing in L2 before, 24.5 -> 23.7 us call after call).  Nothing of it is needed, and the tokens read here, before the wait
// for the kernels before, choose addresses in the table and nothing else.
template <int DT> __device__ __forceinline__ void rows_ahead(const RowsArgs& a) {
    constexpr int LINE = 128, ES = DT == SOLO_DT_F32 ? 4 : 2;
    const int threads = a.ahead_ctas * ROWS_CTA, me = blockIdx.x * ROWS_CTA + threadIdx.x;
    const int lines = (int)((a.width * ES + LINE - 1) / LINE);
    for (int64_t i = me; i < (int64_t)a.ahead_rows * lines; i += threads) {
        const char* const p = (const char*)a.grad + (i / lines) * a.grad_stride * ES + (i % lines) * LINE;
        asm volatile("prefetch.global.L2 [%0];" :: "l"(p));
    }
    if (!a.tokens) return;
    const int acc_lines = (int)((a.width * 4 + LINE - 1) / LINE);
    for (int64_t i = me; i < (int64_t)a.num_tokens * acc_lines; i += threads) {
        const int64_t t = a.token_bytes == 8 ? __ldcg((const long long*)a.tokens + i / acc_lines) : (int64_t)__ldcg((const int*)a.tokens + i / acc_lines);
        if (t < 0 || t >= a.num_rows) continue;
        const char* const p = (const char*)(a.acc + t * a.width) + (i % acc_lines) * LINE;
        asm volatile("prefetch.global.L2 [%0];" :: "l"(p));
    }
}

template <int RV> struct SumShared {
    union {
        float open[2][ROWS_WARPS][RV][32];       // pieces of runs that a warp does not hold whole: what continues one, what begins one
        double join[ROWS_WARPS][RV][32];
    };
    struct Entry { const char* grad; float* row; };
    Entry entry[ROWS_WARPS][WARP_ROWS + REACH];         // where the rows of a warp's entries start
    uint32_t head[ROWS_WARPS];                  // 0: the warp's first run is its own; 1: continues one and ends here; 2: goes on
    int32_t job[2][2];                          // runs to put together: first CTA (-1: none), CTAs after it
    uint32_t job_tok[2];
};

template <bool VEC, int RV> constexpr int SUM_CTAS = VEC && RV == WIDE ? 4 : 3;       // per SM

template <int DT, bool VEC, int RV> __global__ __launch_bounds__(ROWS_CTA, SUM_CTAS<VEC, RV>) void rows_sum_kernel(const __grid_constant__ RowsArgs a) {
    constexpr int SLAB = 32 * RV;
    constexpr uint32_t ALL = 0xFFFFFFFFu, NONE = 0xFFFFFFFFu;
    __shared__ SumShared<RV> s;
    if (blockIdx.x < (unsigned)a.ahead_ctas) rows_ahead<DT>(a);
    pdl_wait();
    pdl_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = a.num_tokens, c = (int)(blockIdx.x / (unsigned)a.slabs), slab = (int)(blockIdx.x % (unsigned)a.slabs);
    const int first_of_second = (n + CTA_ROWS - 1) / CTA_ROWS;          // CTAs over the entries: where first pieces start in `partial`
    const int base = c * CTA_ROWS + warp * WARP_ROWS;
    // This warp's entries and what lies around them; tokens outside the table come last and count as none.
    const int e = base - 1 + lane;
    uint32_t around = e >= 0 && e < n ? a.tok[e] : NONE;
    if (around >= (uint32_t)a.num_rows) around = NONE;
    const int pos = lane < WARP_ROWS + REACH && base + lane < n ? a.pos[base + lane] : 0;
    const uint32_t tok = __shfl_down_sync(ALL, around, 1), next = __shfl_down_sync(ALL, around, 2);
    const uint32_t begins = __ballot_sync(ALL, tok != NONE && tok != around);           // of the lanes up to WARP_ROWS + REACH
    const uint32_t finishes = __ballot_sync(ALL, tok != NONE && tok != next);
    // A run that reaches at most REACH entries into the next CTA is left whole: the last warp takes them, the first one of the
    // next CTA leaves them out.
    int skip = 0, count = __popc(__ballot_sync(ALL, lane < WARP_ROWS && tok != NONE));
    if (warp == 0 && count > 0 && !(begins & 1u)) {
        const int k = __ffs(finishes);
        if (k >= 1 && k <= REACH) skip = k;
    }
    if (warp == ROWS_WARPS - 1 && count == WARP_ROWS) {
        const int k = __ffs(finishes >> (WARP_ROWS - 1)) - 1;
        if (k >= 1 && k <= REACH) count += k;
    }
    const uint32_t mine = (1u << count) - (1u << skip);
    const uint32_t ends = finishes & mine;
    const bool some = count > skip;
    const bool continues = some && !(begins >> skip & 1u);              // the first run began before this warp
    const bool goes_on = some && !(ends >> (count - 1) & 1u);           // the last run ends after it
    const bool through = continues && goes_on && ends == 0;             // and these are one
    const Cols<DT, VEC, RV> cols(slab, a.width);
    const uint32_t borders_before = warp == 0 && continues ? border_before(a.tok, c, 0) : NONE;
    const uint32_t borders_after = goes_on ? border_after(a.tok, n, c, 0) : NONE;
    if (threadIdx.x < 2) s.job[threadIdx.x][0] = -1;
    if (lane == 0) s.head[warp] = continues ? (through ? 2 : 1) : 0;
    float sum[RV] = {};
    // Entries whose loads are under way together, few enough for four CTAs per SM (eight columns per lane, 16,384 tokens of 4096
    // columns: 2 in four CTAs 67.1 us, 2 in three 72.1, 4 in three 74.5, 2 in five 79), or three with four columns per lane (768 columns 22.6 us,
    // in four CTAs 23.7) and without wide accesses (4098 columns 91 us, in four CTAs 102, in two 109).  (Of calls on the same inputs one after
    // another; on inputs that change, 768 columns 23.6 us.)
    constexpr int BATCH = RV == WIDE ? 2 : 4;
    constexpr int ES = DT == SOLO_DT_F32 ? 4 : 2;
    if (lane < count) s.entry[warp][lane] = {(const char*)a.grad + pos * a.grad_stride * ES, a.acc + (int64_t)tok * a.width};
    __syncwarp();
    const uint32_t shared_head = continues ? ends & -ends : 0;          // end of a run that began before, if it is here
    const uint32_t whole = ends & ~shared_head;                         // ends of this warp's own runs
    const uint32_t stops = ends | (goes_on ? 1u << (count - 1) : 0u);
    const auto batch = [&](int k, auto full) {
        constexpr bool FULL = decltype(full)::value;
        typename Cols<DT, VEC, RV>::Raw r[BATCH];
        float v[BATCH][RV];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int x = FULL ? k + b : min(k + b, count - 1);
            const typename SumShared<RV>::Entry at = s.entry[warp][x];
            r[b] = cols.load(at.grad);
            cols.load_f32(at.row, v[b], whole >> x & 1u);
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int x = k + b;
            if (!FULL && x >= count) break;
            cols.add(r[b], sum);
            if (stops >> x & 1u) {
                if (whole >> x & 1u) {
#pragma unroll
                    for (int q = 0; q < RV; ++q) v[b][q] = __fmaf_rn(a.scale, sum[q], v[b][q]);
                    cols.store_f32(s.entry[warp][x].row, v[b]);
                } else {
                    // what continues a run: its end, or all of the entries
                    const int which = shared_head >> x & 1u || through ? 0 : 1;
#pragma unroll
                    for (int q = 0; q < RV; ++q) s.open[which][warp][q][lane] = sum[q];
                }
#pragma unroll
                for (int q = 0; q < RV; ++q) sum[q] = 0.0f;
            }
        }
    };
    int k = skip;
    for (; k + BATCH <= count; k += BATCH) batch(k, std::true_type{});
    if (k < count) batch(k, std::false_type{});
    __syncthreads();
    // Runs of several warps, by the warp that holds the first piece: in this CTA, or (warp 0) of a run from a CTA before.
    for (int side = 0; side < 2; ++side) {
        if (side == 0 ? !(warp == 0 && continues) : !(goes_on && !through)) continue;
        bool open = side == 1 || through;
        float v[RV];
#pragma unroll
        for (int q = 0; q < RV; ++q) v[q] = s.open[side][warp][q][lane];
        for (int u = warp + 1; open && u < ROWS_WARPS; ++u) {
#pragma unroll
            for (int q = 0; q < RV; ++q) v[q] += s.open[0][u][q][lane];
            open = s.head[u] == 2;
        }
        const uint32_t t = __shfl_sync(ALL, tok, side == 0 ? 0 : count - 1);
        if (side == 1 && !open) {
            float* const row = a.acc + (int64_t)t * a.width;
            float old[RV];
            cols.load_f32(row, old);
#pragma unroll
            for (int q = 0; q < RV; ++q) old[q] = __fmaf_rn(a.scale, v[q], old[q]);
            cols.store_f32(row, old);
            continue;
        }
        cols.store_f32(a.partial + (int64_t)(side == 0 ? c : first_of_second + c) * a.width, v);
        const int from = side == 0 ? c - ctas_reached(borders_before, t, [&](int k) { return border_before(a.tok, c, k); }) : c;
        const int to = open ? c + ctas_reached(borders_after, t, [&](int k) { return border_after(a.tok, n, c, k); }) : c;
        __threadfence();
        __syncwarp();
        if (lane == 0 && atomicAdd(&a.counters[(int64_t)from * a.slabs + slab], 1u) == (uint32_t)(to - from)) {
            s.job[side][0] = from;
            s.job[side][1] = to - from;
            s.job_tok[side] = t;
        }
    }
    __syncthreads();
    for (int side = 0; side < 2; ++side) {
        const int from = s.job[side][0], more = s.job[side][1];
        if (from < 0) continue;
        __threadfence();
        double d[RV] = {};
#pragma unroll 4
        for (int p = warp; p <= more; p += ROWS_WARPS) {
            float v[RV] = {};
            cols.load_f32(a.partial + (int64_t)(p == 0 ? first_of_second + from : from + p) * a.width, v);
#pragma unroll
            for (int q = 0; q < RV; ++q) d[q] += (double)v[q];
        }
        __syncthreads();                                                // of the other side's sums
#pragma unroll
        for (int q = 0; q < RV; ++q) s.join[warp][q][lane] = d[q];
        __syncthreads();
        for (int q = warp; q < RV; q += ROWS_WARPS) {
            double all = 0.0;
#pragma unroll
            for (int u = 0; u < ROWS_WARPS; ++u) all += s.join[u][q][lane];
            const int64_t col = (int64_t)slab * SLAB + (VEC ? lane * RV + q : q * 32 + lane);
            if (col < a.width) {
                float* const at = a.acc + (int64_t)s.job_tok[side] * a.width + col;
                *at = __fmaf_rn(a.scale, (float)all, *at);
            }
        }
    }
}

// One launch for at most DIRECT_MOST tokens.
constexpr int DIRECT_WORDS = 4;                        // a warp looks at up to four times 32 tokens
constexpr int DIRECT_MOST = ROWS_WARPS * DIRECT_WORDS * 32;

struct DirectArgs {
    float* acc;
    const void* grad;
    const void* tokens;
    int64_t width, grad_stride;
    int32_t token_bytes, num_tokens, num_rows, slabs;
    float scale;
};

template <int DT, bool VEC> __global__ __launch_bounds__(ROWS_CTA, 4) void rows_direct_kernel(const __grid_constant__ DirectArgs a) {
    constexpr int RV = WIDE, SLAB = 32 * RV, ES = DT == SOLO_DT_F32 ? 4 : 2;
    constexpr uint32_t ALL = 0xFFFFFFFFu;
    __shared__ float part[ROWS_WARPS][RV][32];
    __shared__ uint32_t found[ROWS_WARPS];             // 1: the token is among the warp's, 2: before this CTA's
    pdl_wait();
    pdl_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = (int)(blockIdx.x / (unsigned)a.slabs), slab = (int)(blockIdx.x % (unsigned)a.slabs);
    const int n = a.num_tokens, words = (n + ROWS_CTA - 1) / ROWS_CTA;
    const auto token = [&](int j) { return a.token_bytes == 8 ? ((const int64_t*)a.tokens)[j] : (int64_t)((const int32_t*)a.tokens)[j]; };
    const int64_t t = token(i);
    uint32_t m[DIRECT_WORDS];
    bool before = false;
#pragma unroll
    for (int k = 0; k < DIRECT_WORDS; ++k) {
        const int j = (warp * words + k) * 32 + lane;
        const bool same = k < words && j < n && token(j) == t;
        m[k] = __ballot_sync(ALL, same);
        before |= __any_sync(ALL, same && j < i);
    }
    if (t < 0 || t >= a.num_rows) return;
    const bool have = (m[0] | m[1] | m[2] | m[3]) != 0;
    if (lane == 0) found[warp] = (have ? 1u : 0u) | (before ? 2u : 0u);
    __syncthreads();
    const uint32_t all = __ballot_sync(ALL, lane < ROWS_WARPS && found[lane & (ROWS_WARPS - 1)] & 1u);
    if (__any_sync(ALL, found[lane & (ROWS_WARPS - 1)] & 2u)) return;
    const bool alone = (all & (all - 1)) == 0;         // one warp has all the rows
    if (alone && !have) return;
    const Cols<DT, VEC, RV> cols(slab, a.width);
    float* const row = a.acc + t * a.width;
    float old[RV] = {};
    if (alone) cols.load_f32(row, old);
    float total[RV] = {};
    // (with registers for four CTAs per SM: 1000 tokens of 770 columns 10.0 us, with four rows and what they take 14.3; wide accesses to fp32
    // spill 24 bytes under that limit)
    constexpr int BATCH = VEC ? 4 : 2;
#pragma unroll
    for (int k = 0; k < DIRECT_WORDS; ++k) {
        float sum[RV] = {};
        uint32_t left = m[k];
        const char* const rows = (const char*)a.grad + (warp * words + k) * 32 * a.grad_stride * ES;
        while (left) {
            typename Cols<DT, VEC, RV>::Raw r[BATCH];
            uint32_t after = left;
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                r[b] = cols.load(rows + max(__ffs(after) - 1, 0) * a.grad_stride * ES, after != 0);
                after &= after - 1;
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (left == 0) break;
                cols.add(r[b], sum);
                left &= left - 1;
            }
        }
#pragma unroll
        for (int q = 0; q < RV; ++q) total[q] += sum[q];
    }
    if (alone) {
#pragma unroll
        for (int q = 0; q < RV; ++q) old[q] = __fmaf_rn(a.scale, total[q], old[q]);
        cols.store_f32(row, old);
        return;
    }
#pragma unroll
    for (int q = 0; q < RV; ++q) part[warp][q][lane] = total[q];
    __syncthreads();
    const int64_t col = (int64_t)slab * SLAB + (VEC ? lane * RV + warp : warp * 32 + lane);
    if (warp < RV && col < a.width) {
        float v = 0.0f;
#pragma unroll
        for (int u = 0; u < ROWS_WARPS; ++u) v += part[u][warp % RV][lane];
        row[col] = __fmaf_rn(a.scale, v, row[col]);
    }
}

using RowsKernel = void (*)(const RowsArgs);
template <int RV> RowsKernel rows_kernel_of(int dtype, bool vec) {
    switch (dtype) {
        case SOLO_DT_F32: return vec ? rows_sum_kernel<SOLO_DT_F32, true, RV> : rows_sum_kernel<SOLO_DT_F32, false, RV>;
        case SOLO_DT_BF16: return vec ? rows_sum_kernel<SOLO_DT_BF16, true, RV> : rows_sum_kernel<SOLO_DT_BF16, false, RV>;
        default: return vec ? rows_sum_kernel<SOLO_DT_F16, true, RV> : rows_sum_kernel<SOLO_DT_F16, false, RV>;
    }
}
RowsKernel rows_kernel_for(int dtype, bool vec, int rv) { return rv == WIDE ? rows_kernel_of<WIDE>(dtype, vec) : rows_kernel_of<NARROW>(dtype, vec); }

using DirectKernel = void (*)(const DirectArgs);
DirectKernel direct_kernel_for(int dtype, bool vec) {
    switch (dtype) {
        case SOLO_DT_F32: return vec ? rows_direct_kernel<SOLO_DT_F32, true> : rows_direct_kernel<SOLO_DT_F32, false>;
        case SOLO_DT_BF16: return vec ? rows_direct_kernel<SOLO_DT_BF16, true> : rows_direct_kernel<SOLO_DT_BF16, false>;
        default: return vec ? rows_direct_kernel<SOLO_DT_F16, true> : rows_direct_kernel<SOLO_DT_F16, false>;
    }
}

int launch(const void* k, dim3 grid, unsigned threads, size_t smem, int cluster, void** params, cudaStream_t stream) {
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;    // see pdl_wait
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    if (cudaLaunchKernelExC(&cfg, k, params) != cudaSuccess) {
        cudaGetLastError();
        return SOLO_ECUDA;
    }
    count_launch();
    return SOLO_OK;
}

using SortKernel = void (*)(const SortArgs);
SortKernel sort_kernel_for(int rounds, int bits) {
    if (rounds <= 4) return bits <= 8 ? rows_sort_kernel<4, 8> : rows_sort_kernel<4, DIGIT_MAX>;
    return bits <= 8 ? rows_sort_kernel<SORT_PER_CTA / SORT_CTA, 8> : rows_sort_kernel<SORT_PER_CTA / SORT_CTA, DIGIT_MAX>;
}

// Shared memory and clusters of sixteen, opted in to once per device.
int sort_ready(int& device) {
    static std::atomic<bool> done[64];
    device = -1;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) { cudaGetLastError(); return SOLO_ECUDA; }
    if (done[device]) return SOLO_OK;
    for (int rounds : {4, 16})
        for (int bits : {8, DIGIT_MAX}) {
            const void* k = (const void*)sort_kernel_for(rounds, bits);
            if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared)) != cudaSuccess ||
                cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
                cudaGetLastError();
                return SOLO_ECUDA;
            }
        }
    // How an SM is divided into shared memory and L1.  It has to run empty before it is divided another way, so the counting asks for no more
    // than the sum (3000 tokens of 4096 columns 20.3 us, left to itself 24.7); the sum asks for what four of its CTAs take and little more
    // (16,384 tokens of 4096 columns 67.1 us, left to itself 69.5; 30,000 of 1000 columns 51.8 and 58.7).  Wishes: a refusal does not matter.
    cudaFuncSetAttribute((const void*)rows_rank_kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 30);
    for (int dtype : {SOLO_DT_F32, SOLO_DT_BF16, SOLO_DT_F16})
        for (int rv : {NARROW, WIDE})
            for (bool vec : {false, true})
                cudaFuncSetAttribute((const void*)rows_kernel_for(dtype, vec, rv), cudaFuncAttributePreferredSharedMemoryCarveout, 45);
    cudaGetLastError();
    done[device] = true;
    return SOLO_OK;
}

// Whether the order of a chunk comes from counting or from the sort.  Us with the sum, counting and sorting: 2048 tokens of 768 columns 9.2 and
// 11.8, 4096 11.2 and 14.3, 6000 17.4 and 15.7; of 4096 columns 2048 12.5 and 16.0, 3000 20.3 and 21.0, 4096 27.1 and 25.7; 4096
// of 2000 columns 16.0 and 17.2.
bool rank_first(int n, int64_t num_rows, int64_t width) { return n <= (width <= 2048 ? RANK_MOST : 2048) && num_rows <= RANK_ROWS; }

struct RowsLayout { size_t tok, pos, counters, partial, total; };

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

int64_t slabs_of(int64_t width, int rv) { return (width + 32 * rv - 1) / (32 * rv); }

// One launch, without a workspace.  Its CTAs, one for every token and 256 columns, mostly find that their token is not the first
// of its kind: with 4096 of them it takes 8 to 14 us where the sort and the sum take 15 (1024 tokens of 768 columns 7.4 us, 256 of 4096 10).
bool rows_direct(int64_t num_tokens, int64_t width) { return num_tokens <= DIRECT_MOST && num_tokens * slabs_of(width, WIDE) <= 4096; }

RowsLayout rows_layout(int64_t num_tokens, int64_t width) {
    RowsLayout l;
    const int64_t n = std::min<int64_t>(num_tokens, CHUNK), ctas = (n + CTA_ROWS - 1) / CTA_ROWS;
    l.tok = 0;
    l.pos = l.tok + pad256((size_t)n * 4);
    l.counters = l.pos + pad256((size_t)n * 2);
    l.partial = l.counters + pad256((size_t)(ctas * slabs_of(width, NARROW)) * 4);
    l.total = l.partial + pad256((size_t)(2 * ctas) * (size_t)width * 4);
    return l;
}

constexpr int64_t MOST_WIDTH = (int64_t)1 << 24, MOST_TOKENS = (int64_t)1 << 40, MOST_ELEMS = (int64_t)1 << 60;

// Whether `bytes` at a share memory with one of n pieces of `piece` bytes, the first at b and one every `step` bytes.
bool meets(const void* a, size_t bytes, const void* b, int64_t n, size_t piece, size_t step) {
    const uintptr_t lo = (uintptr_t)a, first = (uintptr_t)b;
    if (bytes == 0 || (first > lo && first - lo >= bytes)) return false;                // all of them behind
    if (first > lo || lo - first < piece) return true;
    if (step == 0) return false;
    const uint64_t i = (lo - first - piece) / step + 1;                                 // the first one that ends behind lo
    return i < (uint64_t)n && (first + i * step <= lo || first + i * step - lo < bytes);
}

}  // namespace
}  // namespace solo

using namespace solo;

extern "C" {

int solo_grad_rows_workspace(int64_t num_tokens, int64_t width, size_t* bytes) {
    if (!bytes || num_tokens < 0 || num_tokens > MOST_TOKENS || width < 1 || width > MOST_WIDTH) return SOLO_EINVAL;
    *bytes = rows_direct(num_tokens, width) ? 0 : rows_layout(num_tokens, width).total;
    return SOLO_OK;
}

int solo_grad_accumulate_rows(const solo_grad_rows_t* r, float scale, void* workspace_dev, void* stream_) {
    if (!r || !r->acc || r->num_rows < 1 || r->num_rows >= ((int64_t)1 << 31) || r->width < 1 || r->width > MOST_WIDTH) return SOLO_EINVAL;
    if (r->num_tokens < 0 || r->num_tokens > MOST_TOKENS || (r->token_bytes != 4 && r->token_bytes != 8)) return SOLO_EINVAL;
    if (r->grad_dtype < SOLO_DT_F32 || r->grad_dtype > SOLO_DT_F16 || r->grad_stride < 0 || !std::isfinite(scale)) return SOLO_EINVAL;
    if (r->num_tokens == 0) return SOLO_OK;
    const bool direct = rows_direct(r->num_tokens, r->width);
    if (!r->tokens || !r->grad || (!workspace_dev && !direct)) return SOLO_EINVAL;
    const int es = r->grad_dtype == SOLO_DT_F32 ? 4 : 2;
    if (((uintptr_t)workspace_dev & 15u) || ((uintptr_t)r->acc & 3u) || ((uintptr_t)r->tokens & (unsigned)(r->token_bytes - 1)) ||
        ((uintptr_t)r->grad & (unsigned)(es - 1)))
        return SOLO_EALIGN;
    if (r->grad_stride > MOST_ELEMS || (r->grad_stride && r->num_tokens - 1 > (MOST_ELEMS - r->width) / r->grad_stride)) return SOLO_EINVAL;
    // What is written, acc and the workspace, lies apart from each other and from what is read.
    const RowsLayout l = rows_layout(r->num_tokens, r->width);
    const size_t row = (size_t)r->width * es, acc_bytes = (size_t)r->num_rows * (size_t)r->width * 4, ws_bytes = direct ? 0 : l.total;
    const auto apart = [&](const void* p, size_t bytes) {
        return !meets(p, bytes, r->tokens, r->num_tokens, r->token_bytes, r->token_bytes) &&
               !meets(p, bytes, r->grad, r->num_tokens, row, (size_t)r->grad_stride * es);
    };
    if (!apart(r->acc, acc_bytes) || !apart(workspace_dev, ws_bytes) || meets(workspace_dev, ws_bytes, r->acc, 1, acc_bytes, 0)) return SOLO_EINVAL;
    cudaStream_t stream = (cudaStream_t)stream_;
    const bool vec = r->width % WIDE == 0 && (((uintptr_t)r->acc | (uintptr_t)r->grad) & 15u) == 0 && (r->grad_stride * es) % 16 == 0;
    if (direct) {
        DirectArgs d;
        std::memset(&d, 0, sizeof(d));
        d.acc = r->acc;
        d.grad = r->grad;
        d.tokens = r->tokens;
        d.width = r->width;
        d.grad_stride = r->grad_stride;
        d.token_bytes = r->token_bytes;
        d.num_tokens = (int32_t)r->num_tokens;
        d.num_rows = (int32_t)r->num_rows;
        d.slabs = (int32_t)slabs_of(r->width, WIDE);
        d.scale = scale;
        void* dp[] = {&d};
        return launch((const void*)direct_kernel_for(r->grad_dtype, vec), dim3((unsigned)(r->num_tokens * d.slabs)), ROWS_CTA, 0, 0, dp, stream);
    }
    int device = -1;
    int rc = sort_ready(device);
    if (rc != SOLO_OK) return rc;
    unsigned char* ws = (unsigned char*)workspace_dev;
    int bits = 1;
    while ((r->num_rows >> bits) != 0) ++bits;                 // the key num_rows stands for tokens outside
    for (int64_t at = 0; at < r->num_tokens; at += CHUNK) {
        const int n = (int)std::min<int64_t>(CHUNK, r->num_tokens - at);
        // Eight columns per lane, or four where they would not fill the GPU once (2048 tokens of 768 columns 14.3 and 12.2 us, 8192
        // 18.9 and 16.3; 16,384 of 4096 columns 72.8 and 76).
        const int64_t blocks = (n + CTA_ROWS - 1) / CTA_ROWS;
        const int rv = blocks * slabs_of(r->width, WIDE) < 4 * sm_count(device) ? NARROW : WIDE;
        const int64_t slabs = slabs_of(r->width, rv), row_ctas = blocks * slabs;
        SortArgs s;
        std::memset(&s, 0, sizeof(s));
        s.tokens = (const char*)r->tokens + at * r->token_bytes;
        s.token_bytes = r->token_bytes;
        s.num_tokens = n;
        s.num_rows = (int32_t)r->num_rows;
        s.passes = (bits + DIGIT_MAX - 1) / DIGIT_MAX;
        s.digit_bits = (bits + s.passes - 1) / s.passes;
        s.tok = (uint32_t*)(ws + l.tok);
        s.pos = (uint16_t*)(ws + l.pos);
        s.counters = (uint32_t*)(ws + l.counters);
        s.num_counters = (int32_t)row_ctas;
        int ctas = 1;
        while (ctas < SORT_CLUSTER && n > ctas * SORT_AIM) ctas *= 2;
        while ((ctas << s.log_per_cta) < n) ++s.log_per_cta;
        void* sp[] = {&s};
        if (rank_first(n, r->num_rows, r->width)) rc = launch((const void*)rows_rank_kernel, dim3((unsigned)((n + 31) / 32)), SORT_CTA, 0, 0, sp, stream);
        else rc = launch((const void*)sort_kernel_for((1 << s.log_per_cta) / SORT_CTA, s.digit_bits), dim3((unsigned)ctas), SORT_CTA, sizeof(SortShared), ctas, sp, stream);
        if (rc != SOLO_OK) return rc;
        RowsArgs a;
        std::memset(&a, 0, sizeof(a));
        a.acc = r->acc;
        a.grad = (const char*)r->grad + at * r->grad_stride * es;
        a.tok = s.tok;
        a.pos = s.pos;
        a.partial = (float*)(ws + l.partial);
        a.counters = s.counters;
        a.width = r->width;
        a.grad_stride = r->grad_stride;
        a.num_tokens = n;
        a.num_rows = s.num_rows;
        a.slabs = (int32_t)slabs;
        a.scale = scale;
        const double row_bytes = (double)r->width * es, all = n * row_bytes, acc_all = (double)n * (double)r->width * 4;
        a.ahead_ctas = (int32_t)std::min<int64_t>(row_ctas, (vec && rv == WIDE ? 4 : 3) * sm_count(device));
        a.ahead_rows = (int32_t)std::min<double>(n, AHEAD / row_bytes);
        if (all + acc_all <= AHEAD) {
            a.tokens = s.tokens;
            a.token_bytes = s.token_bytes;
        }
        void* rp[] = {&a};
        rc = launch((const void*)rows_kernel_for(r->grad_dtype, vec, rv), dim3((unsigned)row_ctas), ROWS_CTA, 0, 0, rp, stream);
        if (rc != SOLO_OK) return rc;
    }
    return SOLO_OK;
}

}  // extern "C"
