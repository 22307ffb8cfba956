// The gradient of an embedding, added to its fp32 accumulator: acc[tok_i, :] += s * g[i, :] (include/solo.h).
//
// Two launches for up to 65,536 tokens.  A cluster of up to eight CTAs sorts the tokens with their positions in its shared memory
// (least significant digit first, stable, so that equal tokens keep their order); then a CTA per run of equal tokens sums
// the run's rows in registers and adds the sum to the accumulator's row, which so is read and written once, without atomics and
// in an order that the tokens alone decide.  Long runs are cut at multiples of 64 in the sorted order; the pieces' sums go to
// the workspace, and the CTA that finishes last adds them up in their order.
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

constexpr int SORT_CTA = 1024;
constexpr int SORT_WARPS = SORT_CTA / 32;
constexpr int SORT_CLUSTER = 8;                        // most CTAs of the sort
constexpr int SORT_PER_CTA = 8192;                     // most tokens of one of them
constexpr int SORT_ROUNDS = SORT_PER_CTA / SORT_CTA;   // tokens per thread
constexpr int SORT_SMALL = 2048;                       // tokens per CTA that the cluster's size aims at
constexpr int CHUNK = SORT_CLUSTER * SORT_PER_CTA;     // tokens per pair of launches
constexpr int DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS;

constexpr int PIECE = 64, PIECE_BACK = 32;             // where long runs are cut, see cut_at
constexpr int ROWS_CTA = 256, ROWS_V = 8;              // threads and elements per thread of the summing kernel, at most

struct SortArgs {
    const void* tokens;
    int32_t token_bytes, num_tokens, per_cta, num_rows, digit_bits, passes;
    uint32_t* tok;              // [num_tokens] sorted; num_rows: outside the table
    uint16_t* pos;              // [num_tokens] position of each in the chunk
    uint32_t* counters;         // zeroed for the kernel after
    int32_t num_counters;
};

struct SortShared {
    uint32_t key[2][SORT_PER_CTA];
    uint16_t val[2][SORT_PER_CTA];
    uint16_t hist[SORT_WARPS][DIGITS];          // of each warp, then how many of a digit lie in the warps before
    uint32_t total[SORT_CLUSTER][DIGITS];       // of each CTA
    uint32_t base[DIGITS];                      // first place of a digit's tokens of this CTA
    uint32_t scan[SORT_WARPS];
};

__global__ __launch_bounds__(SORT_CTA) void rows_sort_kernel(const __grid_constant__ SortArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    SortShared& s = *reinterpret_cast<SortShared*>(smem);
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int me = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    pdl_wait();
    pdl_release();
    cluster.sync();                            // every CTA has started before its memory is written
    for (int i = me * SORT_CTA + tid; i < a.num_counters; i += ctas * SORT_CTA) a.counters[i] = 0;
    const int first = me * a.per_cta;
    const int count = min(max(a.num_tokens - first, 0), a.per_cta);
    for (int j = tid; j < count; j += SORT_CTA) {
        const int64_t t = a.token_bytes == 8 ? ((const int64_t*)a.tokens)[first + j] : (int64_t)((const int32_t*)a.tokens)[first + j];
        s.key[0][j] = t >= 0 && t < a.num_rows ? (uint32_t)t : (uint32_t)a.num_rows;
        s.val[0][j] = (uint16_t)(first + j);
    }
    const int digits = 1 << a.digit_bits;
    const int per_warp = (a.per_cta + SORT_CTA - 1) / SORT_CTA * 32;
    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * a.digit_bits, from = p & 1;
        for (int i = tid; i < SORT_WARPS * digits; i += SORT_CTA) s.hist[i / digits][i % digits] = 0;
        __syncthreads();
        // Place of every token among those of its digit in its warp.
        uint32_t key[SORT_ROUNDS], rank[SORT_ROUNDS];
        uint16_t val[SORT_ROUNDS];
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const int j = warp * per_warp + r * 32 + lane;
            const bool have = r * 32 < per_warp && j < count;
            key[r] = have ? s.key[from][j] : 0;
            val[r] = have ? s.val[from][j] : 0;
            const int d = have ? (int)((key[r] >> shift) & (uint32_t)(digits - 1)) : digits;
            const uint32_t peers = __match_any_sync(0xFFFFFFFFu, d);
            const uint32_t before = peers & ((1u << lane) - 1u);
            rank[r] = have ? s.hist[warp][d] + __popc(before) : 0xFFFFFFFFu;
            __syncwarp();
            if (have && before == 0) s.hist[warp][d] = (uint16_t)(s.hist[warp][d] + __popc(peers));
            __syncwarp();
        }
        __syncthreads();
        for (int d = tid; d < digits; d += SORT_CTA) {
            uint32_t sum = 0;
            for (int w = 0; w < SORT_WARPS; ++w) {
                const uint32_t h = s.hist[w][d];
                s.hist[w][d] = (uint16_t)sum;
                sum += h;
            }
            for (int r = 0; r < ctas; ++r) cluster.map_shared_rank(&s, r)->total[me][d] = sum;
        }
        cluster.sync();
        // Digits before this one in the whole cluster, then the CTAs before this one.
        uint32_t all = 0, mine = 0, upto = 0;
        if (tid < digits) {
            for (int r = 0; r < ctas; ++r) {
                if (r == me) mine = all;
                all += s.total[r][tid];
            }
            upto = all;
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) s.scan[warp] = upto;
        __syncthreads();
        if (tid < digits) {
            uint32_t b = upto - all + mine;
            for (int w = 0; w < warp; ++w) b += s.scan[w];
            s.base[tid] = b;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            if (rank[r] == 0xFFFFFFFFu) continue;
            const int d = (int)((key[r] >> shift) & (uint32_t)(digits - 1));
            const uint32_t to = s.base[d] + s.hist[warp][d] + rank[r];
            const uint32_t cta = to / (uint32_t)a.per_cta, j = to % (uint32_t)a.per_cta;
            SortShared* o = cluster.map_shared_rank(&s, cta);
            o->key[from ^ 1][j] = key[r];
            o->val[from ^ 1][j] = val[r];
        }
        cluster.sync();
    }
    const int last = a.passes & 1;
    for (int j = tid; j < count; j += SORT_CTA) {
        a.tok[first + j] = s.key[last][j];
        a.pos[first + j] = s.val[last][j];
    }
}

struct RowsArgs {
    float* acc;
    const void* grad;
    const uint32_t* tok;
    const uint16_t* pos;
    float* partial;             // [2 (num_tokens / PIECE + 1), width]: pieces that start at a multiple of PIECE, then runs' first pieces
    uint32_t* counters;         // [num_tokens / PIECE + 1, column groups] pieces done, at a run's first cut
    int64_t width, grad_stride;
    int32_t num_tokens, num_rows;
    float scale;
};

template <int DT> __device__ __forceinline__ float row_elem(const void* g, int64_t i) {
    if constexpr (DT == SOLO_DT_F32) return ((const float*)g)[i];
    else if constexpr (DT == SOLO_DT_BF16) return __uint_as_float((uint32_t)((const uint16_t*)g)[i] << 16);
    else return __half2float(((const __half*)g)[i]);
}

// Eight columns of a thread: consecutive ones and 16-byte accesses (VEC), or one in every `nt`.
template <int DT, bool VEC> struct Cols {
    int64_t c0, width;
    int nt;
    __device__ __forceinline__ int64_t at(int k) const { return VEC ? c0 + k : c0 + (int64_t)k * nt; }
    __device__ __forceinline__ bool in(int k) const { return VEC ? c0 < width : at(k) < width; }
    struct Raw { uint32_t w[VEC && DT != SOLO_DT_F32 ? 4 : 8]; };
    __device__ __forceinline__ Raw load(const void* g, int64_t row) const {
        Raw r;
        if constexpr (VEC) {
            constexpr int Q = DT == SOLO_DT_F32 ? 2 : 1;
            const uint4* p = reinterpret_cast<const uint4*>((const char*)g + (row + c0) * (DT == SOLO_DT_F32 ? 4 : 2));
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const uint4 v = c0 < width ? p[q] : make_uint4(0, 0, 0, 0);
                r.w[4 * q] = v.x; r.w[4 * q + 1] = v.y; r.w[4 * q + 2] = v.z; r.w[4 * q + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) r.w[k] = in(k) ? __float_as_uint(row_elem<DT>(g, row + at(k))) : 0u;
        }
        return r;
    }
    __device__ __forceinline__ static void add(const Raw& r, float (&s)[8]) {
        if constexpr (!VEC || DT == SOLO_DT_F32) {
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] += __uint_as_float(r.w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (DT == SOLO_DT_BF16) {
                    s[2 * k] += __uint_as_float(r.w[k] << 16);
                    s[2 * k + 1] += __uint_as_float(r.w[k] & 0xFFFF0000u);
                } else {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r.w[k]));
                    s[2 * k] += f.x;
                    s[2 * k + 1] += f.y;
                }
            }
        }
    }
    __device__ __forceinline__ void load_f32(const float* p, float (&v)[8]) const {
        if constexpr (VEC) {
            if (c0 < width) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float4 f = __ldcg(reinterpret_cast<const float4*>(p + c0) + q);
                    v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) if (in(k)) v[k] = __ldcg(p + at(k));
        }
    }
    __device__ __forceinline__ void store_f32(float* p, const float (&v)[8]) const {
        if constexpr (VEC) {
            if (c0 < width) {
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    reinterpret_cast<float4*>(p + c0)[q] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) if (in(k)) p[at(k)] = v[k];
        }
    }
};

// A run of one token is cut before entry e if e is a multiple of PIECE and the run began PIECE_BACK entries before or earlier:
// pieces are shorter than PIECE + PIECE_BACK, and runs of up to PIECE_BACK are never cut.
__device__ __forceinline__ bool cut_at(const uint32_t* tok, int e, uint32_t t) {
    return e % PIECE == 0 && e >= PIECE_BACK && tok[e - PIECE_BACK] == t;
}

// First entry with a token of at least t: 32 places at a time, the whole warp together.
__device__ __forceinline__ int lower_bound(const uint32_t* tok, int n, uint32_t t) {
    int lo = -1, hi = n;                       // tok[lo] < t <= tok[hi]
    const int lane = threadIdx.x & 31;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int probe = lo + (lane + 1) * step;
        const bool below = probe < hi && tok[probe] < t;
        lo += __popc(__ballot_sync(0xFFFFFFFFu, below)) * step;
        hi = min(hi, lo + step);
    }
    return hi;
}

template <int DT, bool VEC> __global__ __launch_bounds__(ROWS_CTA) void rows_sum_kernel(const __grid_constant__ RowsArgs a) {
    __shared__ bool s_last;
    pdl_wait();
    pdl_release();
    const int lane = threadIdx.x & 31, nt = blockDim.x;
    const int i = blockIdx.x, n = a.num_tokens;
    const uint32_t t = a.tok[i];
    if (t >= (uint32_t)a.num_rows) return;
    const bool run_start = i == 0 || a.tok[i - 1] != t;
    if (!run_start && !cut_at(a.tok, i, t)) return;
    int e = i + 1;
    bool run_end = false;
    for (;; e += 32) {
        const int x = e + lane;
        const bool other = x >= n || a.tok[x] != t;
        const uint32_t stop = __ballot_sync(0xFFFFFFFFu, other || cut_at(a.tok, x, t));
        if (stop) {
            const int k = __ffs(stop) - 1;
            run_end = (__ballot_sync(0xFFFFFFFFu, other) >> k) & 1u;
            e += k;
            break;
        }
    }
    Cols<DT, VEC> cols;
    cols.width = a.width;
    cols.nt = nt;
    cols.c0 = (int64_t)blockIdx.y * nt * ROWS_V + (VEC ? threadIdx.x * ROWS_V : threadIdx.x);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    int j = i;
    for (; j + 4 <= e; j += 4) {
        typename Cols<DT, VEC>::Raw r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = cols.load(a.grad, a.pos[j + k] * a.grad_stride);
#pragma unroll
        for (int k = 0; k < 4; ++k) cols.add(r[k], sum);
    }
    for (; j < e; ++j) cols.add(cols.load(a.grad, a.pos[j] * a.grad_stride), sum);
    float* const row = a.acc + (int64_t)t * a.width;
    if (!(run_start && run_end)) {
        const int begin = lower_bound(a.tok, n, t), end = lower_bound(a.tok, n, t + 1);
        const int cut = (begin + PIECE_BACK + PIECE - 1) / PIECE;              // the run's first cut, in pieces
        const int slots = n / PIECE + 1;
        const int pieces = 1 + (end - 1) / PIECE - cut + 1;
        cols.store_f32(a.partial + (int64_t)(run_start ? slots + cut : i / PIECE) * a.width, sum);
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) s_last = atomicAdd(&a.counters[(int64_t)cut * gridDim.y + blockIdx.y], 1u) == (uint32_t)(pieces - 1);
        __syncthreads();
        if (!s_last) return;
        __threadfence();
        double d[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        cols.load_f32(a.partial + (int64_t)(slots + cut) * a.width, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) d[k] = (double)v[k];
        for (int q = cut; q <= (end - 1) / PIECE; ++q) {
            cols.load_f32(a.partial + (int64_t)q * a.width, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) d[k] += (double)v[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = (float)d[k];
    }
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    cols.load_f32(row, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __fmaf_rn(a.scale, sum[k], v[k]);
    cols.store_f32(row, v);
}

using RowsKernel = void (*)(const RowsArgs);
RowsKernel rows_kernel_for(int dtype, bool vec) {
    switch (dtype) {
        case SOLO_DT_F32: return vec ? rows_sum_kernel<SOLO_DT_F32, true> : rows_sum_kernel<SOLO_DT_F32, false>;
        case SOLO_DT_BF16: return vec ? rows_sum_kernel<SOLO_DT_BF16, true> : rows_sum_kernel<SOLO_DT_BF16, false>;
        default: return vec ? rows_sum_kernel<SOLO_DT_F16, true> : rows_sum_kernel<SOLO_DT_F16, false>;
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

// The sort's shared memory, opted in to once per device.
int sort_ready() {
    static std::atomic<bool> done[64];
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) { cudaGetLastError(); return SOLO_ECUDA; }
    if (!done[device]) {
        if (cudaFuncSetAttribute((const void*)rows_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared)) !=
            cudaSuccess) {
            cudaGetLastError();
            return SOLO_ECUDA;
        }
        done[device] = true;
    }
    return SOLO_OK;
}

struct RowsLayout { size_t tok, pos, counters, partial, total; int64_t groups; int threads; };

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

RowsLayout rows_layout(int64_t num_tokens, int64_t width) {
    RowsLayout l;
    const int64_t n = std::min<int64_t>(num_tokens, CHUNK), cuts = n / PIECE + 1;
    l.threads = (int)std::min<int64_t>(ROWS_CTA, ((width + ROWS_V - 1) / ROWS_V + 31) / 32 * 32);
    l.groups = (width + (int64_t)l.threads * ROWS_V - 1) / ((int64_t)l.threads * ROWS_V);
    l.tok = 0;
    l.pos = l.tok + pad256((size_t)n * 4);
    l.counters = l.pos + pad256((size_t)n * 2);
    l.partial = l.counters + pad256((size_t)(cuts * l.groups) * 4);
    l.total = l.partial + pad256((size_t)(2 * cuts) * (size_t)width * 4);
    return l;
}

constexpr int64_t MOST_WIDTH = (int64_t)1 << 24, MOST_TOKENS = (int64_t)1 << 40;

}  // namespace
}  // namespace solo

using namespace solo;

extern "C" {

int solo_grad_rows_workspace(int64_t num_tokens, int64_t width, size_t* bytes) {
    if (!bytes || num_tokens < 0 || num_tokens > MOST_TOKENS || width < 1 || width > MOST_WIDTH) return SOLO_EINVAL;
    *bytes = rows_layout(num_tokens, width).total;
    return SOLO_OK;
}

int solo_grad_accumulate_rows(const solo_grad_rows_t* r, float scale, void* workspace_dev, void* stream_) {
    if (!r || !r->acc || r->num_rows < 1 || r->num_rows >= ((int64_t)1 << 31) || r->width < 1 || r->width > MOST_WIDTH) return SOLO_EINVAL;
    if (r->num_tokens < 0 || r->num_tokens > MOST_TOKENS || (r->token_bytes != 4 && r->token_bytes != 8)) return SOLO_EINVAL;
    if (r->grad_dtype < SOLO_DT_F32 || r->grad_dtype > SOLO_DT_F16 || r->grad_stride < 0 || !std::isfinite(scale)) return SOLO_EINVAL;
    if (r->num_tokens == 0) return SOLO_OK;
    if (!r->tokens || !r->grad || !workspace_dev) return SOLO_EINVAL;
    const int es = r->grad_dtype == SOLO_DT_F32 ? 4 : 2;
    if (((uintptr_t)workspace_dev & 15u) || ((uintptr_t)r->acc & 3u) || ((uintptr_t)r->tokens & (unsigned)(r->token_bytes - 1)) ||
        ((uintptr_t)r->grad & (unsigned)(es - 1)))
        return SOLO_EALIGN;
    int rc = sort_ready();
    if (rc != SOLO_OK) return rc;
    cudaStream_t stream = (cudaStream_t)stream_;
    const RowsLayout l = rows_layout(r->num_tokens, r->width);
    unsigned char* ws = (unsigned char*)workspace_dev;
    const bool vec = r->width % ROWS_V == 0 && (((uintptr_t)r->acc | (uintptr_t)r->grad) & 15u) == 0 && (r->grad_stride * es) % 16 == 0;
    int bits = 1;
    while ((r->num_rows >> bits) != 0) ++bits;                 // the key num_rows stands for tokens outside
    for (int64_t at = 0; at < r->num_tokens; at += CHUNK) {
        const int n = (int)std::min<int64_t>(CHUNK, r->num_tokens - at);
        SortArgs s;
        std::memset(&s, 0, sizeof(s));
        s.tokens = (const char*)r->tokens + at * r->token_bytes;
        s.token_bytes = r->token_bytes;
        s.num_tokens = n;
        s.num_rows = (int32_t)r->num_rows;
        s.passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
        s.digit_bits = (bits + s.passes - 1) / s.passes;
        s.tok = (uint32_t*)(ws + l.tok);
        s.pos = (uint16_t*)(ws + l.pos);
        s.counters = (uint32_t*)(ws + l.counters);
        s.num_counters = (int32_t)((n / PIECE + 1) * l.groups);
        int ctas = 1;
        while (ctas < SORT_CLUSTER && n > ctas * SORT_SMALL) ctas *= 2;
        s.per_cta = (n + ctas - 1) / ctas;
        void* sp[] = {&s};
        rc = launch((const void*)rows_sort_kernel, dim3((unsigned)ctas), SORT_CTA, sizeof(SortShared), ctas, sp, stream);
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
        a.scale = scale;
        void* rp[] = {&a};
        rc = launch((const void*)rows_kernel_for(r->grad_dtype, vec), dim3((unsigned)n, (unsigned)l.groups), (unsigned)l.threads, 0, 0, rp, stream);
        if (rc != SOLO_OK) return rc;
    }
    return SOLO_OK;
}

}  // extern "C"
