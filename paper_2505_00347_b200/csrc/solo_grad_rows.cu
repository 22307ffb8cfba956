// The gradient of an embedding, added to its fp32 accumulator: acc[tok_i, :] += s * g[i, :] (include/solo.h).
//
// Two launches for up to 65,536 tokens.  A cluster of up to eight CTAs sorts the tokens with their positions in its shared memory
// (least significant digit first, stable, so that equal tokens keep their order); then every warp takes a window of the sorted
// order and 256 columns, sums the rows of each run of equal tokens in registers and adds the sum to the accumulator's row, which so
// is read and written once, without atomics and in an order that the tokens alone decide.  A window holds about the same number of rows
// whatever the tokens are, so that frequent ones cost no more than rare ones.  Long runs are cut at window starts; the
// pieces' sums go to the workspace, and the warp that finishes last adds them up in their order.
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
constexpr int DIGIT_MIN = 5, DIGIT_MAX = 9, DIGITS = 1 << DIGIT_MAX;

constexpr int WINDOW = 32, WINDOW_BACK = 16;           // entries of a warp; where runs are cut, see rows_sum_kernel
constexpr int ROWS_CTA = 256, SLAB = 256;              // threads of the summing kernel; columns of a warp

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
    uint16_t hist[SORT_WARPS * DIGITS];         // [warp][digit] of each warp, then how many of a digit lie in the warps before
    uint32_t part[SORT_CTA];                    // [group of warps][digit]
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
    cluster.barrier_arrive();                   // every CTA has started before its memory is written
    const int per_cta = 1 << a.log_per_cta;
    const int first = me * per_cta;
    const int count = min(max(a.num_tokens - first, 0), per_cta);
    for (int j = tid; j < count; j += SORT_CTA) {
        const int64_t t = a.token_bytes == 8 ? ((const int64_t*)a.tokens)[first + j] : (int64_t)((const int32_t*)a.tokens)[first + j];
        s.item[0][j] = make_uint2(t >= 0 && t < a.num_rows ? (uint32_t)t : (uint32_t)a.num_rows, (uint32_t)(first + j));
    }
    for (int i = me * SORT_CTA + tid; i < a.num_counters; i += ctas * SORT_CTA) a.counters[i] = 0;
    const int digits = 1 << a.digit_bits;
    const int rounds = (per_cta + SORT_CTA - 1) / SORT_CTA;
    uint16_t* const hist = s.hist + warp * digits;
    // for the sums over warps: threads of a group of warps (one for each digit), and the warps of a group
    const int group = tid >> a.digit_bits, digit = tid & (digits - 1), group_warps = digits / 32;
    cluster.barrier_wait();
    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * a.digit_bits, from = p & 1;
        for (int i = lane; i < digits / 2; i += 32) reinterpret_cast<uint32_t*>(hist)[i] = 0;
        __syncthreads();                        // (the tokens)
        // Place of every token among those of its digit in its warp.
        uint2 item[SORT_ROUNDS];
        uint32_t rank[SORT_ROUNDS];
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            if (r < rounds) {
                const int j = (warp * rounds + r) * 32 + lane;
                const bool have = j < count;
                item[r] = have ? s.item[from][j] : make_uint2(0, 0);
                const int d = have ? (int)((item[r].x >> shift) & (uint32_t)(digits - 1)) : digits;
                const uint32_t peers = __match_any_sync(0xFFFFFFFFu, d);
                const uint32_t before = peers & ((1u << lane) - 1u);
                rank[r] = have ? hist[d] + __popc(before) : 0xFFFFFFFFu;
                __syncwarp();
                if (have && before == 0) hist[d] = (uint16_t)(hist[d] + __popc(peers));
                __syncwarp();
            }
        }
        __syncthreads();
        uint32_t sum = 0;
        for (int w = group * group_warps; w < (group + 1) * group_warps; ++w) {
            const uint32_t h = s.hist[w * digits + digit];
            s.hist[w * digits + digit] = (uint16_t)sum;
            sum += h;
        }
        s.part[tid] = sum;
        __syncthreads();
        uint32_t before_group = 0, total = 0;
        for (int g = 0; g < SORT_CTA >> a.digit_bits; ++g) {
            const uint32_t v = s.part[(g << a.digit_bits) + digit];
            if (g < group) before_group += v;
            total += v;
        }
        if (group == 0)
            for (int r = 0; r < ctas; ++r) cluster.map_shared_rank(&s, r)->total[me][digit] = total;
        for (int w = group * group_warps; w < (group + 1) * group_warps; ++w)
            s.hist[w * digits + digit] = (uint16_t)(s.hist[w * digits + digit] + before_group);
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
            if (r < rounds && rank[r] != 0xFFFFFFFFu) {
                const int d = (int)((item[r].x >> shift) & (uint32_t)(digits - 1));
                const uint32_t to = s.base[d] + hist[d] + rank[r];
                cluster.map_shared_rank(&s, to >> a.log_per_cta)->item[from ^ 1][to & (uint32_t)(per_cta - 1)] = item[r];
            }
        }
        cluster.sync();
    }
    const int last = a.passes & 1;
    for (int j = tid; j < count; j += SORT_CTA) {
        const uint2 v = s.item[last][j];
        a.tok[first + j] = v.x;
        a.pos[first + j] = (uint16_t)v.y;
    }
}

struct RowsArgs {
    float* acc;
    const void* grad;
    const uint32_t* tok;
    const uint16_t* pos;
    float* partial;             // [2 windows, width]: pieces that start with a window, then runs' first pieces, at the first cut
    uint32_t* counters;         // [windows, slabs] pieces done, at a run's first cut
    int64_t width, grad_stride;
    int32_t num_tokens, num_rows, slabs;
    float scale;
};

template <int DT> __device__ __forceinline__ float row_elem(const void* g, int64_t i) {
    if constexpr (DT == SOLO_DT_F32) return ((const float*)g)[i];
    else if constexpr (DT == SOLO_DT_BF16) return __uint_as_float((uint32_t)((const uint16_t*)g)[i] << 16);
    else return __half2float(((const __half*)g)[i]);
}

// Eight columns of a thread: consecutive ones and 16-byte accesses (VEC), or one in every 32.
template <int DT, bool VEC> struct Cols {
    int64_t c0, width;
    __device__ __forceinline__ int64_t at(int k) const { return VEC ? c0 + k : c0 + k * 32; }
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

// First and last + 1 entry of token t: half a warp each, sixteen places at a time.
__device__ __forceinline__ void run_bounds(const uint32_t* tok, int n, uint32_t t, int& begin, int& end) {
    const int lane = threadIdx.x & 31, half = lane >> 4, place = lane & 15;
    int lo = -1, hi = n;                       // tok[lo] < target <= tok[hi]
    while (__any_sync(0xFFFFFFFFu, hi - lo > 1)) {
        const int step = (hi - lo + 15) / 16;
        const int probe = lo + (place + 1) * step;
        const bool below = probe < hi && tok[probe] < t + half;
        const uint32_t b = __ballot_sync(0xFFFFFFFFu, below);
        lo += __popc(half ? b >> 16 : b & 0xFFFFu) * step;
        hi = min(hi, lo + step);
    }
    begin = __shfl_sync(0xFFFFFFFFu, hi, 0);
    end = __shfl_sync(0xFFFFFFFFu, hi, 16);
}

// A warp sums the runs that start in its window, and a run that was cut at its start, over its 256 columns.  A run is cut
// at a window's start if it began WINDOW_BACK entries before or earlier, so that short runs are never cut and a warp
// reaches into the next window, but not beyond.
template <int DT, bool VEC> __global__ __launch_bounds__(ROWS_CTA) void rows_sum_kernel(const __grid_constant__ RowsArgs a) {
    constexpr uint32_t ALL = 0xFFFFFFFFu, NONE = 0xFFFFFFFFu;
    pdl_wait();
    pdl_release();
    const int lane = threadIdx.x & 31;
    const int n = a.num_tokens, windows = (n + WINDOW - 1) / WINDOW;
    const int64_t task = (int64_t)blockIdx.x * (ROWS_CTA / 32) + (threadIdx.x >> 5);
    const int w = (int)(task / a.slabs), slab = (int)(task % a.slabs);
    if (w >= windows) return;
    const int base = w * WINDOW, next = base + WINDOW;
    const uint32_t t0 = base + lane < n ? a.tok[base + lane] : NONE;
    const uint32_t t1 = next + lane < n ? a.tok[next + lane] : NONE;
    const int p0 = base + lane < n ? a.pos[base + lane] : 0;
    const int p1 = next + lane < n ? a.pos[next + lane] : 0;
    const uint32_t before = base > 0 ? a.tok[base - 1] : NONE;
    const uint32_t back = base > 0 ? a.tok[base - WINDOW_BACK] : NONE;
    const uint32_t beyond = next + WINDOW < n ? a.tok[next + WINDOW] : NONE;
    uint32_t prev = __shfl_up_sync(ALL, t0, 1);
    if (lane == 0) prev = before;
    const uint32_t rows = (uint32_t)a.num_rows;
    const uint32_t firsts = __ballot_sync(ALL, t0 != prev && t0 < rows);                  // entries that begin a run
    const bool cut0 = t0 == back;                                                         // (lane 0's is used)
    const uint32_t starts = firsts | (__ballot_sync(ALL, lane == 0 && cut0 && t0 < rows));
    if (starts == 0) return;
    const int inside = __popc(__ballot_sync(ALL, t0 < rows));                            // tokens outside come last
    int total = inside;
    bool last_cut = false;
    if (inside == WINDOW) {
        const uint32_t t = __shfl_sync(ALL, t0, WINDOW - 1);
        if (__shfl_sync(ALL, t1, 0) == t) {
            last_cut = __shfl_sync(ALL, t0, WINDOW - WINDOW_BACK) == t;
            if (!last_cut) {
                const uint32_t same = __ballot_sync(ALL, t1 == t);
                total += same == ALL ? WINDOW : __ffs(~same) - 1;
                last_cut = same == ALL && beyond == t;
            }
        }
    }
    const bool first_cut = (firsts & 1u) == 0 && (starts & 1u);                           // the first piece continues a run
    Cols<DT, VEC> cols;
    cols.width = a.width;
    cols.c0 = (int64_t)slab * SLAB + (VEC ? lane * 8 : lane);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    constexpr int BATCH = 4;
    const int begin = __ffs(starts) - 1;
    int piece = begin;                                                                    // first entry of the piece summed
    for (int k = begin; k < total; k += BATCH) {
        typename Cols<DT, VEC>::Raw r[BATCH];
        float v[BATCH][8];
        bool ends[BATCH];
        float* row[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int x = k + b;
            const int pa = __shfl_sync(ALL, p0, x & 31), pb = __shfl_sync(ALL, p1, x & 31);
            const uint32_t t = __shfl_sync(ALL, t0, min(x, WINDOW - 1));
            ends[b] = x == total - 1 || (x < WINDOW - 1 && (starts >> (x + 1)) & 1u);
            row[b] = a.acc + (int64_t)t * a.width;
            if (x < total) {
                r[b] = cols.load(a.grad, (x < WINDOW ? pa : pb) * a.grad_stride);
                if (ends[b]) cols.load_f32(row[b], v[b]);
            }
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int x = k + b;
            if (x < total) {
                cols.add(r[b], sum);
                if (ends[b]) {
                    if ((first_cut && piece == 0) || (last_cut && x == total - 1)) {
                        // a run's first piece lies at its first cut: the next window's start, or the one after if it is the last one's end
                        const int slot = first_cut && piece == 0 ? w : windows + w + (total > WINDOW ? 2 : 1);
                        cols.store_f32(a.partial + (int64_t)slot * a.width, sum);
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q) v[b][q] = __fmaf_rn(a.scale, sum[q], v[b][q]);
                        cols.store_f32(row[b], v[b]);
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q) sum[q] = 0.0f;
                    piece = x + 1;
                }
            }
        }
    }
    if (!first_cut && !last_cut) return;
    __threadfence();
    __syncwarp();
    // Of a run that is cut on both sides of this window there is one piece here.
    const bool one = first_cut && last_cut && (starts & (starts - 1)) == 0;
    for (int side = 0; side < 2; ++side) {
        if (side == 0 ? !first_cut : !last_cut || one) continue;
        const uint32_t t = __shfl_sync(ALL, t0, side == 0 ? 0 : WINDOW - 1);
        int from, to;
        run_bounds(a.tok, n, t, from, to);
        const int cut = (from + WINDOW_BACK + WINDOW - 1) / WINDOW;                       // window of the run's first cut
        const int last = (to - 1) / WINDOW;                                               // window of its last entry
        uint32_t done = 0;
        if (lane == 0) done = atomicAdd(&a.counters[(int64_t)cut * a.slabs + slab], 1u);
        if (__shfl_sync(ALL, done, 0) != (uint32_t)(last - cut + 1)) continue;            // the first piece and one for each window
        __threadfence();
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        double d[8];
        cols.load_f32(a.partial + (int64_t)(windows + cut) * a.width, v);
#pragma unroll
        for (int q = 0; q < 8; ++q) d[q] = (double)v[q];
#pragma unroll 4
        for (int p = cut; p <= last; ++p) {
            cols.load_f32(a.partial + (int64_t)p * a.width, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) d[q] += (double)v[q];
        }
        float* const row = a.acc + (int64_t)t * a.width;
        cols.load_f32(row, v);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = __fmaf_rn(a.scale, (float)d[q], v[q]);
        cols.store_f32(row, v);
    }
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

struct RowsLayout { size_t tok, pos, counters, partial, total; int64_t slabs; };

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

RowsLayout rows_layout(int64_t num_tokens, int64_t width) {
    RowsLayout l;
    const int64_t n = std::min<int64_t>(num_tokens, CHUNK), windows = (n + WINDOW - 1) / WINDOW;
    l.slabs = (width + SLAB - 1) / SLAB;
    l.tok = 0;
    l.pos = l.tok + pad256((size_t)n * 4);
    l.counters = l.pos + pad256((size_t)n * 2);
    l.partial = l.counters + pad256((size_t)(windows * l.slabs) * 4);
    l.total = l.partial + pad256((size_t)(2 * windows) * (size_t)width * 4);
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
    const bool vec = r->width % 8 == 0 && (((uintptr_t)r->acc | (uintptr_t)r->grad) & 15u) == 0 && (r->grad_stride * es) % 16 == 0;
    int bits = 1;
    while ((r->num_rows >> bits) != 0) ++bits;                 // the key num_rows stands for tokens outside
    for (int64_t at = 0; at < r->num_tokens; at += CHUNK) {
        const int n = (int)std::min<int64_t>(CHUNK, r->num_tokens - at), windows = (n + WINDOW - 1) / WINDOW;
        SortArgs s;
        std::memset(&s, 0, sizeof(s));
        s.tokens = (const char*)r->tokens + at * r->token_bytes;
        s.token_bytes = r->token_bytes;
        s.num_tokens = n;
        s.num_rows = (int32_t)r->num_rows;
        s.passes = (bits + DIGIT_MAX - 1) / DIGIT_MAX;
        s.digit_bits = std::max(DIGIT_MIN, (bits + s.passes - 1) / s.passes);
        s.tok = (uint32_t*)(ws + l.tok);
        s.pos = (uint16_t*)(ws + l.pos);
        s.counters = (uint32_t*)(ws + l.counters);
        s.num_counters = (int32_t)(windows * l.slabs);
        int ctas = 1;
        while (ctas < SORT_CLUSTER && n > ctas * SORT_SMALL) ctas *= 2;
        while ((ctas << s.log_per_cta) < n) ++s.log_per_cta;
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
        a.slabs = (int32_t)l.slabs;
        a.scale = scale;
        void* rp[] = {&a};
        const int64_t warps = windows * l.slabs;
        rc = launch((const void*)rows_kernel_for(r->grad_dtype, vec), dim3((unsigned)((warps + ROWS_CTA / 32 - 1) / (ROWS_CTA / 32))), ROWS_CTA, 0, 0,
                    rp, stream);
        if (rc != SOLO_OK) return rc;
    }
    return SOLO_OK;
}

}  // extern "C"
