// Gradient lists before the step: global norm, clipping, accumulation over micro-batches (include/solo.h).
//
// All of these are streams over ragged lists of tensors, a read of 2 or 4 bytes per element and up to
// 8 bytes written and read besides, and one or two operations on it: bound by HBM.  One kernel template serves them.  The list
// is cut into tiles of 8192 elements of one tensor each.  The CTAs, as many as are resident, take the tiles in turn, so that all
// of them work on one stretch of memory (clip of the 125M-parameter set in place: 79 us, with a contiguous share each 89); where every tensor's
// norm is wanted a CTA takes a contiguous share instead, so that its sums need one partial for each tensor that it touches.
// What the next tile is gets looked up while the loads of the present one are under way.
//
// Sums.  A thread sums the (at most 32) powers that it takes from a tile in binary32 and adds that to a binary64 sum;
// threads, CTAs and tensors are summed in binary64 in a fixed order (no atomics), so results do not vary from call to call.
// A binary32 sum that overflowed, or is so small that squares may have been lost below 2^-149, is taken again in binary64
// from the values in memory.  Maxima are maxima of magnitude bit patterns, above all of which NaN lies.
#include "solo.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "solo_device.cuh"
#include "solo_host.h"

namespace solo {
namespace {

constexpr int GCTA = 256;                  // threads per CTA
constexpr int GV = 8;                      // elements per thread and vector: 16 bytes of bf16, 32 of fp32
constexpr int GU = 4;                      // vectors per thread and tile
constexpr int GTILE = GCTA * GV * GU;      // elements per tile
constexpr int GCTAS_PER_SM = 8;            // most CTAs per SM that a launch takes (bounds the workspace)
constexpr int GFINISH_MOST = 16;           // tensors whose norms the last CTA of a pass finishes too
constexpr int GIN_FLIGHT = 98304;          // bytes read and written of the tiles that a writing pass has under way per SM (pass())

enum { OP_NORM = 0, OP_CLIP = 1, OP_ACC = 2, OP_ACC_FIRST = 3 };

struct GradArgs {
    const void* const* src;      // gradients read
    void* const* dst;            // what is written: clipped gradients, accumulators
    const int64_t* numel;
    const int64_t* tile_start;   // [T + 1]
    int64_t tiles;
    int32_t num_tensors;
    int32_t norm_type;           // of the factor's norm (OP_CLIP)
    int32_t num_partials, num_norms;
    int32_t backwards;           // take the list from its end
    float scale, max_norm;
    double* cta_sum;             // [grid] what a CTA's share of the list sums to; null: no norm
    double* slots;               // [grid + T] partial of tensor t from CTA c at c + t: a CTA's last tensor is the next one's
                                 // first at the earliest, so no two partials share an index; null: no per-tensor norms
    const double* partials;      // OP_CLIP: cta_sum of the kernel before, or
    const float* norms;          // norms of the parts
    float* norm_out;             // null, or where the norm goes
    float* tensor_norm;          // the same for every tensor's (with a counter)
    uint32_t* counter;           // CTAs whose sums are written: the last one finishes the norms, and leaves 0; null: not here
    float norm_scale;            // factor of the norms
};

// ---- element types ------------------------------------------------------------------------------------------------

template <int DT> constexpr int DT_BYTES = DT == SOLO_DT_F32 ? 4 : 2;

__device__ __forceinline__ float elem_load(const void* p, int64_t i, std::integral_constant<int, SOLO_DT_F32>) { return ((const float*)p)[i]; }
__device__ __forceinline__ float elem_load(const void* p, int64_t i, std::integral_constant<int, SOLO_DT_BF16>) {
    return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
}
__device__ __forceinline__ float elem_load(const void* p, int64_t i, std::integral_constant<int, SOLO_DT_F16>) {
    return __half2float(((const __half*)p)[i]);
}
__device__ __forceinline__ void elem_store(void* p, int64_t i, float v, std::integral_constant<int, SOLO_DT_F32>) { ((float*)p)[i] = v; }
__device__ __forceinline__ void elem_store(void* p, int64_t i, float v, std::integral_constant<int, SOLO_DT_BF16>) {
    ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ void elem_store(void* p, int64_t i, float v, std::integral_constant<int, SOLO_DT_F16>) {
    ((__half*)p)[i] = __float2half_rn(v);
}

// Eight consecutive elements as they lie in memory.
template <int DT> struct Raw8 { uint4 q[DT_BYTES<DT> / 2]; };

// `wide`: fp32 in one access of 32 bytes (accumulation of 809M elements 1439 -> 1284 us against two of 16).
template <int DT> __device__ __forceinline__ Raw8<DT> load8(const char* p, bool wide) {
    const uint4* a = reinterpret_cast<const uint4*>(p);
    Raw8<DT> r;
    if constexpr (DT == SOLO_DT_F32) {
        if (wide) {
            asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=r"(r.q[0].x), "=r"(r.q[0].y), "=r"(r.q[0].z), "=r"(r.q[0].w), "=r"(r.q[1].x), "=r"(r.q[1].y), "=r"(r.q[1].z), "=r"(r.q[1].w)
                         : "l"(a) : "memory");
        } else {
            r.q[0] = a[0];
            r.q[1] = a[1];
        }
    } else {
        r.q[0] = a[0];
    }
    return r;
}

template <int DT> __device__ __forceinline__ void unpack8(const Raw8<DT>& r, float (&v)[8]) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
    if constexpr (DT == SOLO_DT_F32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[k]);
    } else if constexpr (DT == SOLO_DT_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
            v[2 * k] = f.x;
            v[2 * k + 1] = f.y;
        }
    }
}

template <int DT> __device__ __forceinline__ void store8(char* p, const float (&v)[8], bool wide) {
    uint4* a = reinterpret_cast<uint4*>(p);
    Raw8<DT> r;
    uint32_t* w = reinterpret_cast<uint32_t*>(&r);
    if constexpr (DT == SOLO_DT_F32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(v[k]);
    } else if constexpr (DT == SOLO_DT_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&b);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __half2 b = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&b);
        }
    }
    if constexpr (DT == SOLO_DT_F32) {
        if (wide) {
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" :: "l"(a), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                         : "memory");
        } else {
            a[0] = r.q[0];
            a[1] = r.q[1];
        }
    } else {
        a[0] = r.q[0];
    }
}

// ---- sums ---------------------------------------------------------------------------------------------------------

__device__ __forceinline__ double max_nan(double a, double b) { return (b > a || b != b) ? b : a; }
template <int NT> __device__ __forceinline__ double join(double a, double b) { return NT == SOLO_NORM_MAX ? max_nan(a, b) : a + b; }
__device__ __forceinline__ double join(int nt, double a, double b) { return nt == SOLO_NORM_MAX ? max_nan(a, b) : a + b; }

// A thread's sum of powers (p = 1, 2: binary64) or its largest magnitude (as a bit pattern).
template <int NT> struct Sum {
    double s = 0.0;
    uint32_t m = 0;
    float c[2] = {0.0f, 0.0f};   // powers of up to 32 values
    __device__ __forceinline__ void add(const float (&v)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if constexpr (NT == SOLO_NORM_MAX) m = max(m, __float_as_uint(v[k]) & 0x7FFFFFFFu);
            else if constexpr (NT == SOLO_NORM_1) c[k & 1] = c[k & 1] + fabsf(v[k]);
            else c[k & 1] = __fmaf_rn(v[k], v[k], c[k & 1]);
        }
    }
    // Into the binary64 sum; again(u, v) gives the u-th eight of the values added since the last call.
    template <int N, class Again> __device__ __forceinline__ void settle(Again again) {
        if constexpr (NT == SOLO_NORM_MAX) return;
        const float f = c[0] + c[1];
        c[0] = c[1] = 0.0f;
        // Above 2^-100, what 32 squares lost below 2^-149 is less than 2^-44 of the sum.
        if (f < __int_as_float(0x7F800000) && (NT == SOLO_NORM_1 || f >= 0x1p-100f)) {
            s += (double)f;
            return;
        }
#pragma unroll 1
        for (int u = 0; u < N; ++u) {
            float v[8];
            again(u, v);
            uint32_t any = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) any |= __float_as_uint(v[k]);
            if ((any & 0x7FFFFFFFu) == 0) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k) s = NT == SOLO_NORM_1 ? s + (double)fabsf(v[k]) : __fma_rn((double)v[k], (double)v[k], s);
        }
    }
    __device__ __forceinline__ double value() const { return NT == SOLO_NORM_MAX ? (double)__uint_as_float(m) : s; }
    __device__ __forceinline__ void clear() { s = 0.0; m = 0; }
};

// Sum over the CTA, in every thread.  `box`: one double per warp, free again after the next barrier but one.
__device__ __forceinline__ double cta_join(int nt, double v, double* box) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = join(nt, v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    if ((threadIdx.x & 31) == 0) box[threadIdx.x >> 5] = v;
    __syncthreads();
    double r = box[0];
#pragma unroll
    for (int w = 1; w < GCTA / 32; ++w) r = join(nt, r, box[w]);
    return r;
}

__device__ __forceinline__ double root(int nt, double s) { return nt == SOLO_NORM_2 ? sqrt(s) : s; }

// N of a clip (every CTA computes it for itself, in the same order: a few partials per thread, from L2), and its factor.
__device__ __forceinline__ float clip_factor(const GradArgs& a, double* box, double* norm) {
    double s = 0.0;
    for (int i = threadIdx.x; i < a.num_partials; i += GCTA) s = join(a.norm_type, s, a.partials[i]);
    for (int i = threadIdx.x; i < a.num_norms; i += GCTA) {
        const double v = fabs((double)a.norms[i]);
        s = join(a.norm_type, s, a.norm_type == SOLO_NORM_2 ? v * v : v);
    }
    s = root(a.norm_type, cta_join(a.norm_type, s, box));
    if (a.num_partials) s *= fabs((double)a.scale);
    *norm = s;
    double c = 1.0;
    if (a.num_partials + a.num_norms) {
        c = (double)a.max_norm / (s + 1e-6);
        if (c > 1.0) c = 1.0;                    // a NaN stays
    }
    return (float)((double)a.scale * c);
}

// Largest t with tile_start[t] <= x: 32 places at a time, the whole warp together.
__device__ __forceinline__ int find_tensor(const int64_t* tile_start, int num_tensors, int64_t x) {
    int lo = 0, hi = num_tensors;
    const int lane = threadIdx.x & 31;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int probe = lo + (lane + 1) * step;
        const bool below = probe < hi && tile_start[probe] <= x;
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, below));     // starts do not decrease: the lanes below are the first ones
        lo += n * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// The tensor that a tile belongs to, and the tile.
template <int DS, int DD, bool WRITES> struct Place {
    int t;
    int64_t t0, t1;              // the tensor's tiles
    int64_t n;
    const char* s;
    char* d;
    int head;                    // elements before the first place where vectors of both sides are aligned
    bool vec, wide;

    __device__ __forceinline__ void tensor(const GradArgs& a, int which) {
        t = which;
        t0 = a.tile_start[t];
        t1 = a.tile_start[t + 1];
        n = a.numel[t];
        s = (const char*)a.src[t];
        d = WRITES ? (char*)a.dst[t] : nullptr;
        const uintptr_t sa = (uintptr_t)s, da = (uintptr_t)d;
        // eight elements of the narrower type take 16 bytes; eight of fp32 on a 16-byte boundary two accesses
        constexpr bool BY_DST = WRITES && DT_BYTES<DD> < DT_BYTES<DS>;
        head = BY_DST ? (int)(8 - (da / DT_BYTES<DD>) % 8) % 8 : (int)(8 - (sa / DT_BYTES<DS>) % 8) % 8;
        const uintptr_t sh = sa + head * DT_BYTES<DS>, dh = WRITES ? da + head * DT_BYTES<DD> : 0;
        vec = ((sh | dh) & 15) == 0;
        wide = (((DS == SOLO_DT_F32 ? sh : 0) | (DD == SOLO_DT_F32 ? dh : 0)) & 31) == 0;
        if (!vec) head = 0;
    }
    __device__ __forceinline__ void start(const GradArgs& a, int64_t x) { tensor(a, find_tensor(a.tile_start, a.num_tensors, x)); }
    // To tile x, after or before: the tensors next to the present one, 32 at a time.
    __device__ __forceinline__ void move(const GradArgs& a, int64_t x) {
        if (x >= t0 && x < t1) return;
        const int lane = threadIdx.x & 31;
        int u = t;
        for (;;) {
            int steps;
            if (x >= t1) {
                const int probe = u + 1 + lane;
                steps = __popc(__ballot_sync(0xFFFFFFFFu, probe < a.num_tensors && a.tile_start[probe] <= x));
                u += steps;
            } else {
                const int probe = u - lane;
                steps = __popc(__ballot_sync(0xFFFFFFFFu, probe >= 0 && a.tile_start[probe] > x));
                u -= steps;
            }
            if (steps < 32) break;
        }
        tensor(a, u);
    }
};

// Norms from the CTAs' sums, which other CTAs may just have written.
struct FinishArgs {
    const double* cta_sum;
    const double* slots;
    const int64_t* tile_start;
    int64_t tiles;
    int32_t grid, num_tensors, norm_type;
    float scale;
    float* norm_out;
    float* tensor_norm;
};

__device__ __forceinline__ void finish_total(const FinishArgs& a, double* box) {
    double s = 0.0;
    for (int i = threadIdx.x; i < a.grid; i += GCTA) s = join(a.norm_type, s, __ldcg(a.cta_sum + i));
    s = cta_join(a.norm_type, s, box);
    if (threadIdx.x == 0) *a.norm_out = (float)(fabs((double)a.scale) * root(a.norm_type, s));
}
// by a warp
__device__ __forceinline__ void finish_tensor(const FinishArgs& a, int t) {
    const int lane = threadIdx.x & 31;
    const int64_t t0 = a.tile_start[t], t1 = a.tile_start[t + 1];
    double s = 0.0;
    if (t0 < t1) {
        // tile x lies in the share of CTA ((x + 1) grid - 1) / tiles
        const int64_t c0 = ((t0 + 1) * a.grid - 1) / a.tiles, c1 = (t1 * a.grid - 1) / a.tiles;
        for (int64_t c = c0 + lane; c <= c1; c += 32) s = join(a.norm_type, s, __ldcg(a.slots + c + t));
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s = join(a.norm_type, s, __shfl_xor_sync(0xFFFFFFFFu, s, d));
    if (lane == 0) a.tensor_norm[t] = (float)(fabs((double)a.scale) * root(a.norm_type, s));
}

// ---- the kernel -----------------------------------------------------------------------------------------------------

// DS: type read (gradients); DD: type written; NT: norm type or -1.
template <int OP, int DS, int DD, int NT> __global__ __launch_bounds__(GCTA, OP == OP_ACC || DS == SOLO_DT_F32 ? (OP == OP_NORM ? 4 : 2) : OP == OP_NORM ? 5 : 3) void grad_kernel(const __grid_constant__ GradArgs a) {
    using S = std::integral_constant<int, DS>;
    using D = std::integral_constant<int, DD>;
    constexpr bool WRITES = OP != OP_NORM;
    constexpr bool SUMS = NT >= 0;
    __shared__ double box[2][GCTA / 32];
    int turn = 0;
    pdl_wait();
    pdl_release();
    const int64_t grid = gridDim.x, c = blockIdx.x;
    const bool shares = SUMS && a.slots;
    int64_t x = shares ? a.tiles * c / grid : c;                       // of the tiles in the order taken
    const int64_t end = shares ? a.tiles * (c + 1) / grid : a.tiles, step = shares ? 1 : grid;
    const auto tile = [&](int64_t i) { return a.backwards ? a.tiles - 1 - i : i; };
    float f = a.scale;
    bool have_f = OP != OP_CLIP;
    Sum<NT> sum;
    double share = 0.0;
    Place<DS, DD, WRITES> at;
    if (x < end) at.start(a, tile(x));
    while (x < end) {
        if (OP == OP_CLIP && DS == DD && have_f && f == 1.0f && (const char*)at.d == at.s) {        // in place, by one: nothing changes
            if ((const void*)a.src == (const void*)a.dst) break;                // in none of the tensors
            x += step;
            if (x < end) at.move(a, tile(x));
            continue;
        }
        const int64_t off = tile(x) - at.t0, base = at.head + off * GTILE;
        const bool full = at.vec && base + GTILE <= at.n;
        const int64_t first = off == 0 ? 0 : base;
        const int rest = (int)(full ? base - first : max(min(at.n, base + GTILE) - first, (int64_t)0));   // elements taken one by one
        const char* const s = at.s + first * DT_BYTES<DS>;
        char* const d = at.d + first * DT_BYTES<DD>;
        const char* const sv = at.s + (base + (int)threadIdx.x * GV) * DT_BYTES<DS>;
        char* const dv = at.d + (base + (int)threadIdx.x * GV) * DT_BYTES<DD>;
        const bool wide = at.wide, same = WRITES && (const char*)at.d == at.s;
        const int t = at.t;
        Raw8<DS> g[GU];
        [[maybe_unused]] Raw8<SOLO_DT_F32> acc[OP == OP_ACC ? GU : 1];
        if (full) {
#pragma unroll
            for (int u = 0; u < GU; ++u) {
                g[u] = load8<DS>(sv + u * GCTA * GV * DT_BYTES<DS>, wide);
                if constexpr (OP == OP_ACC) acc[u] = load8<SOLO_DT_F32>(dv + u * GCTA * GV * 4, wide);
            }
        }
        if constexpr (OP == OP_CLIP) {
            if (!have_f) {
                double norm;
                f = clip_factor(a, box[0], &norm);
                have_f = true;
                if (a.norm_out && c == 0 && threadIdx.x == 0) *a.norm_out = (float)norm;
            }
        }
        // (a pass that only reads has other CTAs' loads under way meanwhile, and no registers to spare for a second place)
        if constexpr (WRITES) {
            x += step;
            if (x < end) at.move(a, tile(x));
        }
        if (OP == OP_CLIP && DS == DD && f == 1.0f && same) continue;           // (the tile that was loaded before the factor was known)
        if (full) {
#pragma unroll
            for (int u = 0; u < GU; ++u) {
                float w[GV];
                unpack8<DS>(g[u], w);
                if constexpr (OP == OP_ACC) {
                    float b[GV];
                    unpack8<SOLO_DT_F32>(acc[u], b);
#pragma unroll
                    for (int k = 0; k < GV; ++k) w[k] = __fmaf_rn(f, w[k], b[k]);
                } else if constexpr (WRITES) {
#pragma unroll
                    for (int k = 0; k < GV; ++k) w[k] = f * w[k];
                }
                if constexpr (WRITES) store8<DD>(dv + u * GCTA * GV * DT_BYTES<DD>, w, wide);
                if constexpr (SUMS) sum.add(w);
            }
            if constexpr (SUMS)
                sum.template settle<GU>([&](int u, float (&w)[GV]) {             // from memory again: what was read, or written
                    if constexpr (WRITES) unpack8<DD>(load8<DD>(dv + u * GCTA * GV * DT_BYTES<DD>, wide), w);
                    else unpack8<DS>(load8<DS>(sv + u * GCTA * GV * DT_BYTES<DS>, wide), w);
                });
        }
        for (int i0 = threadIdx.x; i0 < rest; i0 += GCTA * 8) {
            float w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = i0 + k * GCTA;
                w[k] = i < rest ? elem_load(s, i, S{}) : 0.0f;
                if constexpr (OP == OP_ACC) w[k] = i < rest ? __fmaf_rn(f, w[k], elem_load(d, i, D{})) : 0.0f;
                else if constexpr (WRITES) w[k] = f * w[k];
            }
            if constexpr (WRITES) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int i = i0 + k * GCTA;
                    if (i < rest) elem_store(d, i, w[k], D{});
                }
            }
            if constexpr (SUMS) {
                sum.add(w);
                sum.template settle<1>([&](int, float (&v)[8]) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = w[k];
                });
            }
        }
        if constexpr (!WRITES) {
            x += step;
            if (x < end) at.move(a, tile(x));
        }
        if constexpr (SUMS) {
            if (shares && (x >= end || at.t != t)) {
                const double r = cta_join(NT, sum.value(), box[turn]);
                turn ^= 1;
                if (threadIdx.x == 0) a.slots[c + t] = r;
                share = join<NT>(share, r);
                sum.clear();
            }
        }
    }
    if constexpr (SUMS) {
        if (!shares) share = cta_join(NT, sum.value(), box[turn]);
        if (threadIdx.x == 0) a.cta_sum[c] = share;
        if (a.counter) {
            __shared__ bool last;
            if (threadIdx.x == 0) {                                             // (it wrote the slots too)
                __threadfence();
                last = atomicAdd(a.counter, 1u) == (uint32_t)grid - 1u;
            }
            __syncthreads();
            if (last) {
                __threadfence();
                const FinishArgs fin = {a.cta_sum, a.slots, a.tile_start, a.tiles, (int32_t)grid, a.num_tensors, NT, a.norm_scale, a.norm_out, a.tensor_norm};
                if (a.slots)
                    for (int t = threadIdx.x >> 5; t < a.num_tensors; t += GCTA / 32) finish_tensor(fin, t);
                finish_total(fin, box[turn ^ 1]);
                if (threadIdx.x == 0) *a.counter = 0;
            }
        }
    }
    if constexpr (OP == OP_CLIP) {
        if (!have_f && a.norm_out) {                                            // a list without elements
            double norm;
            clip_factor(a, box[0], &norm);
            if (threadIdx.x == 0) *a.norm_out = (float)norm;
        }
    }
}

// Where the last CTA of the pass does not: the total in CTA 0 (where norm_out is given), a tensor per warp in the others.
__global__ __launch_bounds__(GCTA) void grad_finish_kernel(const __grid_constant__ FinishArgs a) {
    __shared__ double box[GCTA / 32];
    pdl_wait();
    pdl_release();
    if (blockIdx.x == 0) {
        if (a.norm_out) finish_total(a, box);
        return;
    }
    const int t = (blockIdx.x - 1) * (GCTA / 32) + (threadIdx.x >> 5);
    if (t < a.num_tensors) finish_tensor(a, t);
}

// ---- instances --------------------------------------------------------------------------------------------------------

using GradKernel = void (*)(const GradArgs);

template <int OP, int DS, int DD> GradKernel by_norm(int nt) {
    if constexpr (OP == OP_CLIP) return grad_kernel<OP, DS, DD, -1>;
    else switch (nt) {
        case SOLO_NORM_MAX: return grad_kernel<OP, DS, DD, SOLO_NORM_MAX>;
        case SOLO_NORM_1: return grad_kernel<OP, DS, DD, SOLO_NORM_1>;
        case SOLO_NORM_2: return grad_kernel<OP, DS, DD, SOLO_NORM_2>;
        default:
            if constexpr (OP == OP_NORM) return nullptr;
            else return grad_kernel<OP, DS, DD, -1>;
    }
}
template <int OP, int DS> GradKernel by_dst(int dd, int nt) {
    if constexpr (OP != OP_CLIP) return by_norm<OP, DS, SOLO_DT_F32>(nt);
    else switch (dd) {
        case SOLO_DT_F32: return by_norm<OP, DS, SOLO_DT_F32>(nt);
        case SOLO_DT_BF16: return by_norm<OP, DS, SOLO_DT_BF16>(nt);
        default: return by_norm<OP, DS, SOLO_DT_F16>(nt);
    }
}
template <int OP> GradKernel by_src(int ds, int dd, int nt) {
    switch (ds) {
        case SOLO_DT_F32: return by_dst<OP, SOLO_DT_F32>(dd, nt);
        case SOLO_DT_BF16: return by_dst<OP, SOLO_DT_BF16>(dd, nt);
        default: return by_dst<OP, SOLO_DT_F16>(dd, nt);
    }
}
GradKernel grad_kernel_for(int op, int ds, int dd, int nt) {
    switch (op) {
        case OP_NORM: return by_src<OP_NORM>(ds, dd, nt);
        case OP_CLIP: return by_src<OP_CLIP>(ds, dd, nt);
        case OP_ACC: return by_src<OP_ACC>(ds, dd, nt);
        default: return by_src<OP_ACC_FIRST>(ds, dd, nt);
    }
}

// Resident CTAs per SM of grad_kernel_for's kernel, at most GCTAS_PER_SM; 0 on error.  Remembered in place: a map would allocate, and
// what that throws would leave through the C calls.
int grad_occupancy(GradKernel k, int op, int ds, int dd, int nt, int device) {
    static std::atomic<int8_t> seen[64][4][3][3][4];
    std::atomic<int8_t>* const at = device >= 0 && device < 64 ? &seen[device][op][ds][dd][nt + 1] : nullptr;
    int n = at ? at->load(std::memory_order_relaxed) : 0;
    if (n > 0) return n;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, (const void*)k, GCTA, 0) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    n = std::min(n, GCTAS_PER_SM);
    if (at) at->store((int8_t)n, std::memory_order_relaxed);
    return n;
}

int launch(const void* k, unsigned grid, void** params, cudaStream_t stream) {
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;    // see pdl_wait
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(GCTA);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelExC(&cfg, k, params) != cudaSuccess) {
        cudaGetLastError();
        return SOLO_ECUDA;
    }
    count_launch();
    return SOLO_OK;
}

}  // namespace
}  // namespace solo

struct solo_grads {
    int device = 0;
    int num_tensors = 0;
    int64_t tiles = 0;
    std::vector<int64_t> numel;
    const int64_t* geom = nullptr;  // device, the caller's: numel[T] | tile_start[T + 1]
};

namespace {

using namespace solo;

bool valid_dtype(int d) { return d >= SOLO_DT_F32 && d <= SOLO_DT_F16; }
bool valid_norm(int n) { return n >= SOLO_NORM_MAX && n <= SOLO_NORM_2; }

int check_list(const solo_grad_list_t* l) {
    if (!l || !l->grads || !l->data || !valid_dtype(l->dtype)) return SOLO_EINVAL;
    if ((uintptr_t)l->data & 7u) return SOLO_EALIGN;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return SOLO_ECUDA; }
    return dev == l->grads->device ? SOLO_OK : SOLO_ESTATE;
}

int check_pair(const solo_grad_list_t* a, const solo_grad_list_t* b) {
    int rc = check_list(a);
    if (rc == SOLO_OK) rc = check_list(b);
    if (rc != SOLO_OK) return rc;
    return a->grads == b->grads || a->grads->numel == b->grads->numel ? SOLO_OK : SOLO_ESTATE;
}

int check_norm(int norm_type, const float* norm_dev, const float* tensor_norm_dev, const void* workspace) {
    if (!valid_norm(norm_type) || !norm_dev || !workspace) return SOLO_EINVAL;
    return (((uintptr_t)norm_dev | (uintptr_t)tensor_norm_dev) & 3u) || ((uintptr_t)workspace & 15u) ? SOLO_EALIGN : SOLO_OK;
}

// One pass over the list; *grid_out: CTAs launched (what the partials are of).
int pass(int op, const solo_grad_list_t* src, const solo_grad_list_t* dst, int norm_type, GradArgs a, cudaStream_t stream,
         int* grid_out = nullptr) {
    const solo_grads* g = src->grads;
    const int dd = dst ? dst->dtype : 0;
    const GradKernel k = grad_kernel_for(op, src->dtype, dd, norm_type);
    if (!k) return SOLO_EINVAL;
    const int per_sm = grad_occupancy(k, op, src->dtype, dd, norm_type, g->device);
    if (per_sm <= 0) return SOLO_ECUDA;
    a.src = (const void* const*)src->data;
    a.dst = dst ? dst->data : nullptr;
    a.numel = g->geom;
    a.tile_start = g->geom + g->num_tensors;
    a.tiles = g->tiles;
    a.num_tensors = g->num_tensors;
    // Passes that write run best with no more under way than it takes.  GIN_FLIGHT makes that three CTAs per SM from 16-bit to 16-bit types and two
    // for all else.  GB/s with two and three, 202M elements: bf16 in place 5680 and 6280, into another list 5910 and 5890; bf16 into fp32 6110
    // and 5660; accumulation of 809M bf16 1235 us with two, 1290 with three to six.  A pass that only reads takes all that fit (7B bf16: 1903 us
    // with four, 1813 with five).
    int most = per_sm;
    if (op != OP_NORM) {
        const int written = dst->dtype == SOLO_DT_F32 ? 4 : 2, read = (src->dtype == SOLO_DT_F32 ? 4 : 2) + (op == OP_ACC ? 4 : 0);
        most = std::min(per_sm, std::max(2, GIN_FLIGHT / (GTILE * (read + written))));
    }
    const int64_t grid = std::max<int64_t>(1, std::min<int64_t>(g->tiles, (int64_t)sm_count(g->device) * most));
    if (grid_out) *grid_out = (int)grid;
    void* params[] = {&a};
    return launch((const void*)k, (unsigned)grid, params, stream);
}

int finish(const solo_grads* g, const GradArgs& a, int grid, int norm_type, float scale, float* norm_dev, float* tensor_norm_dev,
           cudaStream_t stream) {
    FinishArgs f;
    std::memset(&f, 0, sizeof(f));
    f.cta_sum = a.cta_sum;
    f.slots = a.slots;
    f.tile_start = g->geom + g->num_tensors;
    f.tiles = g->tiles;
    f.grid = grid;
    f.num_tensors = g->num_tensors;
    f.norm_type = norm_type;
    f.scale = scale;
    f.norm_out = norm_dev;
    f.tensor_norm = tensor_norm_dev;
    void* params[] = {&f};
    const unsigned blocks = 1u + (tensor_norm_dev ? (unsigned)((g->num_tensors + GCTA / 32 - 1) / (GCTA / 32)) : 0u);
    return launch((const void*)grad_finish_kernel, blocks, params, stream);
}

size_t most_ctas(const solo_grads* g) { return (size_t)sm_count(g->device) * GCTAS_PER_SM; }

// Workspace: counter (16 bytes, zero between calls) | cta_sum | slots.  The last CTA of the pass finishes the total and a few tensors'
// norms, which saves a launch (2 us of the host's 8.5 for a norm); with more tensors a second launch does, with a warp for each, and
// so it does where the calls are captured: the host's time does not count there, and 1 Mi elements take 3.1 us instead of 3.9.
GradArgs norm_args(const solo_grads* g, void* workspace, float scale, float* norm_dev, float* tensor_norm_dev, cudaStream_t stream) {
    GradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.cta_sum = (double*)workspace + 2;
    a.slots = tensor_norm_dev ? a.cta_sum + most_ctas(g) : nullptr;
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusActive;
    if (cudaStreamIsCapturing(stream, &cap) != cudaSuccess) cudaGetLastError();
    if (cap == cudaStreamCaptureStatusNone && (!tensor_norm_dev || g->num_tensors <= GFINISH_MOST)) {
        a.counter = (uint32_t*)workspace;
        a.norm_out = norm_dev;
        a.tensor_norm = tensor_norm_dev;
        a.norm_scale = scale;
    }
    return a;
}

}  // namespace

extern "C" {

int solo_grads_create(const int64_t* numel_host, int num_tensors, int64_t* geom_dev, void* stream_, solo_grads_t** out) {
    if (!out) return SOLO_EINVAL;
    *out = nullptr;
    if (!numel_host || !geom_dev || num_tensors < 1) return SOLO_EINVAL;
    if ((uintptr_t)geom_dev & 7u) return SOLO_EALIGN;
    int64_t tiles = 0;
    for (int t = 0; t < num_tensors; ++t) {
        if (numel_host[t] < 0 || numel_host[t] > ((int64_t)1 << 48)) return SOLO_EINVAL;
        tiles += (numel_host[t] + GTILE - 1) / GTILE;
        if (tiles > ((int64_t)1 << 40)) return SOLO_EINVAL;             // share arithmetic: tiles * CTAs in 64 bits
    }
    cudaStream_t stream = (cudaStream_t)stream_;
    int device = -1;
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;          // the copy below is from this call's memory
    if (cudaGetDevice(&device) != cudaSuccess || cudaStreamIsCapturing(stream, &cap) != cudaSuccess) { cudaGetLastError(); return SOLO_ECUDA; }
    if (cap != cudaStreamCaptureStatusNone) return SOLO_EINVAL;
    solo_grads* g = nullptr;
    try {
        g = new solo_grads();
        g->numel.assign(numel_host, numel_host + num_tensors);
        std::vector<int64_t> geom(g->numel);
        geom.reserve(2 * (size_t)num_tensors + 1);
        int64_t at = 0;
        for (int t = 0; t < num_tensors; ++t) {
            geom.push_back(at);
            at += (numel_host[t] + GTILE - 1) / GTILE;
        }
        geom.push_back(at);
        if (cudaMemcpyAsync(geom_dev, geom.data(), geom.size() * 8, cudaMemcpyHostToDevice, stream) != cudaSuccess) {
            cudaGetLastError();
            delete g;
            return SOLO_ECUDA;
        }
    } catch (const std::bad_alloc&) {
        delete g;
        return SOLO_ENOMEM;
    }
    g->device = device;
    g->num_tensors = num_tensors;
    g->tiles = tiles;
    g->geom = geom_dev;
    *out = g;
    return SOLO_OK;
}

int solo_grads_destroy(solo_grads_t* g) {
    delete g;
    return SOLO_OK;
}

int solo_grads_workspace(const solo_grads_t* g, size_t* bytes) {
    if (!g || !bytes) return SOLO_EINVAL;
    *bytes = (2 + 2 * most_ctas(g) + (size_t)g->num_tensors) * sizeof(double);
    return SOLO_OK;
}

int solo_grad_norm(const solo_grad_list_t* list, int norm_type, float scale, float* norm_dev, float* tensor_norm_dev,
                   void* workspace_dev, void* stream) {
    int rc = check_norm(norm_type, norm_dev, tensor_norm_dev, workspace_dev);
    if (rc == SOLO_OK) rc = check_list(list);
    if (rc != SOLO_OK) return rc;
    if (!std::isfinite(scale)) return SOLO_EINVAL;
    const GradArgs a = norm_args(list->grads, workspace_dev, scale, norm_dev, tensor_norm_dev, (cudaStream_t)stream);
    int grid = 0;
    rc = pass(OP_NORM, list, nullptr, norm_type, a, (cudaStream_t)stream, &grid);
    if (rc != SOLO_OK || a.counter) return rc;
    return finish(list->grads, a, grid, norm_type, scale, norm_dev, tensor_norm_dev, (cudaStream_t)stream);
}

int solo_grad_clip(const solo_grad_list_t* src, const solo_grad_list_t* dst, const float* norms_dev, int num_norms, int norm_type,
                   float max_norm, float scale, void* stream) {
    if (num_norms < 0 || (num_norms && !norms_dev) || !valid_norm(norm_type)) return SOLO_EINVAL;
    if (!std::isfinite(scale) || (num_norms && !(std::isfinite(max_norm) && max_norm >= 0.0f))) return SOLO_EINVAL;
    if (num_norms && ((uintptr_t)norms_dev & 3u)) return SOLO_EALIGN;
    const int rc = check_pair(src, dst);
    if (rc != SOLO_OK) return rc;
    GradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.norms = norms_dev;
    a.num_norms = num_norms;
    a.norm_type = norm_type;
    a.max_norm = max_norm;
    a.scale = scale;
    return pass(OP_CLIP, src, dst, -1, a, (cudaStream_t)stream);
}

int solo_grad_clip_norm(const solo_grad_list_t* src, const solo_grad_list_t* dst, int norm_type, float max_norm, float scale,
                        float* norm_dev, float* tensor_norm_dev, void* workspace_dev, void* stream) {
    int rc = check_norm(norm_type, norm_dev, tensor_norm_dev, workspace_dev);
    if (rc == SOLO_OK) rc = check_pair(src, dst);
    if (rc != SOLO_OK) return rc;
    if (!std::isfinite(scale) || !std::isfinite(max_norm) || !(max_norm >= 0.0f)) return SOLO_EINVAL;
    // the clip finishes the total itself, from the sums, and so needs the workspace for itself until it has run
    GradArgs n = norm_args(src->grads, workspace_dev, scale, nullptr, tensor_norm_dev, (cudaStream_t)stream);
    n.counter = nullptr;
    int grid = 0;
    rc = pass(OP_NORM, src, nullptr, norm_type, n, (cudaStream_t)stream, &grid);
    if (rc != SOLO_OK) return rc;
    if (tensor_norm_dev) {
        rc = finish(src->grads, n, grid, norm_type, scale, nullptr, tensor_norm_dev, (cudaStream_t)stream);
        if (rc != SOLO_OK) return rc;
    }
    GradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.partials = n.cta_sum;
    a.num_partials = grid;
    a.norm_type = norm_type;
    a.max_norm = max_norm;
    a.scale = scale;
    a.norm_out = norm_dev;
    a.backwards = 1;             // what the first pass read last is still in L2
    return pass(OP_CLIP, src, dst, -1, a, (cudaStream_t)stream);
}

int solo_grad_accumulate(const solo_grad_list_t* acc, const solo_grad_list_t* grad, float scale, int first, int norm_type,
                         float* norm_dev, float* tensor_norm_dev, void* workspace_dev, void* stream) {
    int rc = norm_type == -1 ? SOLO_OK : check_norm(norm_type, norm_dev, tensor_norm_dev, workspace_dev);
    if (rc == SOLO_OK) rc = check_pair(acc, grad);
    if (rc != SOLO_OK) return rc;
    if (acc->dtype != SOLO_DT_F32 || !std::isfinite(scale)) return SOLO_EINVAL;
    GradArgs a;
    std::memset(&a, 0, sizeof(a));
    if (norm_type != -1) a = norm_args(acc->grads, workspace_dev, 1.0f, norm_dev, tensor_norm_dev, (cudaStream_t)stream);
    a.scale = scale;
    int grid = 0;
    rc = pass(first ? OP_ACC_FIRST : OP_ACC, grad, acc, norm_type, a, (cudaStream_t)stream, &grid);
    if (rc != SOLO_OK || norm_type == -1 || a.counter) return rc;
    return finish(acc->grads, a, grid, norm_type, 1.0f, norm_dev, tensor_norm_dev, (cudaStream_t)stream);
}

}  // extern "C"
