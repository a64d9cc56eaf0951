// The global norm of a list of gradients, and their clipping.
//
//   norm  = sqrt(sum over all tensors of x^2)
//   scale = norm > max_norm ? max_norm / norm : 1          (1 where the norm is not finite)
//
// Two launches whatever the number of tensors: their addresses travel in the kernel's parameters, 1024 at a time.  The first pass
// leaves a sum per CTA; every CTA of the second adds these up for itself, in one order, so nothing depends on the order
// of execution, nor on the tensors' addresses, and there is no counter to reset.  Squares are taken in fp32 and summed over 64 or 32 entries of a thread, the
// sums in double precision; a sum next to the ends of fp32's range is taken again in double precision, so no gradient is too
// large or too small.
// Both passes are bound by HBM: 1294 MB of bf16 gradients take 183 us for the norm (7.0 TB/s) and 415 us to be scaled into other tensors (6.2 TB/s), one
// after the other 620; the second pass starts at the end, where the first left the last of them in L2.  Where nothing is to be clipped in place it ends at once (126 million
// parameters, 253 MB: 41 us, 0.94 of the copy rate).  Three CTAs per SM, as many as run at a time, with eight granules a thread on the way: four
// (64 registers) 687 us for both passes, six with four granules 682, against 617.  At three the scaling kernel spills 32 bytes.
#pragma once
#include <cfloat>

#include "common.cuh"

namespace picospec {

constexpr int GRAD_FEW = 64, GRAD_MANY = 1024;      // tensors of a launch: two sizes of its parameters
constexpr int GRAD_AHEAD = 8;                       // granules of 16 bytes that a thread has on the way
constexpr int GRAD_TILE = GRAD_AHEAD * THREADS;     // granules of a tile
constexpr int GRAD_CTAS = 3;                        // CTAs per SM, all of them at a time
constexpr int GRAD_PARTS = 2048;                    // most CTAs of a launch: sums that it leaves
constexpr long long GRAD_BF16 = 1ll << 62;          // of a count: the tensor is bf16

template <int CAP> struct GradArgs {
    const void* in[CAP];
    void* out[CAP];
    long long count[CAP];       // entries, and GRAD_BF16
    unsigned tile0[CAP + 1];    // first tile of each tensor; the last: their number
    int n;
    double* parts;              // the first pass: its CTAs' sums
    int all_parts;              // the second: how many there are,
    float max_norm;             //             the limit,
    const float* norm_in;       //             the norm, where the caller has it,
    float* norm_out;            //             where it goes (or null),
    bool inplace;               //             whether every tensor is its own result
};

// A tensor as granules of 16 bytes on 16-byte boundaries, to be scaled; the first and the last may be cut short.
struct GradSpan {
    long long start, count, units;
    int per;
    __host__ __device__ GradSpan(const void* p, long long n, bool bf16) : count(n), per(bf16 ? 8 : 4) {
        const int lead = (int)((16 - ((uintptr_t)p & 15)) & 15) / (bf16 ? 2 : 4);
        start = lead ? lead - per : 0;
        units = n > 0 ? (n - start + per - 1) / per : 0;
    }
};

template <int CAP> __device__ __forceinline__ int grad_tensor(const GradArgs<CAP>& a, unsigned tile) {
    int lo = 0, hi = a.n;               // tile0[lo] <= tile < tile0[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.tile0[mid] <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

// the entries of a granule
__device__ __forceinline__ float grad_value(const uint32_t (&w)[4], int e, bool bf16) {
    if (!bf16) return __uint_as_float(w[e]);
    return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
}
__device__ __forceinline__ uint4 grad_load(const void* p) {
    uint4 r;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}

// Sum of a double per thread over the CTA, the same in every thread; `part`: WARPS doubles.
__device__ __forceinline__ double grad_block_sum(double x, double* part) {
    x = warp_sum(x);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) sum += part[w];
    __syncthreads();
    return sum;
}

// Granules of a tensor's own entries, whatever its address: unit u is the N entries from u N on, the last filled up with zeros.
__host__ __device__ __forceinline__ long long grad_units(long long n, bool bf16) { return (n + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4); }

// The granule `at` of memory behind `base` (on a 16-byte boundary), zero where it is not among the bytes [from, to) of the tensor
template <bool BF16> __device__ __forceinline__ uint4 grad_granule(const char* base, long long at, int from, long long to) {
    const long long b = at * 16;
    if (b >= from && b + 16 <= to) return grad_load(base + b);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (b < to) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!BF16) {
                if (b + 4 * j >= from && b + 4 * j < to) w[j] = *reinterpret_cast<const volatile uint32_t*>(base + b + 4 * j);
                continue;
            }
            if (b + 4 * j >= from && b + 4 * j < to) w[j] = *reinterpret_cast<const volatile unsigned short*>(base + b + 4 * j);
            if (b + 4 * j + 2 >= from && b + 4 * j + 2 < to) w[j] |= (uint32_t)*reinterpret_cast<const volatile unsigned short*>(base + b + 4 * j + 2) << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The 16 bytes from byte `lead` (even) of two granules on
__device__ __forceinline__ uint4 grad_shifted(const uint4& lo, const uint4& hi, int lead) {
    uint32_t c[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if (lead & 8)
#pragma unroll
        for (int i = 0; i < 6; ++i) c[i] = c[i + 2];
    if (lead & 4)
#pragma unroll
        for (int i = 0; i < 5; ++i) c[i] = c[i + 1];
    const int bits = (lead & 3) * 8;
    return make_uint4(__funnelshift_r(c[0], c[1], bits), __funnelshift_r(c[1], c[2], bits), __funnelshift_r(c[2], c[3], bits), __funnelshift_r(c[3], c[4], bits));
}

// A thread's units, and so the order of the sums, do not depend on the address: a tensor off the 16-byte boundaries is read in granules on them,
// and each unit put together from its thread's and the next thread's (600 MB of bf16 102 us, on the boundaries 88); `edge`: those that cross a warp,
// and the one behind the tile.  With consecutive units a warp instead of a CTA the second pass finds less of them in L2 (647 million entries: 630 us
// for both passes, against 617).
template <bool BF16> __device__ __forceinline__ double grad_tile_squares(const void* p, long long count, long long u0, int tid, uint4 (&edge)[GRAD_AHEAD * WARPS + 1]) {
    constexpr int N = BF16 ? 8 : 4;
    const int lane = tid & 31, lead = (int)((uintptr_t)p & 15);
    const char* base = reinterpret_cast<const char*>(p) - lead;
    const long long to = lead + count * (BF16 ? 2 : 4);
    uint4 x[GRAD_AHEAD];
    double sum = 0.0;
    if ((lead == 0 || u0 > 0) && (u0 + GRAD_TILE) * 16 <= to) {         // (all of them whole)
#pragma unroll
        for (int k = 0; k < GRAD_AHEAD; ++k) x[k] = grad_load(base + (u0 + tid + k * THREADS) * 16);
    } else {
#pragma unroll
        for (int k = 0; k < GRAD_AHEAD; ++k) x[k] = grad_granule<BF16>(base, u0 + tid + k * THREADS, lead, to);
    }
    if (lead) {
        __syncthreads();                        // (the tile before is done with)
        if (tid == 0) edge[GRAD_AHEAD * WARPS] = grad_granule<BF16>(base, u0 + GRAD_TILE, lead, to);
#pragma unroll
        for (int k = 0; k < GRAD_AHEAD; ++k)
            if (lane == 0) edge[k * WARPS + (tid >> 5)] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < GRAD_AHEAD; ++k) {
            uint4 y = make_uint4(__shfl_down_sync(0xffffffffu, x[k].x, 1), __shfl_down_sync(0xffffffffu, x[k].y, 1),
                                 __shfl_down_sync(0xffffffffu, x[k].z, 1), __shfl_down_sync(0xffffffffu, x[k].w, 1));
            if (lane == 31) y = edge[k * WARPS + (tid >> 5) + 1];
            x[k] = grad_shifted(x[k], y, lead);
        }
    }
    float s = 0.0f;
    uint32_t any = 0u;
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
        float part = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float v = grad_value(w, j, BF16);
            part = fmaf(v, v, part);
        }
        s += part;
        any |= w[0] | w[1] | w[2] | w[3];
    }
    // in the middle of fp32's range nothing that counts was lost (64 terms below 2^-126 against 1e-24) or ran over
    if (s > 1e-24f && s < 1e36f) return sum + (double)s;
    if ((any & (BF16 ? 0x7FFF7FFFu : 0x7FFFFFFFu)) == 0u) return sum;
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
        for (int j = 0; j < N; ++j) {
            const double v = (double)grad_value(w, j, BF16);
            sum += v * v;
        }
    }
    return sum;
}

template <int CAP> __global__ void __launch_bounds__(THREADS, GRAD_CTAS) grad_squares_kernel(const __grid_constant__ GradArgs<CAP> a) {
    __shared__ double part[WARPS];
    __shared__ uint4 edge[GRAD_AHEAD * WARPS + 1];
    grid_dependency_sync();
    const unsigned tiles = a.tile0[a.n];
    double sum = 0.0;
    for (unsigned t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int i = grad_tensor(a, t);
        const bool bf16 = a.count[i] & GRAD_BF16;
        const long long count = a.count[i] & ~GRAD_BF16, u0 = (long long)(t - a.tile0[i]) * GRAD_TILE;
        sum += bf16 ? grad_tile_squares<true>(a.in[i], count, u0, threadIdx.x, edge) : grad_tile_squares<false>(a.in[i], count, u0, threadIdx.x, edge);
    }
    sum = grad_block_sum(sum, part);
    if (threadIdx.x == 0) a.parts[blockIdx.x] = sum;
}

// x * scale, rounded to the tensor's type; a scale that is no normal fp32 number is taken in double precision
__device__ __forceinline__ float grad_scaled(float x, float scale, double exact) { return scale >= 1e-30f ? x * scale : (float)((double)x * exact); }

template <bool BF16> __device__ __forceinline__ void grad_tile_scale(const void* in, void* out, const GradSpan& g, long long u0, int tid, float scale, double exact) {
    constexpr int N = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4;
    const bool level = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
    const char* src = reinterpret_cast<const char*>(in);
    char* dst = reinterpret_cast<char*>(out);
    uint4 x[GRAD_AHEAD];
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k) {
        const long long e = g.start + (u0 + tid + k * THREADS) * N;
        if (level && e >= 0 && e + N <= g.count) x[k] = grad_load(src + e * SIZE);
    }
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k) {
        const long long e = g.start + (u0 + tid + k * THREADS) * N;
        if (level && e >= 0 && e + N <= g.count) {
            uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (BF16) {
                    const float lo = grad_scaled(grad_value(w, 2 * j, true), scale, exact), hi = grad_scaled(grad_value(w, 2 * j + 1, true), scale, exact);
                    const __nv_bfloat162 y = __floats2bfloat162_rn(lo, hi);
                    w[j] = *reinterpret_cast<const uint32_t*>(&y);
                } else w[j] = __float_as_uint(grad_scaled(__uint_as_float(w[j]), scale, exact));
            }
            asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(dst + e * SIZE), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
        } else {
            for (int j = 0; j < N; ++j) {
                if (e + j < 0 || e + j >= g.count) continue;
                if (BF16) {
                    const float v = __uint_as_float((uint32_t)*reinterpret_cast<const volatile unsigned short*>(src + (e + j) * 2) << 16);
                    *reinterpret_cast<__nv_bfloat16*>(dst + (e + j) * 2) = __float2bfloat16_rn(grad_scaled(v, scale, exact));
                } else *reinterpret_cast<float*>(dst + (e + j) * 4) = grad_scaled(*reinterpret_cast<const volatile float*>(src + (e + j) * 4), scale, exact);
            }
        }
    }
}

template <int CAP> __global__ void __launch_bounds__(THREADS, GRAD_CTAS) grad_scale_kernel(const __grid_constant__ GradArgs<CAP> a) {
    __shared__ double part[WARPS];
    grid_dependency_sync();
    const int tid = threadIdx.x;
    double norm;
    if (a.norm_in) norm = (double)*a.norm_in;
    else {
        double sum = 0.0;
        for (int i = tid; i < a.all_parts; i += THREADS) sum += a.parts[i];
        norm = sqrt(grad_block_sum(sum, part));
    }
    // the norm as it is returned, so that a call that is handed it scales by the same bits; the sum's own where fp32 has no normal number for it
    const float rounded = (float)norm;
    if (a.norm_out && blockIdx.x == 0 && tid == 0) *a.norm_out = rounded;
    if (rounded >= FLT_MIN && rounded <= FLT_MAX) norm = (double)rounded;
    const double exact = norm > (double)a.max_norm && norm < CUDART_INF ? (double)a.max_norm / norm : 1.0;
    if (a.inplace && exact == 1.0) return;
    const float scale = (float)exact;
    const unsigned tiles = a.tile0[a.n];
    // from the end: the first pass left the last tiles in L2
    for (unsigned k = blockIdx.x; k < tiles; k += gridDim.x) {
        const unsigned t = tiles - 1 - k;
        const int i = grad_tensor(a, t);
        if (exact == 1.0 && a.in[i] == a.out[i]) continue;
        const bool bf16 = a.count[i] & GRAD_BF16;
        const GradSpan g(a.in[i], a.count[i] & ~GRAD_BF16, bf16);
        const long long u0 = (long long)(t - a.tile0[i]) * GRAD_TILE;
        if (bf16) grad_tile_scale<true>(a.in[i], a.out[i], g, u0, tid, scale, exact);
        else grad_tile_scale<false>(a.in[i], a.out[i], g, u0, tid, scale, exact);
    }
}

}  // namespace picospec
