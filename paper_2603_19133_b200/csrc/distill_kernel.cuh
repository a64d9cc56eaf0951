// Distillation from a teacher's top entries: the loss of every row and, in the same pass, its gradient.
//
//   s = softmax(l / T);   entries (x_j, t_j), j < n;   A = sum t;   r = max(0, 1 - A) with the tail, else 0;
//   R = sum of s outside the entries
//   loss  = sum_j t_j (ln t_j - ln s(x_j)) + r (ln r - ln R)
//   dl/dl_v = 1/T ((A + r) s_v - t_v)         on the entries
//           = 1/T ((A + r) R - r) s_v / R     elsewhere
//
// s_v / R is the softmax over the entries' complement, so the complement is summed by itself, relative to its own
// maximum: R = 1 - sum over the entries would be lost where the entries hold nearly everything, and so would the gradient
// outside them.  A bit per entry of the slice takes the teacher's entries out of the streaming sum (and finds indices
// that come twice); what concerns the entries is done one by one in double precision.
#pragma once
#include "resident_row.cuh"

namespace picospec {

struct DistillArgs {
    const void* logits;
    long long row_stride;
    int R, V, K;
    const float* temperature;   // [B]
    const int* t_idx;           // [B, R, K]
    const float* t_prob;        // [B, R, K]
    const int* t_count;         // [B, R]
    const float* weight;        // [B, R] or null (1)
    int tail;
    float* loss;                // [B, R] or null
    void* grad;                 // [B, R, V] of the logits' type, or null
    long long grad_stride;
    unsigned* status;
    unsigned long long wait_limit_ns;
    int slice_chunks;
};

// What one warp knows of its part of the row; sums of exponentials are of exp((l - max) / T).
struct __align__(16) DistillRecord {
    double entry_sum;                            // over its entries
    double t, t_log_t, t_x;                      // over its entries: sums of t, t ln t, t (l - entry_max) / T
    float rest_max, rest_sum;                    // outside the entries; the sum up to stream_scale()
    float entry_max;
    unsigned status;
};
constexpr int DISTILL_RECORDS = MAX_CLUSTER * WARPS;

constexpr int DISTILL_ENTRIES = MAX_K / THREADS;        // teacher entries per thread

// Exclude the entries whose bit is set: their weight is zero.
__device__ __forceinline__ void exclude(ChunkRegs<__nv_bfloat16>& r, uint32_t bits) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        if (bits >> (2 * k) & 1u) r.w[k] = (r.w[k] & 0xFFFF0000u) | 0xFF80u;
        if (bits >> (2 * k + 1) & 1u) r.w[k] = (r.w[k] & 0xFFFFu) | 0xFF800000u;
    }
}
__device__ __forceinline__ void exclude(ChunkRegs<float>& r, uint32_t bits) {
#pragma unroll
    for (int k = 0; k < 32; ++k)
        if (bits >> k & 1u) r.f[k] = -CUDART_INF_F;
}
// The bit of virtual entry i of a slice: the word belongs to the lane that holds the entry (ChunkRegs::offset), so a lane
// finds its 32 entries' bits in one word.
template <typename T> __device__ __forceinline__ void entry_bit(int i, int& word, int& bit) {
    constexpr int VEC = StagedRow<T>::GRAIN;
    const int c = i / CHUNK, o = i % CHUNK, j = o / (32 * VEC), lane = o / VEC % 32;
    word = c * 32 + lane;
    bit = j * VEC + o % VEC;
}

// coef exp((l - ref) / T) for the entries of a granule, rounded to the type.  PLAIN: 2^(l c - off) says it (offset_ok).
struct GradientTerms {
    float coef, c, off, ref;
};
__device__ __forceinline__ f32x2 gradient_pair(float l0, float l1, const GradientTerms& t) {
    float x0, x1;
    unpack2(ffma2(pack2(l0, l1), pack2(t.c, t.c), pack2(-t.off, -t.off)), x0, x1);
    return fmul2(pack2(ex2_approx(x0), ex2_approx(x1)), pack2(t.coef, t.coef));
}
template <bool PLAIN> __device__ __forceinline__ uint4 gradient_granule(uint4 q, const GradientTerms& t, const __nv_bfloat16*) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float l0 = __uint_as_float(w[i] << 16), l1 = __uint_as_float(w[i] & 0xFFFF0000u);
        float g0, g1;
        if (PLAIN) {
            unpack2(gradient_pair(l0, l1, t), g0, g1);
        } else {
            g0 = l0 == t.ref ? t.coef : t.coef * 0.0f;
            g1 = l1 == t.ref ? t.coef : t.coef * 0.0f;
        }
        const __nv_bfloat162 p = __floats2bfloat162_rn(g0, g1);
        out[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}
template <bool PLAIN> __device__ __forceinline__ uint4 gradient_granule(uint4 q, const GradientTerms& t, const float*) {
    float l[4], g[4];
    unpack_granule(q, l, (const float*)nullptr);
    if (PLAIN) {
        unpack2(gradient_pair(l[0], l[1], t), g[0], g[1]);
        unpack2(gradient_pair(l[2], l[3], t), g[2], g[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = l[i] == t.ref ? t.coef : t.coef * 0.0f;
    }
    return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
}
__device__ __forceinline__ void store_entry(float* row, long long v, float g) { row[v] = g; }
__device__ __forceinline__ void store_entry(__nv_bfloat16* row, long long v, float g) { row[v] = __float2bfloat16_rn(g); }
__device__ __forceinline__ void store_granule(void* p, uint4 q) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
}

// The virtual entries [begin, end) of a row of gradients; g(i) is the i-th granule from `begin` on.  The output row may lie
// differently against the 16-byte granules than the logits; then, and in the row's partial granules, it is stored by element.
template <typename T, typename F>
__device__ __forceinline__ void store_slice(T* out, int mis, int begin, int end, int row_end, F&& g) {
    constexpr int GRAIN = StagedRow<T>::GRAIN;
    const bool same = (int)(reinterpret_cast<uintptr_t>(out) & 15u) == mis * (int)sizeof(T);
    const int granules = (end - begin + GRAIN - 1) / GRAIN;
    const int first = begin < mis ? 1 : 0, last = begin + granules * GRAIN > row_end ? granules - 1 : granules;      // whole ones
    if (same) {
        T* at = out + (begin - mis) + (long long)(first + (int)threadIdx.x) * GRAIN;
#pragma unroll 2
        for (int i = first + (int)threadIdx.x; i < last; i += THREADS, at += THREADS * GRAIN) store_granule(at, g(i));
    }
    const auto by_element = [&](int i) {
        const uint4 q = g(i);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < GRAIN; ++e) {
            const int v = begin + i * GRAIN + e;
            const uint32_t bits = w[e * (int)sizeof(T) / 4] >> (e * (int)sizeof(T) % 4 * 8);
            if (v < mis || v >= row_end) continue;
            if (sizeof(T) == 2) reinterpret_cast<unsigned short*>(out)[v - mis] = (unsigned short)bits;
            else reinterpret_cast<uint32_t*>(out)[v - mis] = bits;
        }
    };
    if (same) {
        if (threadIdx.x == 0 && first == 1 && granules > 0) by_element(0);
        if (threadIdx.x == 32 && last < granules && last >= first) by_element(last);
    } else {
        for (int i = threadIdx.x; i < granules; i += THREADS) by_element(i);
    }
}

// One cluster per row.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(THREADS, 3) distill_kernel(DistillArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[MAX_SLICE_TILES];
    __shared__ DistillRecord records[DISTILL_RECORDS];
    __shared__ double shared_lse, shared_scale;
    __shared__ float shared_coef, shared_off, shared_ref, shared_top;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t ranks;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    const uint32_t rank = cluster_rank();
    const long long row = blockIdx.x / ranks;
    grid_dependency_sync();

    const StagedRow<T> in(reinterpret_cast<const T*>(a.logits) + row * a.row_stride, a.V);
    T* out = GRAD ? reinterpret_cast<T*>(a.grad) + row * a.grad_stride : nullptr;
    int n = a.t_count[row];
    if (n == 0) {           // (the whole cluster: nothing of this row is looked at)
        if (GRAD) {
            const int begin = min((int)rank * a.slice_chunks * CHUNK, in.end);
            store_slice<T>(out, in.mis, begin, min(begin + a.slice_chunks * CHUNK, in.end), in.end, [](int) { return make_uint4(0u, 0u, 0u, 0u); });
        }
        if (rank == 0 && tid == 0 && a.loss) a.loss[row] = 0.0f;
        return;
    }
    cluster_arrive();
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem + (size_t)a.slice_chunks * CHUNK * sizeof(T));
    for (int w = tid; w < a.slice_chunks * 32; w += THREADS) bits[w] = 0u;
    Slice<T> s;
    s.stage(smem, bars, in, rank, a.slice_chunks, false);

    // the teacher's entries: the slice's own are remembered by the thread that read them
    const float T_ = a.temperature[row / a.R];
    const float c32 = temp_scale(T_);
    unsigned bad = temp_ok(T_) && c32 < CUDART_INF_F ? 0u : ST_TEMPERATURE;
    if (n < 0 || n > a.K) bad |= ST_RANGE, n = 0;
    int at[DISTILL_ENTRIES];        // virtual entry, relative to the slice; -1: none
    float t[DISTILL_ENTRIES];
#pragma unroll
    for (int e = 0; e < DISTILL_ENTRIES; ++e) {
        const int j = tid + e * THREADS;
        at[e] = -1;
        t[e] = 0.0f;
        if (j < n) {
            const int x = __ldg(a.t_idx + row * a.K + j);
            t[e] = __ldg(a.t_prob + row * a.K + j);
            if (x < 0 || x >= a.V || !(t[e] >= 0.0f) || t[e] == CUDART_INF_F) {
                bad |= ST_RANGE;
            } else if (x + in.mis >= s.begin && x + in.mis < s.end) {
                at[e] = x + in.mis - s.begin;
                int word, bit;
                entry_bit<T>(at[e], word, bit);
                if (atomicOr(&bits[word], 1u << bit) >> bit & 1u) bad |= ST_RANGE;     // the same index twice
            }
        }
    }

    // sums that need no logits, while the copies are under way (a warp without entries has none)
    const bool entries_here = warp * 32 < n;
    double st = 0.0, stl = 0.0;
    if (entries_here) {
#pragma unroll
        for (int e = 0; e < DISTILL_ENTRIES; ++e) {
            if (e * THREADS >= n) break;
            if (at[e] >= 0 && t[e] > 0.0f) {
                const double td = (double)t[e];
                st += td;
                stl += td * log(td);
            }
        }
        st = warp_sum(st);
        stl = warp_sum(stl);
    }
    __syncthreads();

    // outside the entries: per warp a running maximum, per lane the sum relative to it
    float m = -CUDART_INF_F, off = 0.0f, sum = 0.0f;
    int late = WAIT_OK;
    for (int c = warp; c < s.chunks; c += WARPS) {
        late = max(late, s.wait(c, false, a.wait_limit_ns));
        ChunkRegs<T> r;
        load_staged(r, s.chunk(c), s.begin + c * CHUNK, in.end, lane);
        if (const uint32_t w = bits[c * 32 + lane]) exclude(r, w);
        const float top = warp_max_redux(r.lane_max_plain());
        if (top > m) {          // (warp-uniform; the sum so far moves to the new reference)
            const float to = __fmul_rn(top, c32);
            if (m > -CUDART_INF_F) sum *= ex2_approx(off - to);
            m = top;
            off = to;
        }
        sum += lane_weight_sum(r, m, c32, off);
    }
    // the entries, in double precision
    const double rT = 1.0 / (double)T_;
    float l[DISTILL_ENTRIES], em = -CUDART_INF_F;
    double es = 0.0, stx = 0.0;
#pragma unroll
    for (int e = 0; e < DISTILL_ENTRIES; ++e) l[e] = -CUDART_INF_F;
    if (entries_here) {
#pragma unroll
        for (int e = 0; e < DISTILL_ENTRIES; ++e) {
            if (at[e] >= 0) {
                late = max(late, s.wait(at[e] / CHUNK, false, a.wait_limit_ns));
                l[e] = entry_value(s.data, at[e], (const T*)nullptr);
                if (l[e] != l[e] || l[e] == CUDART_INF_F) bad |= ST_LOGIT;
                em = fmaxf(em, l[e]);
            }
        }
        em = warp_max(em);
#pragma unroll
        for (int e = 0; e < DISTILL_ENTRIES; ++e) {
            if (e * THREADS >= n) break;
            if (at[e] >= 0) {
                const double x = l[e] > -CUDART_INF_F ? ((double)l[e] - (double)em) * rT : -CUDART_INF;
                if (l[e] > -CUDART_INF_F) es += exp_call(x);
                if (t[e] > 0.0f) stx += (double)t[e] * x;
            }
        }
        es = warp_sum(es);
        stx = warp_sum(stx);
    }
    if (late != WAIT_OK) bad |= ST_INTERNAL;
    const float ws = warp_sum(sum);
    if (ws != ws || m == CUDART_INF_F) bad |= ST_LOGIT;
    bad = __reduce_or_sync(0xffffffffu, bad);
    // the warp's record to every CTA
    cluster_wait();
    {
        DistillRecord d;
        d.entry_sum = es; d.t = st; d.t_log_t = stl; d.t_x = stx;
        d.rest_max = m; d.rest_sum = ws; d.entry_max = em; d.status = bad;
        if (lane < (int)ranks) {
            const uint32_t to = peer_addr(&records[rank * WARPS + warp], (uint32_t)lane);
            constexpr int WORDS = sizeof(DistillRecord) / 16;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) peer_store4(to + 16 * i, reinterpret_cast<const uint4*>(&d)[i]);
        }
    }
    cluster_sync();

    // every CTA puts the records together for itself, in the same order: its first warp
    if (warp == 0) {
        const int count = (int)ranks * WARPS;
        float rm = -CUDART_INF_F, xm = -CUDART_INF_F;
        unsigned all_bad = 0u;
        for (int i = lane; i < count; i += 32) {
            rm = fmaxf(rm, records[i].rest_max);
            xm = fmaxf(xm, records[i].entry_max);
            all_bad |= records[i].status;
        }
        rm = warp_max(rm);
        xm = warp_max(xm);
        all_bad = __reduce_or_sync(0xffffffffu, all_bad);
        const float top = fmaxf(rm, xm);
        if (!(top > -CUDART_INF_F)) all_bad |= ST_LOGIT;
        float coef = CUDART_NAN_F, off_rest = 0.0f;
        double lse = 0.0, scale = CUDART_NAN;
        if (all_bad == 0u) {
            double rest = 0.0, entries = 0.0, A = 0.0, tlt = 0.0, tx = 0.0;
            for (int i = lane; i < count; i += 32) {
                const DistillRecord& d = records[i];
                if (d.rest_max > -CUDART_INF_F)
                    rest += (double)d.rest_sum * stream_scale(d.rest_max, c32) * exp_call(((double)d.rest_max - (double)rm) * rT);
                if (d.entry_max > -CUDART_INF_F) {
                    const double x = ((double)d.entry_max - (double)top) * rT;
                    entries += d.entry_sum * exp_call(x);
                    tx += x * d.t;
                }
                A += d.t; tlt += d.t_log_t; tx += d.t_x;
            }
            rest = warp_sum(rest);
            entries = warp_sum(entries);
            A = warp_sum(A);
            tx = warp_sum(tlt - tx);        // sum of t ln t - t (l - top) / T
            // relative to the row's maximum, as all that follows: logarithms of the sum, and of the rest's share R
            const double log_sum_rest = ((double)rm - (double)top) * rT + log(rest);
            lse = log(entries + exp_call(log_sum_rest));
            const double r = a.tail ? fmax(0.0, 1.0 - A) : 0.0, log_rest = rest > 0.0 ? log_sum_rest - lse : -CUDART_INF;
            if (rank == 0 && lane == 0 && a.loss) a.loss[row] = (float)(tx + A * lse + (r > 0.0 ? r * (log(r) - log_rest) : 0.0));
            if (GRAD) {
                const double w = (a.weight ? (double)a.weight[row] : 1.0) * rT;
                scale = w * (A + r);
                coef = 0.0f;
                if (rest > 0.0) {
                    off_rest = __fmul_rn(rm, c32);
                    coef = (float)(w * ((A + r) * exp_call(log_rest) - r) / rest * stream_scale(rm, c32));
                }
            }
        } else if (rank == 0 && lane == 0) {
            if (a.loss) a.loss[row] = CUDART_NAN_F;
            atomicOr(a.status, all_bad);
        }
        if (lane == 0) {
            shared_lse = lse; shared_scale = scale; shared_top = top;
            shared_coef = coef; shared_off = off_rest; shared_ref = rm;
        }
    }
    if (!GRAD) return;
    __syncthreads();
    GradientTerms terms;
    terms.coef = shared_coef; terms.c = c32; terms.off = shared_off; terms.ref = shared_ref;
    const uint4* granules = reinterpret_cast<const uint4*>(s.data);
    if (offset_ok(terms.off))
        store_slice<T>(out, in.mis, s.begin, s.end, in.end, [&](int i) { return gradient_granule<true>(granules[i], terms, (const T*)nullptr); });
    else
        store_slice<T>(out, in.mis, s.begin, s.end, in.end, [&](int i) { return gradient_granule<false>(granules[i], terms, (const T*)nullptr); });
    __syncthreads();        // the entries' gradients replace what the pass left in their places
    const double w = (a.weight ? (double)a.weight[row] : 1.0) * rT, lse = shared_lse, scale = shared_scale, top = (double)shared_top;
#pragma unroll
    for (int e = 0; e < DISTILL_ENTRIES; ++e)
        if (at[e] >= 0)
            store_entry(out, (long long)(at[e] + s.begin - in.mis), (float)(scale * exp_call(((double)l[e] - top) * rT - lse) - w * (double)t[e]));
}

constexpr int DISTILL_SLICE_BYTES = 66 * 1024;      // three CTAs per SM
constexpr int DISTILL_SLICE_LARGE = 100 * 1024;     // two
constexpr int DISTILL_SMEM_MOST = 190000;           // dynamic shared memory

// bytes of dynamic shared memory: the slice and its entries' bits
inline int distill_smem(int slice_chunks, int elem) { return slice_chunks * (CHUNK * elem + 128); }

}  // namespace picospec
