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

// What one CTA knows about its slice.  Sums of exponentials are of exp((l - max) / T).
struct DistillRecord {
    double rest_sum, entry_sum;                  // outside the entries, over the entries
    double t, t_log_t, t_x;                      // over the slice's entries: sums of t, t ln t, t (l - entry_max) / T
    float rest_max, entry_max;
    unsigned status, pad;
};
static_assert(sizeof(DistillRecord) % 4 == 0, "exchanged word by word");

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

__device__ __forceinline__ uint4 pack_gradient(const float* g, const __nv_bfloat16*) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(g[2 * i], g[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack_gradient(const float* g, const float*) {
    return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
}
__device__ __forceinline__ void store_entry(float* row, long long v, float g) { row[v] = g; }
__device__ __forceinline__ void store_entry(__nv_bfloat16* row, long long v, float g) { row[v] = __float2bfloat16_rn(g); }
__device__ __forceinline__ void store_granule(void* p, uint4 q) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
}

// The gradient of the virtual entries [begin, end) of a row: g(granule of the slice, GRAIN gradients).  The output row may
// lie differently against the 16-byte granules than the logits; then, and in the row's partial granules, it is stored by element.
template <typename T, typename F>
__device__ __forceinline__ void store_slice(T* out, int mis, int begin, int end, int row_end, F&& g) {
    constexpr int GRAIN = StagedRow<T>::GRAIN;
    const bool same = (int)(reinterpret_cast<uintptr_t>(out) & 15u) == mis * (int)sizeof(T);
    for (int v = begin + (int)threadIdx.x * GRAIN; v < end; v += THREADS * GRAIN) {
        float x[GRAIN];
        g((v - begin) / GRAIN, x);
        if (same && v >= mis && v + GRAIN <= row_end) {
            store_granule(out + (v - mis), pack_gradient(x, (const T*)nullptr));
        } else {
#pragma unroll
            for (int e = 0; e < GRAIN; ++e)
                if (v + e >= mis && v + e < row_end) store_entry(out, (long long)(v + e - mis), x[e]);
        }
    }
}

// One cluster per row.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(THREADS, 3) distill_kernel(DistillArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[MAX_SLICE_TILES];
    __shared__ DistillRecord records[MAX_CLUSTER], mine;
    __shared__ double part[WARPS][5];
    __shared__ float part_max[WARPS][2];
    __shared__ unsigned status;
    __shared__ double shared_lse, shared_scale;
    __shared__ float shared_coef, shared_off, shared_ref, shared_top;
    constexpr int GRAIN = StagedRow<T>::GRAIN;
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
            store_slice<T>(out, in.mis, begin, min(begin + a.slice_chunks * CHUNK, in.end), in.end, [](int, float* x) {
#pragma unroll
                for (int e = 0; e < GRAIN; ++e) x[e] = 0.0f;
            });
        }
        if (rank == 0 && tid == 0 && a.loss) a.loss[row] = 0.0f;
        return;
    }
    cluster_arrive();
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem + (size_t)a.slice_chunks * CHUNK * sizeof(T));
    if (tid == 0) status = 0u;
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
#pragma unroll
    for (int e = 0; e < DISTILL_ENTRIES; ++e) {
        l[e] = -CUDART_INF_F;
        if (at[e] >= 0) {
            late = max(late, s.wait(at[e] / CHUNK, false, a.wait_limit_ns));
            l[e] = entry_value(s.data, at[e], (const T*)nullptr);
            if (l[e] != l[e] || l[e] == CUDART_INF_F) bad |= ST_LOGIT;
            em = fmaxf(em, l[e]);
        }
    }
    if (late != WAIT_OK) bad |= ST_INTERNAL;
    em = warp_max(em);
    double es = 0.0, st = 0.0, stl = 0.0, stx = 0.0;
#pragma unroll
    for (int e = 0; e < DISTILL_ENTRIES; ++e) {
        if (at[e] >= 0) {
            const double x = l[e] > -CUDART_INF_F ? ((double)l[e] - (double)em) * rT : -CUDART_INF, td = (double)t[e];
            if (l[e] > -CUDART_INF_F) es += exp_call(x);
            if (td > 0.0) {
                st += td;
                stl += td * log(td);
                stx += td * x;
            }
        }
    }
    const float ws = warp_sum(sum);
    es = warp_sum(es); st = warp_sum(st); stl = warp_sum(stl); stx = warp_sum(stx);
    if (ws != ws || m == CUDART_INF_F) bad |= ST_LOGIT;
    if (lane == 0) {
        part[warp][0] = (double)ws * (m > -CUDART_INF_F ? stream_scale(m, c32) : 1.0);
        part[warp][1] = es; part[warp][2] = st; part[warp][3] = stl; part[warp][4] = stx;
        part_max[warp][0] = m;
        part_max[warp][1] = em;
    }
    if (bad) atomicOr(&status, bad);
    __syncthreads();
    if (tid == 0) {
        DistillRecord d{};
        d.rest_max = d.entry_max = -CUDART_INF_F;
        for (int w = 0; w < WARPS; ++w) {
            d.rest_max = fmaxf(d.rest_max, part_max[w][0]);
            d.entry_max = fmaxf(d.entry_max, part_max[w][1]);
        }
        for (int w = 0; w < WARPS; ++w) {
            if (part_max[w][0] > -CUDART_INF_F) d.rest_sum += part[w][0] * exp_call(((double)part_max[w][0] - (double)d.rest_max) * rT);
            if (part_max[w][1] > -CUDART_INF_F) {
                const double x = ((double)part_max[w][1] - (double)d.entry_max) * rT;
                d.entry_sum += part[w][1] * exp_call(x);
                d.t_x += x * part[w][2];
            }
            d.t += part[w][2]; d.t_log_t += part[w][3]; d.t_x += part[w][4];
        }
        d.status = status;
        mine = d;
    }
    __syncthreads();
    constexpr int WORDS = sizeof(DistillRecord) / 4;
    cluster_wait();
    for (int i = tid; i < (int)ranks * WORDS; i += THREADS)
        peer_store(peer_addr(reinterpret_cast<uint32_t*>(&records[rank]) + i % WORDS, i / WORDS), reinterpret_cast<const uint32_t*>(&mine)[i % WORDS]);
    cluster_sync();

    // every CTA puts the records together for itself, in the same order
    if (tid == 0) {
        float rm = -CUDART_INF_F, xm = -CUDART_INF_F;
        unsigned st_all = 0u;
        for (uint32_t i = 0; i < ranks; ++i) {
            rm = fmaxf(rm, records[i].rest_max);
            xm = fmaxf(xm, records[i].entry_max);
            st_all |= records[i].status;
        }
        double rest = 0.0, entries = 0.0, A = 0.0, tlt = 0.0, tx = 0.0;
        for (uint32_t i = 0; i < ranks; ++i) {
            const DistillRecord& d = records[i];
            if (d.rest_max > -CUDART_INF_F) rest += d.rest_sum * exp_call(((double)d.rest_max - (double)rm) * rT);
            if (d.entry_max > -CUDART_INF_F) {
                entries += d.entry_sum * exp_call(((double)d.entry_max - (double)xm) * rT);
                tx += ((double)d.entry_max - (double)fmaxf(rm, xm)) * rT * d.t;
            }
            A += d.t; tlt += d.t_log_t; tx += d.t_x;
        }
        const float top = fmaxf(rm, xm);
        if (!(top > -CUDART_INF_F)) st_all |= ST_LOGIT;
        float coef = 0.0f, off_rest = 0.0f, ref_rest = 0.0f;
        double lse = 0.0, scale = 0.0;
        if (st_all == 0u) {
            const double rest_part = rest > 0.0 ? rest * exp_call(((double)rm - (double)top) * rT) : 0.0;
            const double entry_part = entries > 0.0 ? entries * exp_call(((double)xm - (double)top) * rT) : 0.0;
            lse = log(rest_part + entry_part);              // relative to the row's maximum, as all that follows
            const double r = a.tail ? fmax(0.0, 1.0 - A) : 0.0;
            const double log_rest = rest > 0.0 ? ((double)rm - (double)top) * rT + log(rest) - lse : -CUDART_INF;       // ln R
            if (rank == 0 && a.loss) a.loss[row] = (float)(tlt - tx + A * lse + (r > 0.0 ? r * (log(r) - log_rest) : 0.0));
            if (GRAD) {
                const double w = (a.weight ? (double)a.weight[row] : 1.0) * rT;
                scale = w * (A + r);
                if (rest > 0.0) {
                    ref_rest = rm;
                    off_rest = __fmul_rn(rm, c32);
                    coef = (float)(w * ((A + r) * exp_call(log_rest) - r) / rest * stream_scale(rm, c32));
                }
            }
        } else {
            if (rank == 0) {
                if (a.loss) a.loss[row] = CUDART_NAN_F;
                atomicOr(a.status, st_all);
            }
            coef = CUDART_NAN_F;
            scale = CUDART_NAN;
        }
        shared_lse = lse; shared_top = top; shared_scale = scale; shared_coef = coef; shared_off = off_rest; shared_ref = ref_rest;
    }
    if (!GRAD) return;
    __syncthreads();
    const float coef = shared_coef, off_rest = shared_off, ref_rest = shared_ref;
    const bool ok = offset_ok(off_rest);
    store_slice<T>(out, in.mis, s.begin, s.end, in.end, [&](int granule, float* x) {
        unpack_granule(reinterpret_cast<const uint4*>(s.data)[granule], x, (const T*)nullptr);
#pragma unroll
        for (int e = 0; e < GRAIN; ++e) x[e] = coef * (ok ? ex2_approx(fmaf(x[e], c32, -off_rest)) : x[e] == ref_rest ? 1.0f : 0.0f);
    });
    __syncthreads();        // the entries' gradients replace what the pass left in their places
    const double w = (a.weight ? (double)a.weight[row] : 1.0) * rT, lse = shared_lse, scale = shared_scale, top = (double)shared_top;
#pragma unroll
    for (int e = 0; e < DISTILL_ENTRIES; ++e)
        if (at[e] >= 0)
            store_entry(out, (long long)(at[e] + s.begin - in.mis), (float)(scale * exp_call(((double)l[e] - top) * rT - lse) - w * (double)t[e]));
}

constexpr int DISTILL_SLICE_BYTES = 64 * 1024;      // three CTAs per SM

// bytes of dynamic shared memory: the slice and its entries' bits
inline int distill_smem(int slice_chunks, int elem) { return slice_chunks * (CHUNK * elem + 128); }

}  // namespace picospec
