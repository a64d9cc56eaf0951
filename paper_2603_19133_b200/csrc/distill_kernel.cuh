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
// that come twice).  Sums over the entries and over the warps are in double precision.  What goes into them -- exponentials of
// exponents formed in double, ln t -- and the row's coefficients of the gradient are fp32, to about 2^-22: the error that the
// streaming sums have anyway.
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
    long long rows;             // B * R
};

// What one warp knows of its part of the row; sums of exponentials are of exp((l - max) / T).
struct __align__(16) DistillRecord {
    double entry_sum;                            // over its entries
    double t, t_log_t, t_x;                      // over its entries: sums of t, t ln t, t (l - entry_max) / T
    float rest_max, rest_sum;                    // outside the entries; the sum up to stream_scale()
    float entry_max;
    unsigned status;
};
constexpr int DISTILL_FEW = THREADS;         // teacher entries up to which a thread has one

// Exclude the entries whose bit is set: their weight is zero.  Most chunks have none or one, in some lane: `any` is the
// warp's bits together, and four entries at a time are passed over where no lane has one.
__device__ __forceinline__ void exclude(ChunkRegs<__nv_bfloat16>& r, uint32_t bits, uint32_t any) {
#pragma unroll
    for (int g = 0; g < 8; ++g) {
        if (any >> (4 * g) & 15u) {
#pragma unroll
            for (int k = 2 * g; k < 2 * g + 2; ++k) {
                if (bits >> (2 * k) & 1u) r.w[k] = (r.w[k] & 0xFFFF0000u) | 0xFF80u;
                if (bits >> (2 * k + 1) & 1u) r.w[k] = (r.w[k] & 0xFFFFu) | 0xFF800000u;
            }
        }
    }
}
__device__ __forceinline__ void exclude(ChunkRegs<float>& r, uint32_t bits, uint32_t any) {
#pragma unroll
    for (int g = 0; g < 8; ++g) {
        if (any >> (4 * g) & 15u) {
#pragma unroll
            for (int k = 4 * g; k < 4 * g + 4; ++k)
                if (bits >> k & 1u) r.f[k] = -CUDART_INF_F;
        }
    }
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

// Stores the gradients of a slice, the virtual entries [begin, end) of a row: g(i) is its i-th granule.  The output row
// may lie differently against the 16-byte granules than the logits; then, and in the row's partial granules, it is stored by
// element.
template <typename T> struct GradientStore {
    static constexpr int GRAIN = StagedRow<T>::GRAIN;
    T* out;
    int mis, begin, row_end, granules, first, last;     // [first, last): the granules that are stored whole
    bool same;
    __device__ __forceinline__ GradientStore(T* row, int misaligned, int slice_begin, int slice_end, int end_of_row)
        : out(row), mis(misaligned), begin(slice_begin), row_end(end_of_row) {
        same = (int)(reinterpret_cast<uintptr_t>(row) & 15u) == mis * (int)sizeof(T);
        granules = (slice_end - begin + GRAIN - 1) / GRAIN;
        first = begin < mis ? 1 : 0;
        last = begin + granules * GRAIN > row_end ? granules - 1 : granules;
    }
    __device__ __forceinline__ void by_element(int i, uint4 q) const {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < GRAIN; ++e) {
            const int v = begin + i * GRAIN + e;
            const uint32_t bits = w[e * (int)sizeof(T) / 4] >> (e * (int)sizeof(T) % 4 * 8);
            if (v < mis || v >= row_end) continue;
            if (sizeof(T) == 2) reinterpret_cast<unsigned short*>(out)[v - mis] = (unsigned short)bits;
            else reinterpret_cast<uint32_t*>(out)[v - mis] = bits;
        }
    }
    // granules [from, to), as far as the slice goes
    template <typename F> __device__ __forceinline__ void store(int from, int to, F&& g) const {
        to = min(to, granules);
        if (!same) {
            for (int i = from + (int)threadIdx.x; i < to; i += THREADS) by_element(i, g(i));
            return;
        }
        const int a = max(from, first), b = min(to, last);
        T* at = out + (begin - mis) + (long long)(a + (int)threadIdx.x) * GRAIN;
#pragma unroll 2
        for (int i = a + (int)threadIdx.x; i < b; i += THREADS, at += THREADS * GRAIN) store_granule(at, g(i));
        if (threadIdx.x == 0 && first == 1 && from == 0 && granules > 0) by_element(0, g(0));
        if (threadIdx.x == 32 && last < granules && last >= max(from, first) && last < to) by_element(last, g(last));
    }
};

// What a thread knows of a row beside its logits.
template <int PER> struct DistillHeader {
    int n;
    float T, weight;
    int index[PER];
    float t[PER];
    // (asked for at once, and in this place: behind the copies of the logits they would wait for those)
    __device__ __forceinline__ void load(const DistillArgs& a, long long row) {
        n = load_now(a.t_count + row);
        T = load_now(a.temperature + row / a.R);
        weight = a.weight ? load_now(a.weight + row) : 1.0f;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int j = (int)threadIdx.x + e * THREADS;
            index[e] = j < a.K ? load_now(a.t_idx + row * a.K + j) : 0;
            t[e] = j < a.K ? load_now(a.t_prob + row * a.K + j) : 0.0f;
        }
    }
};

// A row's loss, and what its gradient takes, from the records of the cluster's warps (by one warp).  It stands between the two
// passes, so its exponentials are short: their errors are those of the streaming sums that they multiply.
struct DistillRow {
    double A, tx, total, rest, far, r;      // tx: sum of t ln t - t (l - top) / T;  total: of exp((l - top) / T);  far: (rest_max - top) / T
    unsigned bad;
};
template <bool GRAD>
__device__ __forceinline__ DistillRow put_together(const DistillRecord* records, int count, int lane, float c32, double rT, float weight, bool tail,
                                                   float& out_scale, float& out_coef, float& out_off, float& out_ref, float& out_top) {
    float rm = -CUDART_INF_F, xm = -CUDART_INF_F;
    DistillRow x{};
    for (int i = lane; i < count; i += 32) {
        rm = fmaxf(rm, records[i].rest_max);
        xm = fmaxf(xm, records[i].entry_max);
        x.bad |= records[i].status;
    }
    rm = warp_max_redux(rm);
    xm = warp_max_redux(xm);
    x.bad = __reduce_or_sync(0xffffffffu, x.bad);
    const float top = fmaxf(rm, xm);
    if (!(top > -CUDART_INF_F)) x.bad |= ST_LOGIT;
    float coef = CUDART_NAN_F, off_rest = 0.0f, scale = CUDART_NAN_F;
    if (x.bad == 0u) {
        double entries = 0.0, tlt = 0.0;
        for (int i = lane; i < count; i += 32) {
            const DistillRecord& d = records[i];
            if (d.rest_max > -CUDART_INF_F)
                x.rest += (double)(d.rest_sum * stream_scale_near(d.rest_max, c32)) * (double)exp_near(((double)d.rest_max - (double)rm) * rT);
            if (d.entry_max > -CUDART_INF_F) {
                const double y = ((double)d.entry_max - (double)top) * rT;
                entries += d.entry_sum * (double)exp_near(y);
                x.tx += y * d.t;
            }
            x.A += d.t;
            x.tx += d.t_x;
            tlt += d.t_log_t;
        }
        x.far = ((double)rm - (double)top) * rT;
        const double factor = rm > -CUDART_INF_F ? (double)exp_near(x.far) : 0.0;
        x.tx = tlt - x.tx;
        warp_sums(x.rest, entries, x.A, x.tx);
        x.total = fma(x.rest, factor, entries);
        x.r = tail ? fmax(0.0, 1.0 - x.A) : 0.0;
        if (GRAD) {
            // (A + r) w / total on the entries, w ((A + r) R - r) / rest elsewhere, R = rest factor / total
            const double w = (double)weight * rT;
            const float by_total = __frcp_rn((float)x.total);
            scale = (float)(w * (x.A + x.r)) * by_total;
            coef = 0.0f;
            if (x.rest > 0.0) {
                off_rest = __fmul_rn(rm, c32);
                const double share = w * fma((x.A + x.r) * factor, x.rest, -x.r * x.total);
                coef = __fdividef((float)share * stream_scale_near(rm, c32), (float)x.rest) * by_total;
            }
        }
    }
    if (lane == 0) {
        out_scale = scale; out_top = top;
        out_coef = coef; out_off = off_rest; out_ref = rm;
    }
    return x;
}
__device__ __forceinline__ void write_loss(const DistillArgs& a, long long row, const DistillRow& x) {
    if (x.bad != 0u) {
        if (a.loss) a.loss[row] = CUDART_NAN_F;
        atomicOr(a.status, x.bad);
    } else if (a.loss) {
        // ln s = (l - top) / T - ln total;  ln R = ln rest + far - ln total
        const double lse = log(x.total);
        double loss = x.tx + x.A * lse;
        if (x.r > 0.0) loss += x.r * (log(x.r) - (x.rest > 0.0 ? log(x.rest) + x.far - lse : -CUDART_INF));
        a.loss[row] = (float)loss;
    }
}

// A cluster takes rows blockIdx / cluster size, and on from there in steps of the number of clusters.  While the gradient of a row is
// written, tile by tile, the next row's tiles are fetched into the place of those that are done.
// Bound: HBM (a read of the logits and a write of the gradient), next the exponential (two per entry at 16 a clock and SM), which the
// waits at the exchange between the passes keep from overlapping: 2048 rows of 128256 bf16 257 us, 4.1 TB/s, 0.64 of the copy rate.
// PER: teacher entries a thread; CTAS: per SM, three, or four where their slices fit (V = 50381 in two slices of 50 KB: 58 -> 53 us
// for 999 rows; at three by their slices the 64 registers that four leave cost 2 %).
template <typename T, bool GRAD, int PER, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) distill_kernel(DistillArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[MAX_SLICE_TILES];
    __shared__ float shared_scale, shared_coef, shared_off, shared_ref, shared_top;
    __shared__ int shared_lost[2];
    constexpr int TILE = TILE_CHUNKS * CHUNK / StagedRow<T>::GRAIN;      // granules
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t ranks;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    const uint32_t rank = cluster_rank();
    const long long clusters = gridDim.x / ranks;
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem + (size_t)a.slice_chunks * CHUNK * sizeof(T));
    DistillRecord* records = reinterpret_cast<DistillRecord*>(bits + a.slice_chunks * 32);      // [2][ranks * WARPS]
    Slice<T> s;
    s.init(smem, bars);
    if (tid < 2) shared_lost[tid] = 0;
    for (int w = tid; w < a.slice_chunks * 32; w += THREADS) bits[w] = 0u;
    cluster_arrive();
    cluster_wait();
    grid_dependency_sync();

    const auto staged = [&](long long r) { return StagedRow<T>(reinterpret_cast<const T*>(a.logits) + r * a.row_stride, a.V); };
    long long row = blockIdx.x / ranks;
    DistillHeader<PER> h;
    h.load(a, row);
    if (h.n != 0) s.stage(staged(row), rank, a.slice_chunks, false);
    uint32_t parity = 0u, copy = 0u;
    for (; row < a.rows; row += clusters) {
        const StagedRow<T> in = staged(row);
        const long long next = row + clusters;
        s.locate(in, rank, a.slice_chunks, false);
        T* out = GRAD ? reinterpret_cast<T*>(a.grad) + row * a.grad_stride : nullptr;
        const GradientStore<T> store(out, in.mis, s.begin, s.end, in.end);
        if (h.n == 0) {         // (the whole cluster: nothing of this row is looked at)
            if (next < a.rows) {
                h.load(a, next);
                if (h.n != 0) s.stage(staged(next), rank, a.slice_chunks, false);
            }
            if (GRAD) store.store(0, store.granules, [](int) { return make_uint4(0u, 0u, 0u, 0u); });
            if (rank == 0 && tid == 0 && a.loss) a.loss[row] = 0.0f;
            continue;
        }

        // the teacher's entries: the slice's own are remembered by the thread that read them
        const float T_ = h.T, weight = h.weight, c32 = temp_scale(T_);
        int n = h.n;
        unsigned bad = temp_ok(T_) && c32 < CUDART_INF_F ? 0u : ST_TEMPERATURE;
        if (n < 0 || n > a.K) bad |= ST_RANGE, n = 0;
        int at[PER];            // virtual entry, relative to the slice; -1: none
        float t[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            at[e] = -1;
            t[e] = h.t[e];
            if (tid + e * THREADS < n) {
                const int x = h.index[e];
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
        if (tid == 0) shared_lost[copy ^ 1u] = 0;
        if (next < a.rows) h.load(a, next);

        // outside the entries: per warp a running maximum, per lane the sum relative to it
        float m = -CUDART_INF_F, off = 0.0f, sum = 0.0f;
        int late = WAIT_OK;
        for (int c = warp; c < s.chunks; c += WARPS) {
            late = max(late, s.wait(c, false, a.wait_limit_ns, parity));
            ChunkRegs<T> r;
            load_staged(r, s.chunk(c), s.begin + c * CHUNK, in.end, lane);
            const uint32_t w = bits[c * 32 + lane];
            if (const uint32_t any = __reduce_or_sync(0xffffffffu, w)) exclude(r, w, any);
            const float top = warp_max_redux(r.lane_max_plain());
            if (top > m) {          // (warp-uniform; the sum so far moves to the new reference)
                const float to = __fmul_rn(top, c32);
                // (beyond offset_ok, where both products may be infinite, any two references are 64 powers of two and more apart)
                if (m > -CUDART_INF_F) sum *= offset_ok(off) && offset_ok(to) ? ex2_approx(off - to) : 0.0f;
                m = top;
                off = to;
            }
            sum += lane_weight_sum(r, m, c32, off);
        }
        // the tiles that the row does not reach have barriers too
        for (int u = (s.chunks + TILE_CHUNKS - 1) / TILE_CHUNKS; u < s.tiles; ++u) late = max(late, mbar_wait_twice(&s.bars[u], parity, a.wait_limit_ns));
        // the entries, in double precision
        const double rT = 1.0 / (double)T_;
        float l[PER], em = -CUDART_INF_F;
        double es = 0.0, st = 0.0, stl = 0.0, stx = 0.0;
#pragma unroll
        for (int e = 0; e < PER; ++e) l[e] = -CUDART_INF_F;
        if (warp * 32 < n) {        // (a warp without entries has none)
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (at[e] >= 0) {
                    late = max(late, s.wait(at[e] / CHUNK, false, a.wait_limit_ns, parity));
                    l[e] = entry_value(s.data, at[e], (const T*)nullptr);
                    if (l[e] != l[e] || l[e] == CUDART_INF_F) bad |= ST_LOGIT;
                    em = fmaxf(em, l[e]);
                }
            }
            em = warp_max_redux(em);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (e * THREADS >= n) break;
                if (at[e] >= 0) {
                    const double x = l[e] > -CUDART_INF_F ? ((double)l[e] - (double)em) * rT : -CUDART_INF, td = (double)t[e];
                    if (l[e] > -CUDART_INF_F) es += (double)exp_near(x);
                    if (td > 0.0) {
                        st += td;
                        stl += td * (double)logf(t[e]);
                        stx += td * x;
                    }
                }
            }
            warp_sums(es, stx, st, stl);
        }
        late = __reduce_max_sync(0xffffffffu, late);       // (one outcome for the warp: each CTA is told by another lane)
        // (a copy may still land in the slice: the cluster gives up)
        if (late == WAIT_LOST && lane < (int)ranks) peer_store(peer_addr(&shared_lost[copy], (uint32_t)lane), 1u);
        if (late != WAIT_OK) bad |= ST_INTERNAL;
        const float ws = warp_sum(sum);
        if (ws != ws || m == CUDART_INF_F) bad |= ST_LOGIT;
        bad = __reduce_or_sync(0xffffffffu, bad);
        // the warp's record to every CTA
        {
            DistillRecord d;
            d.entry_sum = es; d.t = st; d.t_log_t = stl; d.t_x = stx;
            d.rest_max = m; d.rest_sum = ws; d.entry_max = em; d.status = bad;
            if (lane < (int)ranks) {
                const uint32_t to = peer_addr(&records[(copy * ranks + rank) * WARPS + warp], (uint32_t)lane);
                constexpr int WORDS = sizeof(DistillRecord) / 16;
#pragma unroll
                for (int i = 0; i < WORDS; ++i) peer_store4(to + 16 * i, reinterpret_cast<const uint4*>(&d)[i]);
            }
        }
        cluster_sync();
        const bool lost = shared_lost[copy] != 0;
        const bool more = next < a.rows && h.n != 0 && !lost;
        if (!GRAD && more) s.stage(staged(next), rank, a.slice_chunks, false);

        // every CTA puts the records together for itself, in the same order: its first warp
        DistillRow x{};
        if (warp == 0)
            x = put_together<GRAD>(records + copy * ranks * WARPS, (int)ranks * WARPS, lane, c32, rT, weight, a.tail != 0, shared_scale, shared_coef,
                                   shared_off, shared_ref, shared_top);
#pragma unroll
        for (int e = 0; e < PER; ++e) {         // (every warp is done with the bits)
            int word, bit;
            entry_bit<T>(max(at[e], 0), word, bit);
            if (at[e] >= 0) bits[word] = 0u;
        }
        __syncthreads();
        if (rank == 0 && tid == 0) write_loss(a, row, x);
        if (GRAD) {
            GradientTerms terms;
            terms.coef = shared_coef; terms.c = c32; terms.off = shared_off; terms.ref = shared_ref;
            const uint4* granules = reinterpret_cast<const uint4*>(s.data);
            const bool plain = offset_ok(terms.off);
            const StagedRow<T> in_next = staged(next);
            for (int u = 0; u < s.tiles; ++u) {
                if (plain)
                    store.store(u * TILE, (u + 1) * TILE, [&](int i) { return gradient_granule<true>(granules[i], terms, (const T*)nullptr); });
                else
                    store.store(u * TILE, (u + 1) * TILE, [&](int i) { return gradient_granule<false>(granules[i], terms, (const T*)nullptr); });
                __syncthreads();        // the tile is done with, and the entries' gradients below come behind what was stored in their places
                if (more && tid == 0) s.issue(in_next, rank, a.slice_chunks, false, u);
            }
            const double w = (double)weight * rT, scale = (double)shared_scale, largest = (double)shared_top;
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (at[e] >= 0)
                    store_entry(out, (long long)(at[e] + s.begin - in.mis), (float)(scale * exp_call(((double)l[e] - largest) * rT) - w * (double)t[e]));
        }
        if (lost) {
            for (long long r = next; rank == 0 && tid == 0 && a.loss && r < a.rows; r += clusters) a.loss[r] = CUDART_NAN_F;
            break;
        }
        parity ^= 1u;
        copy ^= 1u;
    }
}

constexpr int DISTILL_SLICE_BYTES = 66 * 1024;      // three CTAs per SM with what lies beside the slice, in clusters of up to six; beside the
                                                    // larger records of seven and eight CTAs a full slice leaves room for two
constexpr int DISTILL_SMEM_FOUR = 57000;            // dynamic shared memory up to which four fit
constexpr int DISTILL_SLICE_LARGE = 100 * 1024;     // two
constexpr int DISTILL_SMEM_MOST = 190000;           // dynamic shared memory

// bytes of dynamic shared memory: the slice, its entries' bits, the records of two rows
inline int distill_smem(int slice_chunks, int elem, int cluster) {
    return slice_chunks * (CHUNK * elem + 128) + 2 * cluster * WARPS * (int)sizeof(DistillRecord);
}

}  // namespace picospec
