// Rules on rows of logits: penalties for tokens that a sequence holds already, biases, grammar masks; and their gradient.
//
//   c = occurrences of v among the tokens that the sequence made (history[prompt_length .. length), and the drafted tokens before the row)
//   s = c > 0, or v is in the prompt (history[0 .. prompt_length))
//   y = (s ? (l > 0 ? l / rho : l rho) : l) - frequency c - presence [c > 0] + bias_v;     -inf where the mask forbids v
//   dL/dl = dL/dy (s ? (l > 0 ? 1 / rho : rho) : 1);                                      0 where the mask forbids v
//
// A CTA takes a slice of the vocabulary of a few consecutive rows of one sequence.  It streams the rows through, masks applied, in
// granules of 16 bytes; in place only granules with a forbidden entry are touched.  Then it reads the sequence's history and
// keeps, in shared memory, a word per entry of the slice (count, whether the prompt has it, whether it has a bias); from the words a
// list of those that are not 0, and the entries of the list are computed, in double precision and rounded once
// (penalty and logit may cancel), and stored over what the stream left, which is in L2 still.  They are few, and by themselves they
// keep all threads busy: in the middle of the stream their code ran in a quarter of the warps at a time, for one or two lanes, and did not fit the
// instruction cache (256 x 7 rows of 128256, three penalties: 640 us).
#pragma once
#include "common.cuh"

namespace picospec {

constexpr int RULES_SLICE = 8192;               // most vocabulary entries of a CTA
constexpr int RULES_SLICE_LEAST = 1024;         // fewest, where there are too few rows to fill the GPU (four a thread)
constexpr int RULES_ROWS = 16;                  // most rows of a CTA
constexpr int RULES_AT_ONCE = 4;                // rows of a listed entry that a thread takes together
constexpr int RULES_AHEAD = 4;                  // granules that a thread has on the way
constexpr uint32_t RULES_PROMPT = 1u << 30;     // word of an entry: the prompt has it,
constexpr uint32_t RULES_DRAFT = 1u << 31;      // a drafted token of the CTA's own rows is it,
constexpr uint32_t RULES_BIAS = 1u << 29;       // it has a bias,
constexpr uint32_t RULES_COUNT = (1u << 29) - 1;    // how often it was made before the CTA's first row (2^27 in the history and as many drafts at most)

struct RulesArgs {
    const void* in;             // logits, or the gradient that arrives
    long long in_stride;
    const void* logits;         // backward with repetition: the logits (their signs)
    long long logits_stride;
    void* out;
    long long out_stride;
    int R, V;
    const int* history;         // [B, capacity] or null
    long long history_stride;
    int capacity;
    const int* length;          // [B]
    const int* prompt_length;   // [B] or null (0)
    const int* draft_tok;       // [B, R - 1] or null
    const float* repetition;    // [B] or null, as the next two
    const float* presence;
    const float* frequency;
    const int* bias_idx;        // [B, bias_k] or null
    const float* bias;
    const int* bias_count;      // [B]
    int bias_k;
    const int* mask;            // [mask_rows, words] or null
    long long mask_stride;
    int mask_rows;
    const int* mask_row;        // [B, R] or null (the row itself)
    unsigned* status;
    int slice, slices, row_block, row_blocks;
};

// shared memory: the words, the list of entries whose word is not 0, the biases' places
__host__ __device__ __forceinline__ int rules_smem(int slice, bool sparse, bool bias) { return sparse ? slice * 6 + (bias ? slice * 2 : 0) : 0; }

// `n` bits of a mask from bit `at` on
__device__ __forceinline__ uint32_t mask_bits(const int* words, int at, int n) {
    const uint32_t lo = (uint32_t)__ldg(words + (at >> 5)), hi = (at & 31) + n > 32 ? (uint32_t)__ldg(words + (at >> 5) + 1) : 0u;
    return __funnelshift_r(lo, hi, at & 31) & ((1u << n) - 1u);
}

// How the entries lie in a granule of 16 bytes
template <typename T> struct Granule;
template <> struct Granule<float> {
    static constexpr int N = 4;
    static constexpr uint32_t LOWEST = 0xFF800000u, NOT = 0x7FC00000u;      // -inf, NaN
    using Bits = uint32_t;
    // entries whose bit is 0 become `other`
    static __device__ __forceinline__ void keep(uint32_t (&w)[4], uint32_t bits, uint32_t other) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = bits >> k & 1u ? w[k] : other;
    }
    static __device__ __forceinline__ float value(Bits x) { return __uint_as_float(x); }
    static __device__ __forceinline__ Bits round(double y) { return __float_as_uint((float)y); }
};
template <> struct Granule<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t LOWEST = 0xFF80u, NOT = 0x7FC0u;
    using Bits = unsigned short;
    static __device__ __forceinline__ void keep(uint32_t (&w)[4], uint32_t bits, uint32_t other) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t m = (bits >> (2 * k) & 1u) * 0xFFFFu | (bits >> (2 * k + 1) & 1u) * 0xFFFF0000u;
            w[k] = (w[k] & m) | (other * 0x10001u & ~m);
        }
    }
    static __device__ __forceinline__ float value(Bits x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ Bits round(double y) { return __bfloat16_as_ushort(__double2bfloat16(y)); }
};

// (not the read-only path: the call may work in place)
__device__ __forceinline__ void load_granule(uint32_t (&w)[4], const void* p) {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store_granule(void* p, const uint32_t (&w)[4]) {
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
template <typename B> __device__ __forceinline__ B load_entry(const B* p) { return *reinterpret_cast<const volatile B*>(p); }

// The slice's part of one row as granules on 16-byte boundaries of the output; the first and the last may be cut short.
template <typename T, bool INPLACE>
__device__ __forceinline__ void rules_row(const typename Granule<T>::Bits* in, typename Granule<T>::Bits* out, const int* mask, int v0, int n, uint32_t other, int tid) {
    using G = Granule<T>;
    constexpr int N = G::N;
    constexpr uint32_t FULL = (1u << N) - 1u;
    const int lead = (int)((16 - ((uintptr_t)out & 15)) & 15) / (int)sizeof(T);
    const bool level = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
    const int first = min(lead, n), whole = (n - first) / N, ends = n - whole * N;
    for (int u0 = tid; u0 < whole; u0 += RULES_AHEAD * THREADS) {
        uint32_t x[RULES_AHEAD][4], allowed[RULES_AHEAD];
#pragma unroll
        for (int k = 0; k < RULES_AHEAD; ++k) {
            const int u = u0 + k * THREADS;
            allowed[k] = u >= whole ? 0u : mask ? mask_bits(mask, v0 + first + u * N, N) : FULL;
        }
#pragma unroll
        for (int k = 0; k < RULES_AHEAD; ++k) {
            const auto* p = in + first + (u0 + k * THREADS) * N;
            if (allowed[k] == 0u || (INPLACE && allowed[k] == FULL)) continue;
            if (level) load_granule(x[k], p);
            else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    x[k][j] = sizeof(T) == 4 ? (uint32_t)load_entry(p + j) : (uint32_t)load_entry(p + 2 * j) | (uint32_t)load_entry(p + 2 * j + 1) << 16;
            }
        }
#pragma unroll
        for (int k = 0; k < RULES_AHEAD; ++k) {
            const int u = u0 + k * THREADS;
            if (u >= whole || (INPLACE && allowed[k] == FULL)) continue;
            if (allowed[k] != FULL) G::keep(x[k], allowed[k], other);
            store_granule(out + first + u * N, x[k]);
        }
    }
    if (tid < ends) {
        const int e = tid < first ? tid : tid + whole * N;
        if (mask && !mask_bits(mask, v0 + e, 1)) out[e] = (typename G::Bits)other;
        else if (!INPLACE) out[e] = load_entry(in + e);
    }
}

// One sequence's rules, as the CTA keeps them for its slice [v0, v0 + n) of the rows [i0, i1)
struct RulesSlice {
    uint32_t* word;
    bool exact;                     // how often counts, not just whether
    unsigned short* bias_at;        // 1 + the entry's place in the list of biases, or 0
    int v0, n;

};

__device__ __forceinline__ void rules_count(const RulesSlice& s, int token, bool prompt) {
    const int e = token - s.v0;
    if ((unsigned)e >= (unsigned)s.n) return;
    // (most tokens come more than once: look before the atomic, where it may be spared)
    const uint32_t one = prompt ? RULES_PROMPT : 1u;
    if (!prompt && s.exact) atomicAdd(s.word + e, 1u);
    else if (!(*(volatile uint32_t*)(s.word + e) & one)) atomicOr(s.word + e, one);
}

// Reads `n` tokens with the whole CTA; returns whether any lies outside the vocabulary (per thread).
__device__ __forceinline__ bool rules_history(const RulesSlice& s, const int* tokens, int n, int prompt, int V, int tid) {
    bool bad = false;
    const int head = min(n, (int)((16 - ((uintptr_t)tokens & 15)) & 15) / 4), quads = (n - head) / 4;
    auto take = [&](int t, int at) {
        bad |= (unsigned)t >= (unsigned)V;
        rules_count(s, t, at < prompt);
    };
    const int rest = n - 4 * quads;             // before the first and behind the last quad
    if (tid < rest) {
        const int at = tid < head ? tid : tid + 4 * quads;
        take(__ldg(tokens + at), at);
    }
    constexpr int AHEAD = 4;
    const int4* q = reinterpret_cast<const int4*>(tokens + head);
    for (int k0 = tid; k0 < quads; k0 += AHEAD * THREADS) {
        int4 t[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (k0 + k * THREADS < quads) t[k] = __ldg(q + k0 + k * THREADS);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (k0 + k * THREADS < quads) {
                const int at = head + 4 * (k0 + k * THREADS);
                take(t[k].x, at); take(t[k].y, at + 1); take(t[k].z, at + 2); take(t[k].w, at + 3);
            }
    }
    return bad;
}

template <typename T, bool BACKWARD, bool INPLACE>
__global__ void __launch_bounds__(THREADS) rules_kernel(RulesArgs a) {
    using G = Granule<T>;
    using Bits = typename G::Bits;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int draft[RULES_ROWS], row_mask[RULES_ROWS], first_bad, listed;
    const int tid = threadIdx.x;
    const int slice = blockIdx.x % a.slices, block = blockIdx.x / a.slices % a.row_blocks, b = blockIdx.x / a.slices / a.row_blocks;
    const int i0 = block * a.row_block, i1 = min(a.R, i0 + a.row_block);
    RulesSlice s;
    s.v0 = slice * a.slice;
    s.n = min(a.slice, a.V - s.v0);
    s.word = reinterpret_cast<uint32_t*>(smem);
    unsigned short* list = reinterpret_cast<unsigned short*>(s.word + a.slice);
    s.bias_at = !BACKWARD && a.bias_idx ? list + a.slice : nullptr;
    const bool penalties = a.repetition || (!BACKWARD && (a.presence || a.frequency)), sparse = penalties || s.bias_at;
    if (sparse) {
        for (int i = tid; i < a.slice / 4; i += THREADS) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
        if (s.bias_at)
            for (int i = tid; i < a.slice / 8; i += THREADS) reinterpret_cast<uint4*>(s.bias_at)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (tid == 0) first_bad = a.R, listed = 0;
    grid_dependency_sync();
    // which row of the mask holds for each row: -1 none, -2 one that does not exist
    if (tid < i1 - i0) {
        const long long r = (long long)b * a.R + i0 + tid;
        int m = -1;
        if (a.mask) m = a.mask_row ? a.mask_row[r] : (int)r;
        row_mask[tid] = m < -1 || m >= a.mask_rows ? (a.mask ? -2 : -1) : m;
    }
    __syncthreads();

    // the rows, without what the sequence's own tokens and biases change
    const Bits* in = reinterpret_cast<const Bits*>(a.in) + ((long long)b * a.R + i0) * a.in_stride + s.v0;
    Bits* out = reinterpret_cast<Bits*>(a.out) + ((long long)b * a.R + i0) * a.out_stride + s.v0;
    for (int i = 0; i < i1 - i0; ++i) {
        const int m = row_mask[i];
        if (INPLACE && m < 0) continue;
        rules_row<T, INPLACE>(in + i * a.in_stride, out + i * a.out_stride, m >= 0 ? a.mask + m * a.mask_stride : nullptr, s.v0, s.n, BACKWARD ? 0u : G::LOWEST, tid);
    }

    // the sequence's numbers; `bad`: all of its rows are
    bool bad = false;
    double rho = 1.0, inverse = 1.0, presence = 0.0, frequency = 0.0;
    if (penalties) {
        if (a.repetition) rho = (double)a.repetition[b];
        if (!BACKWARD && a.presence) presence = (double)a.presence[b];
        if (!BACKWARD && a.frequency) frequency = (double)a.frequency[b];
        bad |= !(rho > 0.0 && rho < CUDART_INF) || !(fabs(presence) < CUDART_INF) || !(fabs(frequency) < CUDART_INF);
        inverse = 1.0 / rho;
        s.exact = frequency != 0.0;
        if (a.history) {
            const int length = a.length[b], prompt = a.prompt_length ? a.prompt_length[b] : 0;
            if (length < 0 || length > a.capacity || prompt < 0 || prompt > length) bad = true;
            else bad |= rules_history(s, a.history + b * a.history_stride, length, prompt, a.V, tid);
        }
        if (a.draft_tok) {
            const int* d = a.draft_tok + (long long)b * (a.R - 1);
            for (int j = tid; j < i1 - 1; j += THREADS) {
                const int t = __ldg(d + j), e = t - s.v0;
                if ((unsigned)t >= (unsigned)a.V) atomicMin(&first_bad, j);
                if (j < i0) rules_count(s, t, false);
                else {
                    draft[j - i0] = t;
                    if ((unsigned)e < (unsigned)s.n) atomicOr(s.word + e, RULES_DRAFT);
                }
            }
        }
    }
    if (s.bias_at) {
        const int k = a.bias_count[b];
        if (k < 0 || k > a.bias_k) bad = true;
        else {
            for (int j = tid; j < k; j += THREADS) {
                const int v = __ldg(a.bias_idx + (long long)b * a.bias_k + j), e = v - s.v0;
                bad |= (unsigned)v >= (unsigned)a.V || !(__ldg(a.bias + (long long)b * a.bias_k + j) < CUDART_INF_F);
                if ((unsigned)e < (unsigned)s.n) {
                    // of an entry that comes twice the last counts
                    unsigned short was = s.bias_at[e], seen;
                    while (was < j + 1 && (seen = atomicCAS(s.bias_at + e, was, (unsigned short)(j + 1))) != was) was = seen;
                    atomicOr(s.word + e, RULES_BIAS);
                }
            }
        }
    }
    bad = __syncthreads_or(bad);

    // rows without a value
    for (int i = 0; i < i1 - i0; ++i) {
        if (!bad && i0 + i <= first_bad && row_mask[i] >= -1) continue;
        if (tid == 0 && slice == 0) atomicOr(a.status, ST_RANGE);
        for (int e = tid; e < s.n; e += THREADS) out[i * a.out_stride + e] = (Bits)G::NOT;
    }
    if (bad || !sparse) return;

    // the entries that are concerned, one after the other, and each in every row
    for (int k = tid; k < a.slice / 4; k += THREADS) {      // (slice / 4 is a multiple of THREADS)
        const uint4 w = reinterpret_cast<const uint4*>(s.word)[k];
        const int own = (w.x != 0u) + (w.y != 0u) + (w.z != 0u) + (w.w != 0u);
        if (!__any_sync(0xffffffffu, own)) continue;
        int upto = own, base = 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, upto, d);
            if ((tid & 31) >= d) upto += y;
        }
        if ((tid & 31) == 31) base = atomicAdd(&listed, upto);
        base = __shfl_sync(0xffffffffu, base, 31) + upto - own;
        if (w.x) list[base++] = (unsigned short)(4 * k);
        if (w.y) list[base++] = (unsigned short)(4 * k + 1);
        if (w.z) list[base++] = (unsigned short)(4 * k + 2);
        if (w.w) list[base++] = (unsigned short)(4 * k + 3);
    }
    __syncthreads();
    const int count = listed, rows = min(i1, first_bad + 1) - i0, parts = (rows + RULES_AT_ONCE - 1) / RULES_AT_ONCE;
    for (int q = tid; q < count * parts; q += THREADS) {
        const int part = q / count, e = list[q - part * count], row0 = part * RULES_AT_ONCE;
        Bits x[RULES_AT_ONCE], l[RULES_AT_ONCE];
        uint32_t allowed = 0u;
#pragma unroll
        for (int k = 0; k < RULES_AT_ONCE; ++k) {
            const int m = row0 + k < rows ? row_mask[row0 + k] : -2;
            if (m == -1 || (m >= 0 && mask_bits(a.mask + m * a.mask_stride, s.v0 + e, 1))) allowed |= 1u << k;
        }
#pragma unroll
        for (int k = 0; k < RULES_AT_ONCE; ++k) {
            const int i = row0 + k;
            x[k] = allowed >> k & 1u ? load_entry(in + i * a.in_stride + e) : Bits(0);
            if (BACKWARD) l[k] = allowed >> k & 1u ? load_entry(reinterpret_cast<const Bits*>(a.logits) + ((long long)b * a.R + i0 + i) * a.logits_stride + s.v0 + e) : Bits(0);
            else l[k] = x[k];
        }
        const uint32_t word = s.word[e];
        const double bias = word & RULES_BIAS ? (double)__ldg(a.bias + (long long)b * a.bias_k + s.bias_at[e] - 1) : 0.0;
        int made = (int)(word & RULES_COUNT);
        if (word & RULES_DRAFT)
            for (int j = 0; j < row0; ++j) made += draft[j] == s.v0 + e;
#pragma unroll
        for (int k = 0; k < RULES_AT_ONCE; ++k) {
            if (k > 0 && (word & RULES_DRAFT) && row0 + k < rows) made += draft[row0 + k - 1] == s.v0 + e;
            if (!(allowed >> k & 1u)) continue;
            double y = (double)G::value(x[k]);
            if (made > 0 || (word & RULES_PROMPT)) y *= G::value(l[k]) > 0.0f ? inverse : rho;
            if (!BACKWARD) {
                if (made > 0) y = y - frequency * (double)made - presence;
                if (word & RULES_BIAS) y += bias;
            }
            out[(row0 + k) * a.out_stride + e] = G::round(y);
        }
    }
}

// ---- tokens behind the history ---------------------------------------------------------------

struct AppendArgs {
    int* history;               // [B, capacity]
    long long history_stride;
    int capacity, B, G;
    const int* length;          // [B]
    const int* draft_tok;       // [B, G] or null
    const int* accept_len;      // [B] or null (0)
    const int* token;           // [B] or null
    int* length_out;            // [B], may be `length`
    unsigned* status;
};

// A warp per sequence: every lane has read the length before it is written.  Bound by the launch.
__global__ void __launch_bounds__(THREADS) append_kernel(AppendArgs a) {
    grid_dependency_sync();
    const int lane = threadIdx.x & 31;
    const long long b = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (b >= a.B) return;
    const int length = a.length[b], accepted = a.accept_len ? a.accept_len[b] : 0, last = a.token ? a.token[b] : 0;
    const int n = accepted + (a.token ? 1 : 0);
    const int* d = a.draft_tok + b * a.G;
    bool bad = length < 0 || length > a.capacity || accepted > a.G || n > a.capacity - length || last < 0;
    if (!bad && accepted >= 0)
        for (int j = lane; j < accepted; j += 32) bad |= d[j] < 0;
    bad = __any_sync(0xffffffffu, bad) && accepted >= 0;
    const bool write = !bad && accepted >= 0;
    if (write) {
        int* h = a.history + b * a.history_stride + length;
        for (int j = lane; j < n; j += 32) h[j] = j < accepted ? d[j] : last;
    }
    if (lane == 0) {
        a.length_out[b] = write ? length + n : length;
        if (bad) atomicOr(a.status, ST_RANGE);
    }
}

}  // namespace picospec
