// Rules on rows of logits: penalties for tokens that a sequence holds already, biases, grammar masks; and their gradient.
//
//   c = occurrences of v among the tokens that the sequence made (history[prompt_length .. length), and the drafted tokens before the row)
//   s = c > 0, or v is in the prompt (history[0 .. prompt_length))
//   y = (s ? (l > 0 ? l / rho : l rho) : l) - frequency c - presence [c > 0] + bias_v;     -inf where the mask forbids v
//   dL/dl = dL/dy (s ? (l > 0 ? 1 / rho : rho) : 1);                                      0 where the mask forbids v
//
// A CTA takes a slice of the vocabulary of a few consecutive rows of one sequence.  It reads the sequence's history once and
// keeps, in shared memory, a word per entry of the slice (count, whether the prompt has it) and a bit per entry that any rule but
// the mask may change; the rows then stream past in granules of 16 bytes.  Nearly all granules have no such bit: they are copied, or
// in place not even read.  The others are computed in double precision, entry by entry, and rounded once: differences of penalty and
// logit may cancel, and there are few of them.
#pragma once
#include "common.cuh"

namespace picospec {

constexpr int RULES_SLICE = 8192;               // most vocabulary entries of a CTA
constexpr int RULES_SLICE_LEAST = 1024;         // fewest, where there are too few rows to fill the GPU
constexpr int RULES_ROWS = 16;                  // most rows of a CTA
constexpr int RULES_AHEAD = 4;                  // granules that a thread has on the way
constexpr uint32_t RULES_PROMPT = 1u << 30;     // word of an entry: the prompt has it,
constexpr uint32_t RULES_DRAFT = 1u << 31;      // a drafted token of the CTA's own rows is it,
constexpr uint32_t RULES_COUNT = (1u << 30) - 1;    // how often it was made before the CTA's first row

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

// shared memory: the words, the bits (one word more: a granule may look past the end), the biases' places
__host__ __device__ __forceinline__ int rules_smem(int slice, bool bias) { return slice * 4 + (slice / 32 + 4) * 4 + (bias ? slice * 2 : 0); }

// `n` bits from bit `at` of an array of words; `behind`: whether the word behind may be read too
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int at, int n) {
    const uint32_t lo = words[at >> 5], hi = (at & 31) + n > 32 ? words[(at >> 5) + 1] : 0u;
    return __funnelshift_r(lo, hi, at & 31) & ((1u << n) - 1u);
}
__device__ __forceinline__ uint32_t mask_bits(const int* words, int at, int n) {
    const uint32_t lo = (uint32_t)__ldg(words + (at >> 5)), hi = (at & 31) + n > 32 ? (uint32_t)__ldg(words + (at >> 5) + 1) : 0u;
    return __funnelshift_r(lo, hi, at & 31) & ((1u << n) - 1u);
}

// 16 bytes of logits: entries by number
template <typename T> struct Granule;
template <> struct Granule<float> {
    static constexpr int N = 4;
    static constexpr uint32_t LOWEST = 0xFF800000u, NOT = 0x7FC00000u;
    uint32_t w[4];
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(w[e]); }
    __device__ __forceinline__ void set(int e, double y) { w[e] = __float_as_uint((float)y); }
    __device__ __forceinline__ void put(int e, uint32_t pattern) { w[e] = pattern; }
    __device__ __forceinline__ void fill(uint32_t pattern) { w[0] = w[1] = w[2] = w[3] = pattern; }
};
template <> struct Granule<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t LOWEST = 0xFF80u, NOT = 0x7FC0u;
    uint32_t w[4];
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16); }
    __device__ __forceinline__ void put(int e, uint32_t pattern) {
        w[e >> 1] = e & 1 ? (w[e >> 1] & 0xFFFFu) | pattern << 16 : (w[e >> 1] & 0xFFFF0000u) | pattern;
    }
    __device__ __forceinline__ void set(int e, double y) { put(e, __bfloat16_as_ushort(__double2bfloat16(y))); }
    __device__ __forceinline__ void fill(uint32_t pattern) { w[0] = w[1] = w[2] = w[3] = pattern | pattern << 16; }
};
template <typename T> using Pattern = typename std::conditional<sizeof(T) == 2, unsigned short, uint32_t>::type;

// (not the read-only path: the call may work in place)
__device__ __forceinline__ void load_granule(uint32_t (&w)[4], const void* p) {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store_granule(void* p, const uint32_t (&w)[4]) {
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}

// One sequence's rules, as the CTA keeps them for its slice [v0, v0 + n) of the rows [i0, i1)
struct RulesSlice {
    uint32_t *word, *touched;
    unsigned short* bias_at;        // 1 + the entry's place in the list of biases, or 0
    const float* bias;
    const int* draft;               // shared: the drafted tokens of the CTA's own rows, from row i0 on
    double rho, inverse, presence, frequency;
    int v0, n;

    // How often entry e was made before the CTA's row `ahead` (rows counted from its first), and whether it was seen at all
    __device__ __forceinline__ void look(int e, int ahead, int& count, bool& seen) const {
        const uint32_t x = word[e];
        count = (int)(x & RULES_COUNT);
        if (x & RULES_DRAFT)
            for (int j = 0; j < ahead; ++j) count += draft[j] == v0 + e;
        seen = count > 0 || (x & RULES_PROMPT);
    }
    __device__ __forceinline__ double forward(int e, int ahead, float l) const {
        int count;
        bool seen;
        look(e, ahead, count, seen);
        double y = (double)l;
        if (seen) y *= l > 0.0f ? inverse : rho;
        if (count > 0) y = y - frequency * (double)count - presence;
        if (bias_at) {
            const int at = bias_at[e];
            if (at) y += (double)__ldg(bias + at - 1);
        }
        return y;
    }
    __device__ __forceinline__ double backward(int e, int ahead, float l, float g) const {
        int count;
        bool seen;
        look(e, ahead, count, seen);
        return seen ? (double)g * (l > 0.0f ? inverse : rho) : (double)g;
    }
};

__device__ __forceinline__ void rules_mark(const RulesSlice& s, int e) {
    // (most tokens come more than once: look before the atomic)
    if (!(*(volatile uint32_t*)(s.touched + (e >> 5)) >> (e & 31) & 1u)) atomicOr(s.touched + (e >> 5), 1u << (e & 31));
}
__device__ __forceinline__ void rules_count(const RulesSlice& s, int token, bool prompt) {
    const int e = token - s.v0;
    if ((unsigned)e >= (unsigned)s.n) return;
    if (!prompt) atomicAdd(s.word + e, 1u);
    else if (!(*(volatile uint32_t*)(s.word + e) & RULES_PROMPT)) atomicOr(s.word + e, RULES_PROMPT);
    rules_mark(s, e);
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
    constexpr int N = G::N;
    constexpr uint32_t FULL = (1u << N) - 1u;
    constexpr uint32_t FORBIDDEN = BACKWARD ? 0u : G::LOWEST;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int draft[RULES_ROWS], first_bad;
    const int tid = threadIdx.x;
    const int slice = blockIdx.x % a.slices, block = blockIdx.x / a.slices % a.row_blocks, b = blockIdx.x / a.slices / a.row_blocks;
    const int i0 = block * a.row_block, i1 = min(a.R, i0 + a.row_block);
    RulesSlice s;
    s.v0 = slice * a.slice;
    s.n = min(a.slice, a.V - s.v0);
    s.word = reinterpret_cast<uint32_t*>(smem);
    s.touched = s.word + a.slice;
    s.bias_at = !BACKWARD && a.bias_idx ? reinterpret_cast<unsigned short*>(s.touched + a.slice / 32 + 4) : nullptr;
    s.draft = draft;
    for (int i = tid; i < rules_smem(a.slice, s.bias_at != nullptr) / 16; i += THREADS) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) first_bad = a.R;
    __syncthreads();
    grid_dependency_sync();

    // the sequence's numbers; `bad`: all of its rows are
    bool bad = false;
    const float rho = a.repetition ? a.repetition[b] : 1.0f, presence = !BACKWARD && a.presence ? a.presence[b] : 0.0f, frequency = !BACKWARD && a.frequency ? a.frequency[b] : 0.0f;
    bad |= !(rho > 0.0f && rho < CUDART_INF_F) || !(fabsf(presence) < CUDART_INF_F) || !(fabsf(frequency) < CUDART_INF_F);
    s.rho = (double)rho;
    s.inverse = 1.0 / (double)rho;
    s.presence = (double)presence;
    s.frequency = (double)frequency;
    if (a.repetition || (!BACKWARD && (a.presence || a.frequency))) {
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
                    if ((unsigned)e < (unsigned)s.n) {
                        atomicOr(s.word + e, RULES_DRAFT);
                        rules_mark(s, e);
                    }
                }
            }
        }
    }
    if (s.bias_at) {
        const int k = a.bias_count[b];
        if (k < 0 || k > a.bias_k) bad = true;
        else {
            s.bias = a.bias + (long long)b * a.bias_k;
            for (int j = tid; j < k; j += THREADS) {
                const int v = __ldg(a.bias_idx + (long long)b * a.bias_k + j), e = v - s.v0;
                bad |= (unsigned)v >= (unsigned)a.V || !(__ldg(s.bias + j) < CUDART_INF_F);
                if ((unsigned)e < (unsigned)s.n) {
                    // of an entry that comes twice the last counts
                    unsigned short was = s.bias_at[e], seen;
                    while (was < j + 1 && (seen = atomicCAS(s.bias_at + e, was, (unsigned short)(j + 1))) != was) was = seen;
                    rules_mark(s, e);
                }
            }
        }
    }
    bad = __syncthreads_or(bad);

    for (int i = i0; i < i1; ++i) {
        const long long r = (long long)b * a.R + i;
        const T* in = reinterpret_cast<const T*>(a.in) + r * a.in_stride + s.v0;
        const T* logits = BACKWARD && a.logits ? reinterpret_cast<const T*>(a.logits) + r * a.logits_stride + s.v0 : nullptr;
        T* out = reinterpret_cast<T*>(a.out) + r * a.out_stride + s.v0;
        const int* mask = nullptr;
        bool row_bad = bad || i > first_bad;
        if (a.mask) {
            const long long m = a.mask_row ? (long long)a.mask_row[r] : r;
            if (m < -1 || m >= a.mask_rows) row_bad = true;
            else if (m >= 0) mask = a.mask + m * a.mask_stride;
        }
        if (row_bad && tid == 0 && slice == 0) atomicOr(a.status, ST_RANGE);
        // granules start on 16-byte boundaries of the output: the first and the last may be cut short
        const int lead = (int)((16 - ((uintptr_t)out & 15)) & 15) / (int)sizeof(T);
        const bool level = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
        const int start = lead ? lead - N : 0, units = (s.n - start + N - 1) / N;
        for (int u0 = tid; u0 < units; u0 += RULES_AHEAD * THREADS) {
            G x[RULES_AHEAD];
            uint32_t allowed[RULES_AHEAD], touched[RULES_AHEAD];
            // full granules: what there is to do, and the loads
#pragma unroll
            for (int k = 0; k < RULES_AHEAD; ++k) {
                const int e = start + (u0 + k * THREADS) * N;
                allowed[k] = FULL; touched[k] = 0u;
                if (e < 0 || e + N > s.n || row_bad) continue;
                if (mask) allowed[k] = mask_bits(mask, s.v0 + e, N);
                touched[k] = bits_at(s.touched, e, N) & allowed[k];
                if (allowed[k] == 0u || (INPLACE && allowed[k] == FULL && touched[k] == 0u)) continue;
                if (level) load_granule(x[k].w, in + e);
                else
#pragma unroll
                    for (int j = 0; j < N; ++j) x[k].put(j, reinterpret_cast<const volatile Pattern<T>*>(in + e)[j]);
            }
#pragma unroll
            for (int k = 0; k < RULES_AHEAD; ++k) {
                const int e = start + (u0 + k * THREADS) * N;
                if (e >= s.n) continue;
                if (e < 0 || e + N > s.n || row_bad) {          // cut short, or without a value
                    for (int j = max(0, -e); j < N && e + j < s.n; ++j) {
                        Pattern<T>* p = reinterpret_cast<Pattern<T>*>(out + e + j);
                        if (row_bad) *p = (Pattern<T>)G::NOT;
                        else if (mask && !mask_bits(mask, s.v0 + e + j, 1)) *p = (Pattern<T>)FORBIDDEN;
                        else {
                            const bool t = bits_at(s.touched, e + j, 1);
                            if (INPLACE && !t) continue;
                            G y;
                            y.put(0, *reinterpret_cast<const volatile Pattern<T>*>(in + e + j));
                            if (t) y.set(0, BACKWARD ? s.backward(e + j, i - i0, logits ? load_logit(logits, e + j) : 0.0f, y.get(0)) : s.forward(e + j, i - i0, y.get(0)));
                            *p = (Pattern<T>)(y.w[0] & (sizeof(T) == 2 ? 0xFFFFu : 0xFFFFFFFFu));
                        }
                    }
                    continue;
                }
                if (INPLACE && allowed[k] == FULL && touched[k] == 0u) continue;
                if (allowed[k] == 0u) x[k].fill(FORBIDDEN);
                else {
                    if (touched[k]) {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (touched[k] >> j & 1u)
                                x[k].set(j, BACKWARD ? s.backward(e + j, i - i0, logits ? load_logit(logits, e + j) : 0.0f, x[k].get(j)) : s.forward(e + j, i - i0, x[k].get(j)));
                    }
                    if (allowed[k] != FULL) {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (!(allowed[k] >> j & 1u)) x[k].put(j, FORBIDDEN);
                    }
                }
                store_granule(out + e, x[k].w);
            }
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
