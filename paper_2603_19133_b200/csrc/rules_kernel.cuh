// Rules on rows of logits: penalties for tokens that a sequence holds already, biases, grammar masks; and their gradient.
//
//   c = occurrences of v among the tokens that the sequence made (history[prompt_length .. length), and the drafted tokens before the row)
//   s = c > 0, or v is in the prompt (history[0 .. prompt_length))
//   y = (s ? (l > 0 ? l / rho : l rho) : l) - frequency c - presence [c > 0] + bias_v;     -inf where the mask forbids v
//   dL/dl = dL/dy (s ? (l > 0 ? 1 / rho : rho) : 1);                                      0 where the mask forbids v
//
// Two kernels.  The first, a cluster per sequence, reads the history and leaves the list of the entries that penalties and biases
// concern, in the order of the vocabulary, with their counts.  The second streams the rows, 8 KB of up to four rows of a sequence per CTA, and
// changes what the list and the masks say while they are in shared memory; in place only what the rules concern is touched.  Listed entries
// are computed in double precision and rounded once: penalty and logit may cancel, and they are few.
//
// What bounds it: HBM for many rows (256 x 7 rows of 128256 bf16 entries under three penalties: the second kernel takes 140 us, 6.6 TB/s, what a copy
// takes; both 157 us).  For few rows, or long histories (8 sequences of up to 100000 tokens: 50 to 55 us), the chain of barriers and L2 latencies of the
// first.  Before this split every CTA read the history for its slice of the vocabulary: 244 us and 91 us, and the CTA with the frequent tokens, which come
// first in a vocabulary, was the last to end.  Where histories are short and CTAs few that is still the shorter chain (1 x 1, 500 tokens: 6.7 us,
// with the first kernel 9.9), so there it stays (OWN below).
#pragma once
#include <type_traits>

#include "resident_row.cuh"

namespace picospec {

constexpr int RULES_PIECE = 8192;               // most bytes of a row that a CTA has in shared memory at a time: its slice of the vocabulary
constexpr int RULES_SEGMENT = 1024;             // entries per mark in the list; the fewest of a slice
constexpr int RULES_PLACE = 8192;               // entries of a slice in place, where nothing is staged
constexpr int RULES_ROWS = 4;                   // most rows of a CTA
constexpr int RULES_THREADS = 128;
constexpr int RULES_CHUNK = 512;                // listed entries of a CTA in place
constexpr int RULES_DRAFTED = 512;              // listed entries of a CTA whose drafted tokens are counted beforehand,
constexpr int RULES_FEW = 64;                   // if there are more than so many before the CTA's rows
constexpr int RULES_AHEAD = 4;                  // granules that a thread has on the way
constexpr int RULES_TOKENS = 8;                 // tokens that a thread of the second kernel has on the way
constexpr int RULES_QUADS = 2;                  // times four tokens that a thread has on the way, and as many behind them
constexpr int RULES_OWN = 4096;                 // most tokens of a sequence that the CTAs of the rows read themselves
constexpr int RULES_LIST_THREADS = 512;
constexpr int RULES_LIST_TWO = 112 << 10;       // shared memory of the first kernel up to which an SM has two CTAs
constexpr int RULES_PART = 1 << 19;             // vocabulary entries that the first kernel takes together
constexpr int RULES_WORDS = 24576;              // listed entries that it takes together
constexpr int RULES_SHARE = 2048;               // tokens that are worth a CTA of their own
constexpr uint32_t RULES_PROMPT = 1u << 30;     // word of a listed entry: the prompt has it,
constexpr uint32_t RULES_DRAFT = 1u << 31;      // a drafted token is it,
constexpr uint32_t RULES_BIAS = 1u << 29;       // it has a bias,
constexpr uint32_t RULES_COUNT = (1u << 29) - 1;    // how often it was made (2^27 in the history and as many drafts at most)

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
    unsigned long long wait_limit_ns;
    // the list (null without penalties and biases): per sequence [head] words, [most] entries and their biases' places (1 + it, or 0)
    int* heads;                 // 0: all rows are bad; 1: the first drafted token that is; then the first place in the list of each segment, and the end
    uint2* entries;             // (entry, word), in the order of the entries
    int* bias_at;
    int head;
    int most;
    int words;                  // the first kernel: words that its shared memory has
    int slice, slices, row_block, row_blocks;
    int first_ctas;             // CTAs of the second kernel that may start while the first runs
};

__host__ __device__ __forceinline__ int rules_head(int V) { return 2 + (V + RULES_SEGMENT - 1) / RULES_SEGMENT + 1; }
__host__ __device__ __forceinline__ int rules_bits(int V) { return ((V < RULES_PART ? V : RULES_PART) + 31) / 32; }

// `n` bits of an array of words from bit `at` on
__device__ __forceinline__ uint32_t bits_of(const uint32_t* words, int at, int n) {
    const uint32_t lo = words[at >> 5], hi = (at & 31) + n > 32 ? words[(at >> 5) + 1] : 0u;
    return __funnelshift_r(lo, hi, at & 31) & ((1u << n) - 1u);
}

// How the entries lie in a granule of 16 bytes
template <typename T> struct Granule;
template <> struct Granule<float> {
    static constexpr int N = 4;
    static constexpr uint32_t LOWEST = 0xFF800000u, NOT = 0x7FC00000u;      // -inf, NaN
    using Bits = uint32_t;
    static __device__ __forceinline__ float value(Bits x) { return __uint_as_float(x); }
    static __device__ __forceinline__ Bits round(double y) { return __float_as_uint((float)y); }
};
template <> struct Granule<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t LOWEST = 0xFF80u, NOT = 0x7FC0u;
    using Bits = unsigned short;
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
// shared -> global, whole granules, and the groups of such copies that one thread has under way
__device__ __forceinline__ void bulk_store(void* dst_gmem, const void* src_smem, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst_gmem), "r"(smem_addr(src_smem)), "r"(bytes) : "memory");
}
// global -> L2, whole granules: a hint that no one waits for
__device__ __forceinline__ void bulk_prefetch(const void* src_gmem, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src_gmem), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
template <typename B> __device__ __forceinline__ B load_entry(const B* p) { return *reinterpret_cast<const volatile B*>(p); }

// What lies before the first and behind the last whole granule of a row's part, by a warp.  `mask`: the words of the row's mask from the
// slice's first entry on, or null.
template <typename T, bool INPLACE>
__device__ __forceinline__ void rules_ends(const typename Granule<T>::Bits* in, typename Granule<T>::Bits* out, const uint32_t* mask, int first, int whole, int n, uint32_t other, int lane) {
    constexpr int N = Granule<T>::N;
    if (lane >= n - whole * N) return;
    const int e = lane < first ? lane : lane + whole * N;
    if (mask && !bits_of(mask, e, 1)) out[e] = (typename Granule<T>::Bits)other;
    else if (!INPLACE) out[e] = load_entry(in + e);
}

// `other` where a granule's mask forbids an entry: the granule at once, or entry by entry, so that nothing has to be read and other threads
// may write the entries that are allowed
template <typename T> __device__ __forceinline__ void rules_forbid(typename Granule<T>::Bits* p, uint32_t forbidden, uint32_t other) {
    constexpr int N = Granule<T>::N;
    if (forbidden == (1u << N) - 1u) {
        const uint32_t w = sizeof(T) == 2 ? other * 0x10001u : other;
        *reinterpret_cast<uint4*>(p) = make_uint4(w, w, w, w);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (forbidden >> j & 1u) p[j] = (typename Granule<T>::Bits)other;
    }
}

// The whole granules of a row's part, by the CTA's threads.  In place only what the mask forbids is written.
template <typename T, bool INPLACE>
__device__ __forceinline__ void rules_row(const typename Granule<T>::Bits* in, typename Granule<T>::Bits* out, const uint32_t* mask, int first, int whole, uint32_t other, int tid) {
    constexpr int N = Granule<T>::N;
    constexpr uint32_t FULL = (1u << N) - 1u;
    const bool level = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
    for (int u0 = tid; u0 < whole; u0 += RULES_AHEAD * RULES_THREADS) {
        uint32_t x[RULES_AHEAD][4], forbidden[RULES_AHEAD];
#pragma unroll
        for (int k = 0; k < RULES_AHEAD; ++k) {
            const int u = u0 + k * RULES_THREADS;
            forbidden[k] = u < whole && mask ? bits_of(mask, first + u * N, N) ^ FULL : 0u;
        }
        if (!INPLACE) {
#pragma unroll
            for (int k = 0; k < RULES_AHEAD; ++k) {
                const auto* p = in + first + (u0 + k * RULES_THREADS) * N;
                if (u0 + k * RULES_THREADS >= whole || forbidden[k] == FULL) continue;
                if (level) load_granule(x[k], p);
                else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        x[k][j] = sizeof(T) == 4 ? (uint32_t)load_entry(p + j) : (uint32_t)load_entry(p + 2 * j) | (uint32_t)load_entry(p + 2 * j + 1) << 16;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < RULES_AHEAD; ++k) {
            auto* p = out + first + (u0 + k * RULES_THREADS) * N;
            if (!INPLACE && u0 + k * RULES_THREADS < whole && forbidden[k] != FULL) store_granule(p, x[k]);
            if (forbidden[k]) rules_forbid<T>(p, forbidden[k], other);
        }
    }
}

// The place of a vocabulary entry in a list that is in their order, or -1.
__device__ __forceinline__ int rules_find(const uint2* list, int count, int entry) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int)list[mid].x <= entry) lo = mid;
        else hi = mid;
    }
    return count > 0 && (int)list[lo].x == entry ? lo : -1;
}

// ---- the list -------------------------------------------------------------------------------------
// A bit per vocabulary entry, the number of bits before each word of them, and a word per entry whose bit is set: the place of an entry in the
// list is a count of bits, so nothing is sorted and the list does not depend on the order of execution.

// Tokens as a CTA reads them: the first quads of each thread are kept for the second time.
struct RulesTokens {
    const int* tokens;
    int4 kept[RULES_QUADS];
    __device__ __forceinline__ static int head_of(const int* p) { return (int)((16 - ((uintptr_t)p & 15)) & 15) / 4; }
    // `capacity`: tokens that may be read from `p` on, whether they count or not
    __device__ __forceinline__ void start(const int* p, int capacity) {
        tokens = p;
        load(kept, threadIdx.x, (capacity - head_of(p)) / 4);
    }
    __device__ __forceinline__ void load(int4 (&t)[RULES_QUADS], int at, int quads) const {
        const int4* q = reinterpret_cast<const int4*>(tokens + head_of(tokens));
#pragma unroll
        for (int k = 0; k < RULES_QUADS; ++k)
            if (at + k * RULES_LIST_THREADS < quads) t[k] = __ldg(q + at + k * RULES_LIST_THREADS);
    }
    // f(Few, place of the first) for the first `n`, by the whole CTA; the next loads are under way meanwhile
    template <int K> struct Few {
        static constexpr int COUNT = K;
        int t[K];
    };
    template <typename F> __device__ __forceinline__ void each(int n, F&& f) const {
        constexpr int NT = RULES_LIST_THREADS;
        const int tid = threadIdx.x, head = min(n, head_of(tokens)), quads = (n - head) / 4;
        const int rest = n - 4 * quads;             // before the first and behind the last quad
        if (tid < rest) {
            const int at = tid < head ? tid : tid + 4 * quads;
            f(Few<1>{{__ldg(tokens + at)}}, at);
        }
        int4 t[RULES_QUADS];
#pragma unroll
        for (int k = 0; k < RULES_QUADS; ++k) t[k] = kept[k];
        for (int q0 = tid; q0 < quads; q0 += RULES_QUADS * NT) {
            int4 next[RULES_QUADS];
            load(next, q0 + RULES_QUADS * NT, quads);
#pragma unroll
            for (int k = 0; k < RULES_QUADS; ++k) {
                if (q0 + k * NT < quads) f(Few<4>{{t[k].x, t[k].y, t[k].z, t[k].w}}, head + 4 * (q0 + k * NT));
                t[k] = next[k];
            }
        }
    }
};

__device__ __forceinline__ uint32_t peer_load(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// A cluster per sequence: its CTAs share the tokens of the history, put their bits together, count each for itself, and each adds up and writes a part
// of the list.  Drafted tokens and biases are the first CTA's.  Counting in a CTA's own words first keeps the frequent tokens' atomics apart: those of
// one CTA that owns them all took most of the time.  About ten barriers of 0.5 to 1 us, four of the cluster; one CTA per sequence with 4000 tokens
// takes 18 us cold, sixteen with 100000 take 37.
__global__ void __launch_bounds__(RULES_LIST_THREADS, 2) rules_list_kernel(RulesArgs a) {
    constexpr int NT = RULES_LIST_THREADS;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int warp_bits[NT / 32], first_bad;
    __shared__ uint32_t any_bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t ranks;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    const uint32_t rank = cluster_rank();
    const int b = blockIdx.x / ranks;
    const int words = rules_bits(a.V);
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem);
    uint32_t* before = bits + words;
    uint32_t* word = before + words;
    if (tid == 0) first_bad = a.R, any_bad = 0u;
    __syncthreads();
    cluster_arrive();
    grid_dependency_sync();
    const bool penalties = a.repetition || a.presence || a.frequency, counted = penalties && a.history;
    const int length = counted ? __ldg(a.length + b) : 0, prompt = counted && a.prompt_length ? __ldg(a.prompt_length + b) : 0;
    const float rho = a.repetition ? __ldg(a.repetition + b) : 1.0f, presence = a.presence ? __ldg(a.presence + b) : 0.0f, frequency = a.frequency ? __ldg(a.frequency + b) : 0.0f;
    const int given = a.bias_idx ? __ldg(a.bias_count + b) : 0;
    const int* drafts = penalties && a.draft_tok ? a.draft_tok + (long long)b * (a.R - 1) : nullptr;
    const int* bias_idx = a.bias_idx + (long long)b * a.bias_k;
    const int drafted = drafts && rank == 0 ? a.R - 1 : 0, biased = rank == 0 ? given : 0;
    int* head = a.heads + (long long)b * a.head;
    uint2* entries = a.entries + (long long)b * a.most;
    int* bias_at = a.bias_at + (long long)b * a.most;
    bool bad = !(rho > 0.0f && rho < CUDART_INF_F) || !(fabsf(presence) < CUDART_INF_F) || !(fabsf(frequency) < CUDART_INF_F);
    bad |= length < 0 || length > a.capacity || prompt < 0 || prompt > length || given < 0 || given > a.bias_k;
    // this CTA's tokens, a multiple of four of them; where it has all of them they are on the way before their number is known
    RulesTokens tokens{};
    const int all = ranks == 1 ? a.capacity : min(max(length, 0), a.capacity);
    const int share = ((all + (int)ranks - 1) / (int)ranks + 3) / 4 * 4, t0 = min(all, (int)rank * share);
    if (counted) tokens.start(a.history + b * a.history_stride + t0, min(share, all - t0));
    for (int i = tid; i < words; i += NT) bits[i] = 0u;
    cluster_wait();
    if (bad) {                                  // (the same in every thread of the cluster)
        if (rank == 0 && tid == 0) head[0] = 1;
        return;
    }
    const int mine_tokens = max(0, min(share, length - t0));
    int base = 0;                               // listed so far
    for (int v0 = 0; v0 < a.V; v0 += RULES_PART) {
        const int n = min(RULES_PART, a.V - v0), own = (n + 31) / 32;
        for (int i = tid; v0 > 0 && i < own; i += NT) bits[i] = 0u;
        __syncthreads();
        // which entries.  Most tokens come more than once: bits are looked at before they are set, those of several tokens together.
        auto mark = [&](const auto& few) {
            constexpr int K = std::decay_t<decltype(few)>::COUNT;
            bool good = true, set[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const unsigned e = (unsigned)(few.t[k] - v0);
                good &= (unsigned)few.t[k] < (unsigned)a.V;
                set[k] = e < (unsigned)n && !(bits[e >> 5] >> (e & 31) & 1u);
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (set[k]) atomicOr(bits + ((unsigned)(few.t[k] - v0) >> 5), 1u << ((few.t[k] - v0) & 31));
            return good;
        };
        using One = RulesTokens::Few<1>;
        tokens.each(mine_tokens, [&](const auto& few, int) { bad |= !mark(few); });
        for (int j = tid; j < drafted; j += NT)
            if (!mark(One{{__ldg(drafts + j)}})) atomicMin(&first_bad, j);
        for (int j = tid; j < biased; j += NT) bad |= !mark(One{{__ldg(bias_idx + j)}}) || !(__ldg(a.bias + (long long)b * a.bias_k + j) < CUDART_INF_F);
        bad = __syncthreads_or(bad);
        if (ranks > 1) {
            if (bad && tid < (int)ranks) peer_store(peer_addr(&any_bad, tid), 1u);
            cluster_sync();
            bad = any_bad != 0u;
            // a part of the words each, from all CTAs to all
            if (!bad)
                for (int w = (int)rank * NT + tid; w < own; w += (int)ranks * NT) {
                    uint32_t x = 0u;
                    for (uint32_t k = 0; k < ranks; ++k) x |= peer_load(peer_addr(bits + w, k));
                    for (uint32_t k = 0; k < ranks; ++k) peer_store(peer_addr(bits + w, k), x);
                }
            cluster_sync();
        }
        if (bad) {
            if (rank == 0 && tid == 0) head[0] = 1;
            return;
        }
        // how many before each word: a warp has consecutive words
        const int per = (own + NT - 1) / NT * 32, w0 = min(own, warp * per), w1 = min(own, w0 + per);
        int mine = 0;
        for (int w = w0 + lane; w < w1; w += 32) mine += __popc(bits[w]);
        mine = warp_sum(mine);
        if (lane == 0) warp_bits[warp] = mine;
        __syncthreads();
        int total = 0, at = 0;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) {
            if (w < warp) at += warp_bits[w];
            total += warp_bits[w];
        }
        for (int w = w0; w < w1; w += 32) {
            const int own_bits = w + lane < w1 ? __popc(bits[w + lane]) : 0;
            int upto = own_bits;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += y;
            }
            if (w + lane < w1) before[w + lane] = (uint32_t)(at + upto - own_bits);
            at += __shfl_sync(0xffffffffu, upto, 31);
        }
        __syncthreads();
        if (rank == 0)
            for (int i = tid; i < (n + RULES_SEGMENT - 1) / RULES_SEGMENT; i += NT) head[2 + v0 / RULES_SEGMENT + i] = base + (int)before[i * (RULES_SEGMENT / 32)];
        // their words, as many as there is room for at a time
        for (int p0 = 0; p0 < total; p0 += a.words) {
            const int room = min(a.words, total - p0);
            for (int i = tid; i < room; i += NT) word[i] = 0u;
            __syncthreads();
            auto place = [&](int t) {           // -1: not here
                const unsigned e = (unsigned)(t - v0);
                if ((unsigned)t >= (unsigned)a.V || e >= (unsigned)n) return -1;
                const int p = (int)before[e >> 5] + __popc(bits[e >> 5] & ((1u << (e & 31)) - 1u)) - p0;
                return (unsigned)p < (unsigned)room ? p : -1;
            };
            auto set = [&](int p, uint32_t bit) {
                if (p >= 0 && !(word[p] & bit)) atomicOr(word + p, bit);
            };
            const bool exact = frequency != 0.0f;       // (else only whether it was made matters)
            tokens.each(mine_tokens, [&](const auto& few, int i) {
                constexpr int K = std::decay_t<decltype(few)>::COUNT;
                int p[K];
#pragma unroll
                for (int k = 0; k < K; ++k) p[k] = place(few.t[k]);
                if (exact && t0 + i >= prompt) {
#pragma unroll
                    for (int k = 0; k < K; ++k)
                        if (p[k] >= 0) atomicAdd(word + p[k], 1u);
                } else {
                    uint32_t bit[K];
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const bool made = t0 + i + k >= prompt;
                        bit[k] = p[k] < 0 ? 0u : made ? 1u : RULES_PROMPT;
                        if (p[k] >= 0 && !(made && exact) && (word[p[k]] & bit[k])) bit[k] = 0u;
                    }
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        if (!bit[k]) continue;
                        if (bit[k] == 1u && exact) atomicAdd(word + p[k], 1u);
                        else atomicOr(word + p[k], bit[k]);
                    }
                }
            });
            for (int j = tid; j < drafted; j += NT) set(place(__ldg(drafts + j)), RULES_DRAFT);
            for (int j = tid; j < biased; j += NT) set(place(__ldg(bias_idx + j)), RULES_BIAS);
            if (ranks > 1) cluster_sync();
            else __syncthreads();
            // this CTA's part of the places
            const int part = (room + (int)ranks - 1) / (int)ranks, q0 = min(room, (int)rank * part), q1 = min(room, q0 + part);
            for (int p = q0 + tid; p < q1; p += NT) {
                // the word whose bits reach over the place, and the bit
                int lo = 0, hi = own, left;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if ((int)before[mid] <= p0 + p) lo = mid;
                    else hi = mid;
                }
                left = p0 + p - (int)before[lo];
                uint32_t x = bits[lo], at_bit = 0u;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) {
                    const int low = __popc(x & ((1u << d) - 1u));
                    if (left >= low) left -= low, x >>= d, at_bit += d;
                }
                uint32_t y = word[p];
                if (ranks > 1) {
                    uint32_t flags = 0u, count = 0u;
#pragma unroll 8
                    for (uint32_t k = 0; k < ranks; ++k) {
                        const uint32_t z = peer_load(peer_addr(word + p, k));
                        flags |= z & ~RULES_COUNT;
                        count += z & RULES_COUNT;
                    }
                    y = flags | count;
                }
                entries[base + p0 + p] = make_uint2((uint32_t)(v0 + lo * 32) + at_bit, y);
                if (given) bias_at[base + p0 + p] = 0;
            }
            // of an index that comes twice the last counts
            if (given) {
                __syncthreads();
                for (int j = tid; j < given; j += NT) {
                    const int p = place(__ldg(bias_idx + j));
                    if (p >= q0 && p < q1) atomicMax(bias_at + base + p0 + p, j + 1);
                }
            }
            if (ranks > 1) cluster_sync();      // (nobody's words go while a peer may read them)
            else __syncthreads();
        }
        base += total;
    }
    if (rank == 0 && tid == 0) {
        head[0] = 0;
        head[1] = first_bad;
        head[2 + (a.V + RULES_SEGMENT - 1) / RULES_SEGMENT] = base;
    }
}

// ---- the rows ------------------------------------------------------------------------------------
// Pieces of rows pass through shared memory by bulk copies, and the CTA's threads only change what the rules change: no registers and few instructions
// per entry.  A CTA has up to four pieces, all at once: a ring of three with a barrier per
// row took 182 us where this takes 159 (256 x 7), pieces of two or three rows 166 and 164, 256 threads 184.  Rows of which the mask leaves little are
// filled and the few entries fetched; rows whose input and output lie differently on 16-byte boundaries are written by the threads.  In place the threads
// write what the masks forbid, entry by entry, without reading, and each CTA takes an equal part of the list (512 entries), wherever it lies (512 x 1 rows
// of 262144 under masks: 60 us; filling them takes 74).
// With a list this kernel's CTAs start while the one above runs, but that it waited for the kernels before it says nothing of what this one sees
// of them: nothing is read or written ahead of this kernel's own wait, the rows are only asked into L2 (256 x 7 157 us, without 159).  Not under
// masks, which say that some rows are not read (64 x 8 gradient 82 us with and without).
//
// OWN: without the first kernel.  The CTA reads the history itself and has a word for every entry of its slice, and a list of those whose word is not 0.
// That is repeated for every slice and block of rows, and shorter where both are few.
template <typename T, bool BACKWARD, bool INPLACE, bool OWN>
__global__ void __launch_bounds__(RULES_THREADS, OWN ? 6 : 8) rules_kernel(RulesArgs a) {
    using G = Granule<T>;
    using Bits = typename G::Bits;
    constexpr int N = G::N, NT = RULES_THREADS, MASK = RULES_PIECE / (int)sizeof(T) / 32 + 1;
    constexpr uint32_t OTHER = BACKWARD ? 0u : G::LOWEST;
    extern __shared__ __align__(128) unsigned char smem[];
    // of each row: drafted token, row of the mask (-1 none, -2 one that does not exist), where its whole granules begin, how many there are,
    // whether it passes through shared memory, whether its mask leaves little
    __shared__ int draft[RULES_ROWS], row_mask[RULES_ROWS], row_first[RULES_ROWS], row_whole[RULES_ROWS];
    __shared__ bool staged[RULES_ROWS], tight[RULES_ROWS];
    __shared__ uint32_t mask_words[INPLACE ? 1 : RULES_ROWS][MASK];
    __shared__ int drafted[INPLACE || OWN ? RULES_FEW : RULES_DRAFTED];
    __shared__ int first_bad, listed;
    __shared__ uint64_t bar;
    const int tid = threadIdx.x, lane = tid & 31;
    const int slice = blockIdx.x % a.slices, block = blockIdx.x / a.slices % a.row_blocks, b = blockIdx.x / a.slices / a.row_blocks;
    const int i0 = block * a.row_block, rows = min(a.R, i0 + a.row_block) - i0;
    // (in place the CTAs behind the vocabulary's slices have a part of the list alone)
    const bool listed_alone = INPLACE && !OWN && (long long)slice * a.slice >= a.V;
    const int v0 = listed_alone ? 0 : slice * a.slice, n = listed_alone ? 0 : min(a.slice, a.V - v0);
    const int stage_bytes = a.slice * (int)sizeof(T);
    const bool sparse = OWN || a.heads;
    uint32_t* own_word = reinterpret_cast<uint32_t*>(smem + (INPLACE ? 0 : a.row_block * stage_bytes));        // OWN: a word per entry,
    unsigned short* own_bias = reinterpret_cast<unsigned short*>(own_word + a.slice);                          // 1 + its place in the biases,
    unsigned short* own_list = own_bias + (!BACKWARD && a.bias_idx ? a.slice : 0);                             // and the list
    if (OWN) {
        const int words = a.slice / 4 + (!BACKWARD && a.bias_idx ? a.slice / 8 : 0);
        for (int i = tid; i < words; i += NT) reinterpret_cast<uint4*>(own_word)[i] = make_uint4(0u, 0u, 0u, 0u);
        if (tid == 0) first_bad = a.R, listed = 0;
    }
    const Bits* in = reinterpret_cast<const Bits*>(a.in) + ((long long)b * a.R + i0) * a.in_stride + v0;
    Bits* out = reinterpret_cast<Bits*>(a.out) + ((long long)b * a.R + i0) * a.out_stride + v0;
    const Bits* signs = BACKWARD && a.logits ? reinterpret_cast<const Bits*>(a.logits) + ((long long)b * a.R + i0) * a.logits_stride + v0 : nullptr;
    auto level = [&](int i) { return (((uintptr_t)(in + i * a.in_stride) ^ (uintptr_t)(out + i * a.out_stride)) & 15) == 0; };
    auto first_of = [&](int i) { return min(n, (int)((16 - ((uintptr_t)(out + i * a.out_stride) & 15)) & 15) / (int)sizeof(T)); };
    // Ahead of the wait nothing is read or written: while the list is put together the rows are only asked into L2, by the CTAs that start at once
    if (!INPLACE && !OWN && sparse && !a.mask && blockIdx.x < (unsigned)a.first_ctas && tid < rows && level(tid)) {
        const int first = first_of(tid), bytes = (n - first) / N * 16;
        if (bytes) bulk_prefetch(in + tid * a.in_stride + first, (uint32_t)bytes);
    }
    grid_dependency_sync();
    const int* head = sparse && !OWN ? a.heads + (long long)b * a.head : nullptr;
    const int seg0 = 2 + (INPLACE ? 0 : v0 / RULES_SEGMENT), seg1 = 2 + ((INPLACE ? a.V : v0 + n) + RULES_SEGMENT - 1) / RULES_SEGMENT;
    int state = 0, bad_draft = a.R, from = 0, to = 0;           // the list's part: [from, to)
    if (head) state = head[0], bad_draft = head[1], from = head[seg0], to = head[seg1];
    // OWN: the sequence's numbers and each thread's first tokens are on the way while the masks are looked at
    double rho = 1.0, inverse = 1.0, presence = 0.0, frequency = 0.0;
    const bool counted = OWN && a.history && (a.repetition || a.presence || a.frequency);
    const int* history = counted ? a.history + b * a.history_stride : nullptr;
    int length = 0, prompt = 0, given = 0, tokens[RULES_TOKENS];
    if (OWN) {
        if (counted) {
            length = __ldg(a.length + b);
            if (a.prompt_length) prompt = __ldg(a.prompt_length + b);
#pragma unroll
            for (int k = 0; k < RULES_TOKENS; ++k) tokens[k] = tid + k * NT < a.capacity ? __ldg(history + tid + k * NT) : 0;
        }
        if (!BACKWARD && a.bias_idx) given = __ldg(a.bias_count + b);
    }
    if (!INPLACE && tid == 0) {
        mbar_init(&bar, rows);
        mbar_init_fence();
    }
    auto mask_of = [&](int i) {                 // the words of row i's mask from entry v0 on, or null
        if (row_mask[i] < 0) return (const uint32_t*)nullptr;
        return INPLACE ? reinterpret_cast<const uint32_t*>(a.mask) + row_mask[i] * a.mask_stride + v0 / 32 : (const uint32_t*)mask_words[INPLACE ? 0 : i];
    };
    bool plain = true;                          // nothing is left to the threads of the rows that this warp looked at
    for (int i = tid >> 5; i < rows; i += NT / 32) {
        const long long r = (long long)b * a.R + i0 + i;
        int m = -1;
        if (a.mask) m = a.mask_row ? a.mask_row[r] : (int)r;
        if (a.mask && (m < -1 || m >= a.mask_rows)) m = -2;
        bool little = false;
        if (!INPLACE && m >= 0) {
            // where a mask allows an entry in 64 at most, the row is filled and the allowed entries are fetched one by one (512 rows of 151936: 45 us;
            // read, masked and written 54)
            int some = 0;
            const int words = (n + 31) / 32, there = (a.V + 31) / 32 - v0 / 32;
            for (int w = lane; w < min(words + 1, there); w += 32) {
                const uint32_t x = (uint32_t)__ldg(a.mask + m * a.mask_stride + v0 / 32 + w);
                mask_words[INPLACE ? 0 : i][w] = x;
                if (w < words) some += __popc(w * 32 + 32 <= n ? x : x & ((1u << (n & 31)) - 1u));
            }
            little = 64 * warp_sum(some) <= n;
        }
        const bool through = !INPLACE && !little && level(i);
        const int first = first_of(i), whole = (n - first) / N;
        if (lane == 0) row_mask[i] = m, row_first[i] = first, row_whole[i] = whole, staged[i] = through, tight[i] = little;
        plain &= through && whole * N == n;
    }
    const bool by_threads = __syncthreads_or(!plain);

    if (!INPLACE && tid < rows) {               // a thread per row: its copy
        const uint32_t bytes = staged[tid] ? (uint32_t)row_whole[tid] * 16u : 0u;
        if (bytes) {
            mbar_expect_tx(&bar, bytes);
            bulk_load(smem + tid * stage_bytes, in + tid * a.in_stride + row_first[tid], bytes, &bar, l2_evict_first_policy());
        }
        mbar_arrive(&bar);
    }
    const int* drafts = sparse && a.draft_tok ? a.draft_tok + (long long)b * (a.R - 1) : nullptr;
    if (sparse) {
        if (a.repetition) rho = (double)__ldg(a.repetition + b);
        if (!BACKWARD && a.presence) presence = (double)__ldg(a.presence + b);
        if (!BACKWARD && a.frequency) frequency = (double)__ldg(a.frequency + b);
        if (drafts && tid < rows - 1) draft[tid] = __ldg(drafts + i0 + tid);
    }
    if (OWN) {
        bool bad = !(rho > 0.0 && rho < CUDART_INF) || !(fabs(presence) < CUDART_INF) || !(fabs(frequency) < CUDART_INF);
        auto push = [&](int e) { own_list[atomicAdd(&listed, 1)] = (unsigned short)e; };
        auto set = [&](int e, uint32_t bit) {
            if (!(*(volatile uint32_t*)(own_word + e) & bit) && atomicOr(own_word + e, bit) == 0u) push(e);
        };
        auto add = [&](int e) {
            if (atomicAdd(own_word + e, 1u) == 0u) push(e);
        };
        if (length < 0 || length > a.capacity || prompt < 0 || prompt > length) bad = true;
        else
            for (int k0 = tid; k0 < length; k0 += RULES_TOKENS * NT) {
#pragma unroll
                for (int k = 0; k < RULES_TOKENS; ++k) {
                    if (k0 + k * NT >= length) continue;
                    bad |= (unsigned)tokens[k] >= (unsigned)a.V;
                    if ((unsigned)(tokens[k] - v0) >= (unsigned)n) continue;
                    if (k0 + k * NT < prompt) set(tokens[k] - v0, RULES_PROMPT);
                    else add(tokens[k] - v0);
                }
#pragma unroll
                for (int k = 0; k < RULES_TOKENS; ++k) {
                    const int at = k0 + (RULES_TOKENS + k) * NT;
                    if (at < length) tokens[k] = __ldg(history + at);
                }
            }
        for (int j = tid; drafts && j < i0 + rows - 1; j += NT) {
            const int t = __ldg(drafts + j);
            if ((unsigned)t >= (unsigned)a.V) atomicMin(&first_bad, j);
            if ((unsigned)(t - v0) >= (unsigned)n) continue;
            if (j < i0) add(t - v0);
            else set(t - v0, RULES_DRAFT);
        }
        if (given < 0 || given > a.bias_k) bad = true;
        else
            for (int j = tid; j < given; j += NT) {
                const int t = __ldg(a.bias_idx + (long long)b * a.bias_k + j), e = t - v0;
                bad |= (unsigned)t >= (unsigned)a.V || !(__ldg(a.bias + (long long)b * a.bias_k + j) < CUDART_INF_F);
                if ((unsigned)e >= (unsigned)n) continue;
                // of an index that comes twice the last counts
                unsigned short was = own_bias[e], seen;
                while (was < j + 1 && (seen = atomicCAS(own_bias + e, was, (unsigned short)(j + 1))) != was) was = seen;
                set(e, RULES_BIAS);
            }
        state = __syncthreads_or(bad);
        bad_draft = first_bad, to = listed;
    } else if (sparse) {
        // drafted tokens before the CTA's rows: some by themselves, many counted for the list's first entries
        for (int q = tid; i0 > RULES_FEW && !INPLACE && q < RULES_DRAFTED; q += NT) drafted[q] = 0;
        if (drafts && i0 <= RULES_FEW && tid < i0) drafted[tid] = __ldg(drafts + tid);
        if (INPLACE) from = min(slice * RULES_CHUNK, to), to = min(to, from + RULES_CHUNK);        // an equal part, wherever it lies
    }
    const uint2* list = a.entries + (long long)b * a.most + from;
    uint2 mine = make_uint2(0u, 0u);            // the thread's next entry, on the way
    if (sparse && !OWN && state == 0 && tid < to - from) mine = list[tid];
    // rows that the threads write, with the mask alone so far, and what lies before and behind the whole granules of all rows
    if (by_threads) {
        for (int i = 0; i < rows; ++i)
            if (tight[i])
                for (int u = tid; u < row_whole[i]; u += NT) rules_forbid<T>(out + i * a.out_stride + row_first[i] + u * N, (1u << N) - 1u, OTHER);
            else if (INPLACE ? row_mask[i] >= 0 : !staged[i]) rules_row<T, INPLACE>(in + i * a.in_stride, out + i * a.out_stride, mask_of(i), row_first[i], row_whole[i], OTHER, tid);
        for (int i = tid >> 5; i < rows; i += NT / 32)
            rules_ends<T, INPLACE>(in + i * a.in_stride, out + i * a.out_stride, mask_of(i), row_first[i], row_whole[i], n, OTHER, lane);
    }
    inverse = 1.0 / rho;
    // (rows from `good` on have no value; where all are bad nothing else of the list is there)
    const int good = state != 0 ? 0 : max(0, min(rows, bad_draft + 1 - i0)), count = state != 0 ? 0 : to - from;
    if (sparse || by_threads) __syncthreads();
    if (!INPLACE && !OWN && drafts && i0 > RULES_FEW) {  // where in the list the drafted tokens before the CTA's rows are is looked up
        for (int j = tid; j < i0; j += NT) {
            const int t = __ldg(drafts + j), q = t >= v0 && t < v0 + n ? rules_find(list, count, t) : -1;
            if (q >= 0 && q < RULES_DRAFTED) atomicAdd(&drafted[q], 1);
        }
        __syncthreads();
    }

    // A listed entry as a thread holds it; drafted tokens before the CTA's rows count as made.
    struct Entry {
        int e;
        uint32_t word;
        double bias;
    };
    auto entry_of = [&](int q, uint2 w) {       // w = list[q]; OWN: q is the entry itself
        if (OWN) {
            Entry x{q, own_word[q], 0.0};
            if (x.word & RULES_BIAS) x.bias = (double)__ldg(a.bias + (long long)b * a.bias_k + own_bias[q] - 1);
            return x;
        }
        Entry x{(int)w.x - v0, w.y, 0.0};
        if (w.y & RULES_BIAS) x.bias = (double)__ldg(a.bias + (long long)b * a.bias_k + a.bias_at[(long long)b * a.most + from + q] - 1);
        if (i0 > 0 && (w.y & RULES_DRAFT)) {
            if (!INPLACE && i0 > RULES_FEW && q < RULES_DRAFTED) x.word += (uint32_t)drafted[q];
            else
                for (int j = 0; j < i0; ++j) x.word += (i0 <= RULES_FEW ? drafted[j] : __ldg(drafts + j)) == (int)w.x;
        }
        return x;
    };
    auto value_of = [&](const Entry& w, int made, Bits x, Bits l) {
        double y = (double)G::value(x);
        if (made > 0 || (w.word & RULES_PROMPT)) y *= G::value(l) > 0.0f ? inverse : rho;
        if (!BACKWARD) {
            if (made > 0) y = y - frequency * (double)made - presence;
            if (w.word & RULES_BIAS) y += w.bias;
        }
        return G::round(y);
    };
    // rows of which the mask leaves little: what it allows, whether in the list or not
    if (!INPLACE && by_threads)
        for (int i = 0; i < good; ++i) {
            if (!tight[i]) continue;
            for (int w = tid; w < (n + 31) / 32; w += NT)
                for (uint32_t x = mask_words[INPLACE ? 0 : i][w]; x; x &= x - 1u) {
                    const int e = w * 32 + __ffs(x) - 1;
                    if (e >= n) break;
                    const Bits y = load_entry(in + i * a.in_stride + e), l = BACKWARD && signs ? load_entry(signs + i * a.logits_stride + e) : y;
                    const int q = !OWN ? rules_find(list, count, v0 + e) : own_word[e] != 0u ? e : -1;
                    Bits value = y;
                    if (q >= 0) {
                        const Entry own = entry_of(q, OWN ? make_uint2(0u, 0u) : list[q]);
                        int made = (int)(own.word & RULES_COUNT);
                        if (own.word & RULES_DRAFT)
                            for (int j = 0; j < i; ++j) made += draft[j] == v0 + e;
                        value = value_of(own, made, y, l);
                    }
                    out[i * a.out_stride + e] = value;
                }
        }
    if (!INPLACE) {
        const bool landed = mbar_wait_twice(&bar, 0u, a.wait_limit_ns) == WAIT_OK;
        for (int i = 0; landed && i < good; ++i) {
            const uint32_t* mask = mask_of(i);
            if (!staged[i] || !mask) continue;
            Bits* data = reinterpret_cast<Bits*>(smem + i * stage_bytes);
            for (int u = tid; u < row_whole[i]; u += NT) {
                const uint32_t forbidden = bits_of(mask, row_first[i] + u * N, N) ^ ((1u << N) - 1u);
                if (forbidden) rules_forbid<T>(data + u * N, forbidden, OTHER);
            }
        }
        if (__syncthreads_or(!landed)) {
            if (tid == 0) atomicOr(a.status, ST_INTERNAL);
            for (int i = 0; i < rows; ++i)
                for (int e = tid; e < n; e += NT) out[i * a.out_stride + e] = (Bits)G::NOT;
            return;
        }
    }
    // the listed entries, each in all rows: in shared memory, or in the output itself where the threads have written the row, or the entry
    // lies before or behind its whole granules
    for (int q = tid; q < count; q += NT) {
        const Entry w = entry_of(OWN ? own_list[q] : q, mine);
        if (!OWN && q + NT < count) mine = list[q + NT];
        Bits x[RULES_ROWS], l[RULES_ROWS];
        Bits* at[RULES_ROWS];
#pragma unroll
        for (int i = 0; i < RULES_ROWS; ++i) {
            at[i] = nullptr;
            if (i >= good || row_mask[i] < -1 || tight[i]) continue;
            const uint32_t* mask = mask_of(i);
            if (mask && !bits_of(mask, w.e, 1)) continue;
            const bool inside = !INPLACE && staged[i] && (unsigned)(w.e - row_first[i]) < (unsigned)(row_whole[i] * N);
            at[i] = inside ? reinterpret_cast<Bits*>(smem + i * stage_bytes) + w.e - row_first[i] : out + i * a.out_stride + w.e;
            x[i] = load_entry(inside ? at[i] : in + i * a.in_stride + w.e);
            l[i] = BACKWARD ? load_entry(signs + i * a.logits_stride + w.e) : x[i];
        }
        int made = (int)(w.word & RULES_COUNT);
#pragma unroll
        for (int i = 0; i < RULES_ROWS; ++i) {
            if (i > 0 && i < rows && (w.word & RULES_DRAFT)) made += draft[i - 1] == v0 + w.e;
            if (at[i]) *at[i] = value_of(w, made, x[i], l[i]);
        }
    }
    if (!INPLACE) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (tid < good && staged[tid] && row_mask[tid] > -2 && row_whole[tid] > 0) {
            bulk_store(out + tid * a.out_stride + row_first[tid], smem + tid * stage_bytes, (uint32_t)row_whole[tid] * 16u);
            bulk_commit();
            bulk_wait_read();                   // (before the shared memory goes)
        }
    }

    // rows without a value
    for (int i = 0; i < rows; ++i) {
        if (i < good && row_mask[i] >= -1) continue;
        if (tid == 0 && slice == 0) atomicOr(a.status, ST_RANGE);
        for (int e = tid; e < n; e += NT) out[i * a.out_stride + e] = (Bits)G::NOT;
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

// A warp per sequence: every lane has read the length before it is written.  Bound by the launch (512 sequences, drafts of 8: 4.7 us a call from
// Python, 1.5 us in a graph).
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
