// Tokens drawn from dense rows of logits, each sequence with its own temperature, top-k, top-p and min-p.
//
//   w_v = exp((l_v - max l) / T), Z = sum w;  order: (logit descending, index ascending)
//   kept = the longest prefix of the order whose entries have rank < top_k, (sum of w before them) < top_p Z and
//          w >= min_p (the first entry always has)
//   the token by a two-level inverse CDF over the kept entries in the order of the vocabulary: chunks of 1024, then entries
//
// A cluster holds the row in shared memory.  The kept prefix ends at one value of the logit, so nothing is sorted: the
// values are counted in bins of the logit's bit pattern (made monotone), the bin in which the prefix ends is split again
// until a bin is one value, and of the entries that tie at it the ones with the lowest index are kept.  Counts are
// integers and masses behind a decision are sums of double-precision weights in a fixed order, so results do not depend
// on the order of the atomics.  Z is an fp32-accumulated sum; a cut or a draw that is within its error of a border is
// decided again with the exact one.
#pragma once
#include "precise_kernels.cuh"
#include "resident_row.cuh"

namespace picospec {

struct SampleArgs {
    const void* logits;
    long long row_stride;
    int R, V, nch;
    const float* temperature;   // [B]
    const int* top_k;           // [B] or null; 0: off
    const float* top_p;         // [B] or null; >= 1: off
    const float* min_p;         // [B] or null; 0: off
    const float* u;             // [B, R, 2]
    int* token;                 // [B, R]
    float* prob;                // [B, R] or null
    float* logprob;             // [B, R] or null
    int* count;                 // [B, R] or null
    unsigned* status;
    unsigned long long* slow_rows;
    unsigned long long wait_limit_ns;
    int slice_chunks;
};

constexpr int SAMPLE_BINS = 2 * THREADS;        // two per thread
constexpr int SAMPLE_SLICE_BYTES = 54 * 1024;   // three CTAs per SM with what lies beside the slice
constexpr int SAMPLE_MAX_CHUNKS = 4 * THREADS;  // four per thread in the scans over a row's chunks
static_assert(MAX_CLUSTER * MAX_SLICE_BYTES / (2 * CHUNK) <= SAMPLE_MAX_CHUNKS, "scan over a row's chunks");

// Monotone bit patterns: a larger logit has a larger key; -0 and +0 have the same.
template <typename T> struct Key;
template <> struct Key<float> {
    static constexpr uint32_t LOWEST = 0x00800000u;     // the lowest finite logit (-inf is 0x007FFFFF)
    static __device__ __forceinline__ uint32_t of(float l) {
        const uint32_t b = __float_as_uint(l + 0.0f);
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    static __device__ __forceinline__ float value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
};
template <> struct Key<__nv_bfloat16> {
    static constexpr uint32_t LOWEST = 0x0080u;         // (-inf is 0x007F)
    static __device__ __forceinline__ uint32_t of(float l) { return Key<float>::of(l) >> 16; }
    static __device__ __forceinline__ float value(uint32_t k) {
        return __uint_as_float(k & 0x8000u ? (k & 0x7FFFu) << 16 : (~k & 0xFFFFu) << 16);
    }
};

// Shared memory beside the slice.  What a peer writes or reads exists twice, and two uses of a copy have a barrier of the
// cluster between them in which the other copy was used.
struct SampleShared {
    float2* record;         // [nch] of the whole row: chunk maximum, sum relative to it
    double* mass;           // [3][nch] chunk masses, relative to the row's maximum; [2]: from the records, the CTA's own
    int* ties;              // [2][nch]
    float* group_max;       // [slice_chunks * 32] maximum of a lane's entries of a chunk
    uint32_t* bins;         // [2][2][SAMPLE_BINS] counts, fixed-point masses
    double* table;          // exp_by_table
};
inline __host__ __device__ size_t sample_layout(SampleShared* s, unsigned char* base, int slice_chunks, int nch, int elem) {
    size_t at = (size_t)slice_chunks * CHUNK * elem + 16;
    const auto take = [&](size_t bytes) {
        unsigned char* p = base + at;
        at += (bytes + 15) / 16 * 16;
        return p;
    };
    SampleShared x;
    x.record = (float2*)take((size_t)nch * 8);
    x.mass = (double*)take((size_t)nch * 24);
    x.ties = (int*)take((size_t)nch * 8);
    x.group_max = (float*)take((size_t)slice_chunks * 128);
    x.bins = (uint32_t*)take(4 * SAMPLE_BINS * 4);
    x.table = (double*)take(EXP_STEPS * 8);
    if (s) *s = x;
    return at;
}

// One row, seen by one CTA of its cluster.
template <typename T> struct SampleRow {
    using K = Key<T>;
    const SampleArgs& a;
    SampleShared sh;
    Slice<T> s;
    uint32_t rank, ranks;
    int mis, tid, lane, warp, first_chunk;
    double* scan_tot;           // shared [WARPS]
    double (*pair)[MAX_CLUSTER][2];     // shared [2][MAX_CLUSTER][2]: sums of the CTAs
    float c32, top;             // scale, largest logit
    double rT;                  // 1 / T
    double Z;
    int table_at, bins_at, pair_at;     // copies to use next

    __device__ __forceinline__ double weight(float l) const { return exp_by_table(((double)l - (double)top) * rT, sh.table); }
    // entry `o` of a chunk in a lane's order (ChunkRegs::offset) as an offset in the chunk's memory, and in the vocabulary
    __device__ __forceinline__ int place(int o) const { return o < mis ? o + CHUNK : o; }
    // the lane's entries of chunk c whose logit is at least `low`: f(logit, its offset in the chunk's memory)
    template <typename F> __device__ __forceinline__ void entries_from(int c, float low, F&& f) const {
        const bool any = sh.group_max[c * 32 + lane] >= low;
        if (!__any_sync(0xffffffffu, any)) return;
        if (any) {
            const unsigned char* data = s.chunk(c);
#pragma unroll 1
            for (int j = 0; j < ChunkRegs<T>::NVEC; ++j) {
                const int o = (j * 32 + lane) * ChunkRegs<T>::VEC;
#pragma unroll
                for (int e = 0; e < ChunkRegs<T>::VEC; ++e) {
                    const int at = place(o + e);
                    if (first_chunk * CHUNK + c * CHUNK + at - mis >= a.V) continue;
                    const float l = entry_value(data, at, (const T*)nullptr);
                    if (l >= low) f(l, at);
                }
            }
        }
        __syncwarp();
    }

    // x = (top - l) log2(e) / T, monotone in l
    __device__ __forceinline__ float distance(float l, float off) const {
        return offset_ok(off) ? fmaxf(0.0f, fmaf(-l, c32, off)) : l == top ? 0.0f : CUDART_INF_F;
    }

    // Counts of the whole cluster: this thread's bins 2 tid and 2 tid + 1.  The other copy is cleared for the next use.
    __device__ __forceinline__ void gather_bins(uint32_t count[2], double mass[2]) {
        uint32_t* mine = sh.bins + bins_at * 2 * SAMPLE_BINS;
        cluster_sync();
        count[0] = count[1] = 0u;
        mass[0] = mass[1] = 0.0;
        for (uint32_t r = 0; r < ranks; ++r) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                count[i] += peer_load(peer_addr(mine + 2 * tid + i, r));
                mass[i] += (double)peer_load(peer_addr(mine + SAMPLE_BINS + 2 * tid + i, r));
            }
        }
        bins_at ^= 1;
        uint32_t* other = sh.bins + bins_at * 2 * SAMPLE_BINS;
        for (int i = tid; i < 2 * SAMPLE_BINS; i += THREADS) other[i] = 0u;
        __syncthreads();
    }

    // Exact masses of the entries with key > k1 and key >= k0 over the whole row.
    __device__ __forceinline__ void exact_above(uint32_t k1, uint32_t k0, double& above, double& from) {
        double s1 = 0.0, s0 = 0.0;
        const float low = K::value(k0);
        for (int c = warp; c < s.chunks; c += WARPS)
            entries_from(c, low, [&](float l, int) {
                const double w = weight(l);
                s0 += w;
                if (K::of(l) > k1) s1 += w;
            });
        s1 = warp_sum(s1);
        s0 = warp_sum(s0);
        __shared__ double part[WARPS][2];
        if (lane == 0) part[warp][0] = s1, part[warp][1] = s0;
        __syncthreads();
        if (tid < 2 * (int)ranks) {
            double t = 0.0;
            for (int w = 0; w < WARPS; ++w) t += part[w][tid & 1];
            const uint32_t to = peer_addr(&pair[pair_at][rank][tid & 1], tid >> 1);
            peer_store(to, (uint32_t)__double2loint(t));
            peer_store(to + 4, (uint32_t)__double2hiint(t));
        }
        cluster_sync();
        above = from = 0.0;
        for (uint32_t r = 0; r < ranks; ++r) {
            above += pair[pair_at][r][0];
            from += pair[pair_at][r][1];
        }
        pair_at ^= 1;
    }

    // Per chunk of the row: the exact mass of the entries with key > cut, and the number of entries with key == cut.
    // MASSES false: only the number of entries with key >= cut.  Returns the copy of the tables that holds them.
    template <bool MASSES> __device__ __forceinline__ int chunk_table(uint32_t cut, bool count_all) {
        const int t = table_at;
        table_at ^= 1;
        const float low = K::value(cut);
        for (int c = warp; c < s.chunks; c += WARPS) {
            double m = 0.0;
            int n = 0;
            entries_from(c, low, [&](float l, int) {
                const bool tie = K::of(l) == cut;
                if (MASSES && (!tie || count_all)) m += weight(l);
                if (tie || count_all) ++n;
            });
            m = warp_sum(m);
            n = warp_sum(n);
            const int at = t * a.nch + first_chunk + c;
            if (lane < (int)ranks) {
                const uint32_t to = peer_addr(sh.mass + at, lane);
                peer_store(to, (uint32_t)__double2loint(m));
                peer_store(to + 4, (uint32_t)__double2hiint(m));
                peer_store(peer_addr(sh.ties + at, lane), (uint32_t)n);
            }
        }
        cluster_sync();
        return t;
    }
    // The exact Z and the number of finite entries.
    __device__ __forceinline__ int exact_total() {
        const int t = chunk_table<true>(K::LOWEST, true);
        double m = 0.0;
        for (int i = 0; i < 4; ++i) {
            const int c = 4 * tid + i;
            if (c < a.nch) m += sh.mass[t * a.nch + c];
        }
        block_scan_incl(m, scan_tot, Z);
        return t;
    }
};

// the smallest of the threads' values, seen by all (two barriers)
__device__ __forceinline__ int block_min(int v, int* shared) {
    if (threadIdx.x == 0) *shared = 0x7FFFFFFF;
    __syncthreads();
    v = __reduce_min_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0 && v != 0x7FFFFFFF) atomicMin(shared, v);
    __syncthreads();
    const int r = *shared;
    __syncthreads();
    return r;
}

constexpr int NONE = 0x7FFFFFFF;
constexpr int MAX_TURNS = 200;

// Where the kept prefix ends: entries with key > key are kept, and the first `ties` (by index) of those with key == key.
struct SampleCut {
    uint32_t key;
    int ties;
    int count;
};

template <typename T> struct SampleLimits {
    int k;              // 0x7FFFFFFF: off
    double p, m;        // p >= 1, m <= 0: off
};

// The end of the prefix among bins of one value each.  `before`, `mass_before`: entries and mass above the bins.  pz: top_p Z.
template <typename T>
__device__ __forceinline__ SampleCut cut_in_values(SampleRow<T>& row, const SampleLimits<T>& lim, uint32_t ktop, uint32_t klow,
                                                   const uint32_t count[2], long long before, double mass_before, double pz,
                                                   int* shared_min) {
    using K = Key<T>;
    __shared__ SampleCut found;
    double w[2], n_all, m_all;
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = count[i] ? row.weight(K::value(ktop - (uint32_t)(2 * row.tid + i))) : 0.0;
    const double n_here = (double)count[0] + (double)count[1], m_here = (double)count[0] * w[0] + (double)count[1] * w[1];
    const double n_upto = block_scan_incl(n_here, row.scan_tot, n_all), m_upto = block_scan_incl(m_here, row.scan_tot, m_all);
    double nb = (double)before + n_upto - n_here, mb = mass_before + m_upto - m_here;
    int first = NONE;
    SampleCut mine{};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        double keep = (double)count[i];
        if (lim.m > 0.0 && w[i] < lim.m) keep = 0.0;
        keep = fmin(keep, fmax(0.0, (double)lim.k - nb));
        if (lim.p < 1.0) keep = fmin(keep, mb >= pz ? 0.0 : w[i] > 0.0 ? ceil((pz - mb) / w[i]) : keep);
        if (nb == 0.0 && count[i]) keep = fmax(keep, 1.0);      // the first entry is kept whatever the limits
        if (count[i] && keep < (double)count[i] && first == NONE) {
            first = 2 * row.tid + i;
            mine.key = ktop - (uint32_t)first;
            mine.ties = (int)keep;
            mine.count = (int)(nb + keep);
        }
        nb += (double)count[i];
        mb += (double)count[i] * w[i];
    }
    const int at = block_min(first, shared_min);
    if (at == NONE) {           // every entry of the bins is kept
        if (row.tid == 0) found = SampleCut{klow, NONE, (int)((double)before + n_all)};
    } else if (first == at) {
        found = mine;
    }
    __syncthreads();
    const SampleCut r = found;
    __syncthreads();
    return r;
}

// A logit that every entry of the kept prefix reaches, from the largest entry of each group of 32: k of them, or the
// share p of the mass, at or above a value bound the prefix to it.  Else by top-p alone: entries below (1 - p) Z / V hold less than
// 1 - p in all.  -inf: no bound.
template <typename T>
__device__ __forceinline__ float prefix_bound(SampleRow<T>& row, const SampleLimits<T>& lim, int* shared_min) {
    constexpr float STEPS = 8.0f;           // bins per factor of two
    const float off = __fmul_rn(row.top, row.c32);
    uint32_t* counts = row.sh.bins + row.bins_at * 2 * SAMPLE_BINS;
    for (int i = row.tid; i < row.s.chunks * 32; i += THREADS) {
        const float g = row.sh.group_max[i];
        if (!(g > -CUDART_INF_F)) continue;
        const float x = row.distance(g, off) * STEPS;
        if (x < (float)SAMPLE_BINS) atomicAdd(&counts[(int)x], 1u);
    }
    uint32_t count[2];
    double unused[2];
    row.gather_bins(count, unused);
    double n_all, m_all, w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = (double)count[i] * (double)exp2f(-(float)(2 * row.tid + i + 1) / STEPS);    // at least
    const double n = block_scan_incl((double)count[0] + (double)count[1], row.scan_tot, n_all);
    const double m = block_scan_incl(w[0] + w[1], row.scan_tot, m_all);
    const double want = lim.p * row.Z * (1.0 + 1e-4);
    int first = NONE;
    if (n >= (double)lim.k || (lim.p < 1.0 && m >= want)) first = 2 * row.tid + 1;
    if (n - (double)count[1] >= (double)lim.k || (lim.p < 1.0 && m - w[1] >= want)) first = 2 * row.tid;
    first = block_min(first, shared_min);
    double x = first == NONE ? 1e30 : (double)(first + 1) / STEPS;
    if (lim.p < 1.0) x = fmin(x, log2((double)row.a.V / ((1.0 - lim.p) * row.Z)));
    if (lim.m > 0.0) x = fmin(x, -log2(lim.m));
    // down by more than the roundings of x and of this division
    const double low = (double)row.top - (x * (1.0 + 1e-5) + 1e-4) / (double)row.c32 - fabs((double)row.top) * 1e-6;
    return x >= 1e29 || !(low > -3.4e38) ? -CUDART_INF_F : __double2float_rd(low);
}

template <typename T>
__device__ __forceinline__ SampleCut find_cut(SampleRow<T>& row, const SampleLimits<T>& lim, bool& exact, int* shared_min) {
    using K = Key<T>;
    const float bound = prefix_bound<T>(row, lim, shared_min);
    uint32_t ktop = K::of(row.top), klow = bound > -CUDART_INF_F ? max(K::of(bound), K::LOWEST) : K::LOWEST;
    if (klow > ktop) klow = ktop;
    long long before = 0;
    double mass_before = 0.0;
    // Each turn leaves one bin of the range or leaves out one at least.  Masses of bins are rounded up, so a turn may take a
    // bin before the right one; one whose bins are that wide has few of any weight.
    for (int turn = 0; turn < MAX_TURNS; ++turn) {
        int shift = 0;
        while (((ktop - klow) >> shift) >= (uint32_t)SAMPLE_BINS) ++shift;
        uint32_t* counts = row.sh.bins + row.bins_at * 2 * SAMPLE_BINS;
        const float low = K::value(klow);
        for (int c = row.warp; c < row.s.chunks; c += WARPS)
            row.entries_from(c, low, [&](float l, int) {
                const uint32_t k = K::of(l);
                if (k > ktop) return;
                const uint32_t b = (ktop - k) >> shift;
                atomicAdd(&counts[b], 1u);
                if (shift > 0 && lim.p < 1.0) {         // a share of the bin's largest weight, in steps of 2^-12, rounded up
                    const float most = K::value(ktop - (b << shift));
                    atomicAdd(&counts[SAMPLE_BINS + b], (uint32_t)fminf(4096.0f, ceilf(ex2_approx((l - most) * row.c32) * 4096.0f)));
                }
            });
        uint32_t count[2];
        double mass[2];
        row.gather_bins(count, mass);
        if (shift == 0) {
            if (lim.p >= 1.0) return cut_in_values<T>(row, lim, ktop, klow, count, before, mass_before, 0.0, shared_min);
            for (;;) {
                const double g = exact ? 0.0 : GUARD_Z, pz = lim.p * row.Z;
                const SampleCut x = cut_in_values<T>(row, lim, ktop, klow, count, before, mass_before, pz * (1.0 - g), shared_min);
                if (exact) return x;
                const SampleCut y = cut_in_values<T>(row, lim, ktop, klow, count, before, mass_before, pz * (1.0 + g), shared_min);
                if (x.key == y.key && x.ties == y.ties) return x;
                row.exact_total();
                exact = true;
            }
        }
        // the bin in which the prefix ends
        double n_all, m_all, w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t b = (uint32_t)(2 * row.tid + i);
            w[i] = lim.p < 1.0 && count[i] ? mass[i] * (1.0 / 4096.0) * row.weight(K::value(ktop - (b << shift))) : 0.0;
        }
        const double n_here = (double)count[0] + (double)count[1], m_here = w[0] + w[1];
        double nb = (double)before + block_scan_incl(n_here, row.scan_tot, n_all) - n_here;
        double mb = mass_before + block_scan_incl(m_here, row.scan_tot, m_all) - m_here;
        int first = NONE, first_sure = NONE;       // first_sure: by top-k or min-p, which are exact here
        const double nb_first = nb;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (count[i]) {
                const uint32_t b = (uint32_t)(2 * row.tid + i), hi = ktop - (b << shift);
                const uint32_t lo = hi - klow >= (1u << shift) ? hi - (1u << shift) + 1u : klow;
                const bool sure = nb + (double)count[i] >= (double)lim.k || (lim.m > 0.0 && row.weight(K::value(lo)) < lim.m);
                if (sure && first_sure == NONE) first_sure = (int)b;
                if ((sure || (lim.p < 1.0 && mb + w[i] >= lim.p * row.Z)) && first == NONE) first = (int)b;
            }
            nb += (double)count[i];
            mb += w[i];
        }
        first_sure = block_min(first_sure, shared_min);
        first = block_min(first, shared_min);
        if (first == NONE) {        // no limit is reached, by the masses of the bins: the last value that there is
            const int last = count[1] ? 2 * row.tid + 1 : count[0] ? 2 * row.tid : -1;
            first = block_min(last >= 0 ? -last : NONE, shared_min);
            if (first == NONE) return SampleCut{klow, NONE, (int)before};
            first = -first;
        }
        __shared__ long long shared_before[2];
        if (row.tid == first / 2) {
            shared_before[0] = (long long)nb_first + (first & 1 ? count[0] : 0u);
            shared_before[1] = shared_before[0] + (first & 1 ? count[1] : count[0]);
        }
        __syncthreads();
        const long long upto = shared_before[0], behind = shared_before[1];
        __syncthreads();
        const uint32_t hi = ktop - ((uint32_t)first << shift), lo = hi - klow >= (1u << shift) ? hi - (1u << shift) + 1u : klow;
        if (lim.p < 1.0) {
            // is the end of the mass in this bin, exactly?
            double above, from;
            row.exact_above(hi, lo, above, from);
            const double pz = lim.p * row.Z;
            if (!exact && (fabs(above - pz) <= GUARD_Z * pz || fabs(from - pz) <= GUARD_Z * pz)) {
                row.exact_total();
                exact = true;
            }
            const double at = lim.p * row.Z;
            if (above >= at && hi < ktop) {             // before it
                klow = hi + 1u;
                continue;
            }
            if (from < at && first != first_sure && lo > klow) {        // behind it
                ktop = lo - 1u;
                before = behind;
                mass_before = from;
                continue;
            }
            mass_before = above;
        }
        ktop = hi;
        klow = lo;
        before = upto;
    }
    if (row.tid == 0) atomicOr(row.a.status, ST_INTERNAL);
    return SampleCut{klow, NONE, -1};
}

template <typename T>
__global__ void __launch_bounds__(THREADS, 3) sample_kernel(SampleArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[MAX_SLICE_TILES];
    __shared__ double scan_tot[WARPS];
    __shared__ double pair[2][MAX_CLUSTER][2];
    __shared__ int shared_min, shared_chunk, shared_kept;
    __shared__ float part_max[WARPS];
    using K = Key<T>;
    SampleRow<T> row{a};
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(row.ranks));
    row.rank = cluster_rank();
    row.tid = threadIdx.x; row.lane = threadIdx.x & 31; row.warp = threadIdx.x >> 5;
    row.scan_tot = scan_tot;
    row.pair = pair;
    row.table_at = row.bins_at = row.pair_at = 0;
    sample_layout(&row.sh, smem, a.slice_chunks, a.nch, (int)sizeof(T));
    const int tid = row.tid, lane = row.lane, warp = row.warp;
    const long long r = blockIdx.x / row.ranks;
    const int b = (int)(r / a.R);
    cluster_arrive();
    exp_table(row.sh.table);
    for (int i = tid; i < 4 * SAMPLE_BINS; i += THREADS) row.sh.bins[i] = 0u;
    grid_dependency_sync();

    const StagedRow<T> in(reinterpret_cast<const T*>(a.logits) + r * a.row_stride, a.V);
    row.mis = in.mis;
    row.first_chunk = (int)row.rank * a.slice_chunks;
    row.s.stage(smem, bars, in, row.rank, a.slice_chunks, true);
    const float temperature = a.temperature[b];
    row.c32 = temp_scale(temperature);
    row.rT = 1.0 / (double)temperature;
    SampleLimits<T> lim;
    const int k = a.top_k ? a.top_k[b] : 0;
    const float p = a.top_p ? a.top_p[b] : 1.0f, m = a.min_p ? a.min_p[b] : 0.0f;
    lim.k = k > 0 && k < a.V ? k : NONE;
    lim.p = (double)p;
    lim.m = (double)m;
    unsigned bad = temp_ok(temperature) && row.c32 < CUDART_INF_F ? 0u : ST_TEMPERATURE;
    if (k < 0 || !(p > 0.0f) || !(m >= 0.0f && m <= 1.0f)) bad |= ST_RANGE;

    // statistics of the chunks, to every CTA of the cluster
    cluster_wait();
    for (int c = warp; c < row.s.chunks; c += WARPS) {
        const int late = row.s.wait(c, in.mis != 0, a.wait_limit_ns);
        ChunkRegs<T> x;
        load_staged_shifted(x, row.s.chunk(c), row.s.begin + c * CHUNK, in.end, in.mis, lane);
        const float g = x.lane_max_plain();
        row.sh.group_max[c * 32 + lane] = g;
        float top = warp_max_redux(g);
        const float sum = warp_sum(lane_weight_sum(x, top, row.c32, top > -CUDART_INF_F ? __fmul_rn(top, row.c32) : 0.0f));
        if (late != WAIT_OK) top = CUDART_NAN_F;
        if (lane < 2 * (int)row.ranks)
            peer_store(peer_addr(reinterpret_cast<float*>(row.sh.record + row.first_chunk + c) + (lane & 1), lane >> 1),
                       __float_as_uint(lane & 1 ? sum : top));
    }
    cluster_sync();

    float top = -CUDART_INF_F;
    for (int c = tid; c < a.nch; c += THREADS) {
        const float2 x = row.sh.record[c];
        if (x.x != x.x) bad |= ST_INTERNAL;
        else if (x.x == CUDART_INF_F || x.y != x.y) bad |= ST_LOGIT;
        top = fmaxf(top, x.x);
    }
    top = warp_max_redux(top);
    if (lane == 0) part_max[warp] = top;
    bad = __reduce_or_sync(0xffffffffu, bad);
    __shared__ unsigned shared_bad;
    if (tid == 0) shared_bad = 0u;
    __syncthreads();
    if (lane == 0 && bad) atomicOr(&shared_bad, bad);
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, part_max[w]);
    __syncthreads();
    bad = shared_bad;
    if (!(top > -CUDART_INF_F) && !(bad & ST_INTERNAL)) bad |= ST_LOGIT;
    if (bad) {                  // (the same in every CTA)
        if (row.rank == 0 && tid == 0) {
            atomicOr(a.status, bad);
            a.token[r] = -1;
            if (a.prob) a.prob[r] = -1.0f;
            if (a.logprob) a.logprob[r] = CUDART_NAN_F;
            if (a.count) a.count[r] = -1;
        }
        return;
    }
    row.top = top;
    // fp32-accumulated chunk masses on the scale of the exact ones
    double z = 0.0;
    for (int i = 0; i < 4; ++i) {
        const int c = 4 * tid + i;
        if (c >= a.nch) break;
        const float2 x = row.sh.record[c];
        const double mass = x.x > -CUDART_INF_F ? (double)x.y * stream_scale(x.x, row.c32) * exp_call(((double)x.x - (double)top) * row.rT) : 0.0;
        row.sh.mass[2 * a.nch + c] = mass;
        z += mass;
    }
    block_scan_incl(z, scan_tot, row.Z);

    const bool limited = lim.k != NONE || lim.p < 1.0 || lim.m > 0.0;
    bool exact = false;
    SampleCut cut{K::LOWEST, NONE, 0};
    int t = 2;                  // the table of the draw
    if (limited) {
        cut = find_cut<T>(row, lim, exact, &shared_min);
        t = row.template chunk_table<true>(cut.key, false);
    } else if (a.count) {
        const int n = row.template chunk_table<false>(K::LOWEST, true);
        double finite = 0.0, all;
        for (int c = tid; c < a.nch; c += THREADS) finite += (double)row.sh.ties[n * a.nch + c];
        block_scan_incl(finite, scan_tot, all);
        cut.count = (int)all;
    }

    // level 1
    const float u0 = a.u[2 * r], u1 = a.u[2 * r + 1];
    const double cut_weight = limited ? row.weight(K::value(cut.key)) : 0.0;
    double W = 0.0;
    for (;;) {
        double mass[4], mine = 0.0, ties = 0.0, unused;
        int kept[4], n[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 4 * tid + i;
            n[i] = limited && c < a.nch ? row.sh.ties[t * a.nch + c] : 0;
            ties += (double)n[i];
        }
        double ties_before = limited ? block_scan_incl(ties, scan_tot, unused) - ties : 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 4 * tid + i;
            kept[i] = (int)fmin((double)n[i], fmax(0.0, (double)cut.ties - ties_before));
            ties_before += (double)n[i];
            mass[i] = c < a.nch ? row.sh.mass[t * a.nch + c] + (double)kept[i] * cut_weight : 0.0;
            mine += mass[i];
        }
        double upto = block_scan_incl(mine, scan_tot, W) - mine;
        const double target = (double)u0 * W, guard = limited || exact ? 0.0 : GUARD_Z * W;
        int first = NONE, last = -1, close = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 4 * tid + i;
            upto += mass[i];
            if (c < a.nch) {
                if (mass[i] > 0.0 && upto > target && first == NONE) first = c;
                if (mass[i] > 0.0) last = c;
                if (guard > 0.0 && fabs(upto - target) <= guard) close = 1;
            }
        }
        close = __syncthreads_or(close);
        if (close) {            // (untruncated rows only)
            t = row.exact_total();
            exact = true;
            continue;
        }
        first = block_min(first, &shared_min);
        if (first == NONE) first = -block_min(last >= 0 ? -last : NONE, &shared_min);     // the last rounding
        #pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * tid + i == first) shared_chunk = first, shared_kept = kept[i];
        __syncthreads();
        break;
    }
    if (exact && row.rank == 0 && tid == 0) atomicAdd(a.slow_rows, 1ull);

    // level 2: by the CTA that holds the chunk
    const int chunk = shared_chunk, chunk_ties = shared_kept, local = chunk - row.first_chunk;
    if (local < 0 || local >= row.s.chunks) return;
    float l[4];
    double w[4], tie[4], ties = 0.0, mine = 0.0, total, unused;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = 4 * tid + i;
        l[i] = chunk * CHUNK + e < a.V ? entry_value(row.s.chunk(local), in.mis + e, (const T*)nullptr) : -CUDART_INF_F;
        tie[i] = limited && K::of(l[i]) == cut.key ? 1.0 : 0.0;
        ties += tie[i];
    }
    double ties_before = limited ? block_scan_incl(ties, scan_tot, unused) - ties : 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool keep = l[i] > -CUDART_INF_F && (!limited || K::of(l[i]) > cut.key || (tie[i] > 0.0 && ties_before < (double)chunk_ties));
        ties_before += tie[i];
        w[i] = keep ? row.weight(l[i]) : 0.0;
        mine += w[i];
    }
    double upto = block_scan_incl(mine, scan_tot, total) - mine;
    int first = NONE, last = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        upto += w[i];
        if (w[i] > 0.0) {
            last = 4 * tid + i;
            if (upto > (double)u1 * total && first == NONE) first = last;
        }
    }
    first = block_min(first, &shared_min);
    if (first == NONE) first = -block_min(last >= 0 ? -last : NONE, &shared_min);
    if (tid == first / 4) {
        const int i = first & 3;
        a.token[r] = chunk * CHUNK + first;
        double wi = 0.0, li = 0.0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j == i) wi = w[j], li = (double)l[j];
        if (a.prob) a.prob[r] = (float)(wi / W);
        if (a.logprob) a.logprob[r] = (float)((li - (double)top) * row.rT - log(row.Z));
        if (a.count) a.count[r] = cut.count;
    }
}

inline int sample_smem(int slice_chunks, int nch, int elem) { return (int)sample_layout(nullptr, nullptr, slice_chunks, nch, elem); }

}  // namespace picospec
