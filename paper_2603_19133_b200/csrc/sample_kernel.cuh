// Tokens drawn from dense rows of logits, each sequence with its own temperature, top-k, top-p and min-p.
//
//   w_v = exp((l_v - max l) / T), Z = sum w;  order: (logit descending, index ascending)
//   kept = the longest prefix of the order whose entries have rank < top_k, (sum of w before them) < top_p Z and
//          w >= min_p (the first entry always has)
//   the token by a two-level inverse CDF over the kept entries in the order of the vocabulary: chunks of 1024, then entries
//
// A cluster holds the row in shared memory.  Nothing is sorted: the kept prefix ends at one value of the logit, and
// of the entries that tie there those with the lowest index are kept.  The value is found by counting logits in bins of
// their bit patterns (made monotone) within bounds on where it lies; bf16 values get a bin each, of an fp32 row the few
// entries of the bin in question are put in order.  min_p is a bound on the logit itself.
//
// Counts are integers and masses that decide are double-precision sums in a fixed order, so that results do not depend on the
// order of the atomics.  Where fp32 sums suffice -- the chunk masses of a row without limits, Z of a row whose prefix
// ends among entries that weigh -- a cut or a draw within their error of a border is decided again with exact ones.
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
constexpr int SAMPLE_LIST = THREADS;            // entries of a bin that are put in order
constexpr int SAMPLE_SLICE_BYTES = 72 * 1024;   // two CTAs per SM with what lies beside the slice
constexpr int SAMPLE_SLICE_PLAIN = 54 * 1024;   // three, for rows without limits
constexpr int SAMPLE_SMEM_MOST = 227000;        // dynamic shared memory
constexpr int SAMPLE_CLUSTER = 8;               // CTAs of a cluster at most
constexpr int SAMPLE_DENSE_HITS = 6;            // of a lane's 32 entries: beyond, all of them are looked at in turn
constexpr int SAMPLE_STEPS = 256;               // powers in the exponential's table
constexpr int MAX_TURNS = 200;
constexpr int NONE = 0x7FFFFFFF;

// Monotone bit patterns: a larger logit has a larger key; -0 and +0 have the same.  No logit has the key just below that of 0
// (the pattern of -0), whose value would compare as 0: the ends of a range of keys are moved off it.
template <typename T> struct Key;
template <typename T> __device__ __forceinline__ uint32_t upper_end(uint32_t k) { return k == Key<T>::ABSENT ? k - 1u : k; }
template <typename T> __device__ __forceinline__ uint32_t lower_end(uint32_t k) { return k == Key<T>::ABSENT ? k + 1u : k; }
template <> struct Key<float> {
    static constexpr uint32_t LOWEST = 0x00800000u;     // the lowest finite logit (-inf is 0x007FFFFF)
    static constexpr uint32_t ABSENT = 0x7FFFFFFFu;
    static __device__ __forceinline__ uint32_t of(float l) {
        const uint32_t b = __float_as_uint(l + 0.0f);
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    static __device__ __forceinline__ float value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
};
template <> struct Key<__nv_bfloat16> {
    static constexpr uint32_t LOWEST = 0x0080u;         // (-inf is 0x007F)
    static constexpr uint32_t ABSENT = 0x7FFFu;
    static __device__ __forceinline__ uint32_t of(float l) { return Key<float>::of(l) >> 16; }
    static __device__ __forceinline__ float value(uint32_t k) {
        return __uint_as_float(k & 0x8000u ? (k & 0x7FFFu) << 16 : (~k & 0xFFFFu) << 16);
    }
};

// bit e: low <= entry e of the granule (<= high, unless `open`)
__device__ __forceinline__ uint32_t granule_between(uint4 q, float low, float high, bool open, const __nv_bfloat16*) {
    const __nv_bfloat162 lo = __float2bfloat162_rn(low), hi = __float2bfloat162_rn(high);       // (exact: bf16 values)
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
        uint32_t in = __hge2_mask(x, lo);
        if (!open) in &= __hle2_mask(x, hi);
        m |= in & (0x00020001u << (2 * i));
    }
    return (m | m >> 16) & 0xFFu;
}
__device__ __forceinline__ uint32_t granule_between(uint4 q, float low, float high, bool open, const float*) {
    float l[4];
    unpack_granule(q, l, (const float*)nullptr);
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) m |= l[i] >= low && (open || l[i] <= high) ? 1u << i : 0u;
    return m;
}

struct SampleRecord {       // of a chunk
    float top, sum;         // maximum, sum of the exponentials relative to it
    int finite, pad;        // number of finite entries (rows without limits); -1: the chunk came too late
};
struct SampleEntry {
    uint32_t key;
    int index;              // in the vocabulary
};
struct SampleSorted {
    double weight;
    uint32_t key;
    int index;
};
// What a CTA of the cluster found in a pass, for its peers to read.
struct SampleFound {
    double above, total;    // exact masses
    int n_above, listed;
};

// Shared memory: what has a fixed size, then what goes by the number of chunks, then the slice.  What a peer writes or reads exists
// twice, and two uses of a copy have a barrier of the cluster between them in which the other copy was used.
template <typename T> struct SamplePlaces {
    static constexpr int LISTS = sizeof(T) == 4;                // (lists are of fp32 rows: bf16 bins end at one value each)
    static constexpr int TABLE = 0;                             // double [SAMPLE_STEPS]
    static constexpr int SCAN = TABLE + SAMPLE_STEPS * 8;       // double [WARPS][2]
    static constexpr int FOUND = SCAN + WARPS * 16;             // SampleFound [2]
    static constexpr int INTS = FOUND + 2 * (int)sizeof(SampleFound) + 16;      // int [WARPS]
    static constexpr int BINS = INTS + WARPS * 4;               // uint32_t [2][2][SAMPLE_BINS]
    static constexpr int LIST = BINS + 4 * SAMPLE_BINS * 4;     // SampleEntry [2][SAMPLE_LIST]: this CTA's entries of a bin
    static constexpr int SORTED = LIST + LISTS * 2 * SAMPLE_LIST * (int)sizeof(SampleEntry);    // SampleSorted [SAMPLE_LIST]: the row's, in order
    static constexpr int RECORD = SORTED + LISTS * SAMPLE_LIST * (int)sizeof(SampleSorted);     // SampleRecord [nch] of the whole row
    static_assert(FOUND % 16 == 0 && INTS % 16 == 0 && BINS % 16 == 0 && RECORD % 16 == 0 && sizeof(SampleRecord) == 16, "alignment");
    static __host__ __device__ constexpr int part(int nch) { return RECORD + 16 * nch; }        // double [2][nch] chunk masses found in a pass
    static __host__ __device__ constexpr int mass(int nch) { return RECORD + 32 * nch; }        // double [nch] put together, by this CTA for itself
    static __host__ __device__ constexpr int ties(int nch) { return RECORD + 40 * nch; }        // int [2][nch]
    static __host__ __device__ constexpr int group_max(int nch) { return RECORD + 48 * nch; }   // float [slice_chunks * 32] maximum of a lane's entries of a chunk
    static __host__ __device__ constexpr int data(int nch, int slice_chunks) { return (group_max(nch) + slice_chunks * 128 + 127) / 128 * 128; }
    static __host__ __device__ constexpr int total(int nch, int slice_chunks) { return data(nch, slice_chunks) + slice_chunks * CHUNK * (int)sizeof(T) + 16; }
};
// (the compiler sees that what it points to is shared memory)
template <typename P> __device__ __forceinline__ P* shared_at(int offset) {
    extern __shared__ __align__(128) unsigned char smem[];
    return reinterpret_cast<P*>(smem + offset);
}

// Double-precision weights exp((l - top) / T), to about one unit in the last place: y = (l - top) 256 log2(e) / T, n = y rounded
// to an integer, f = y - n, and the weight is 2^(n / 256) (1 + z + z^2/2 + z^3/6 + z^4/24) with z = f ln 2 / 256, |z| < 0.00136 (the
// next term is below 2^-54).  The powers 2^(j / 256) lie in shared memory.  Nine double-precision
// operations and a conversion, against thirteen in exp_by_table; 32 entries of 8 warps take 2750 cycles by themselves, 4500 in this kernel.
struct SampleWeight {
    double top, scale;      // scale: 256 log2(e) / T
    float cut;              // lower logits, -inf too, are taken as this one, whose weight is lost in every sum, unless it is the lowest there is
    // The cut lies 600 T below the largest logit, rounded down.  Where fp32 has no value within 100 T of that, the next
    // one below stands for all others, with a scale that leaves it exp(-600).
    __device__ __forceinline__ void init(float largest, double rT) {
        constexpr double FAR = 600.0;
        top = (double)largest;
        scale = (double)SAMPLE_STEPS * 1.4426950408889634074 * rT;
        const float below = Key<float>::value(max(Key<float>::of(largest) - 1u, Key<float>::LOWEST));
        cut = fmaxf(Key<float>::value(Key<float>::LOWEST), fminf(below, __double2float_rd(top - FAR / rT)));
        if ((top - (double)below) * rT > 100.0) {
            cut = below;
            scale = (double)SAMPLE_STEPS * 1.4426950408889634074 * FAR / (top - (double)below);
        }
    }
    __device__ __forceinline__ double operator()(float l) const {
        constexpr double Z = 0.69314718055994530942 / SAMPLE_STEPS, ROUND = 6755399441055744.0;      // 1.5 * 2^52
        const double d = (double)fmaxf(l, cut) - top;      // (no branch: several of these run side by side)
        const double t = fma(d, scale, ROUND);
        const int n = __double2loint(t);
        const double f = fma(d, scale, -(t - ROUND));
        const double p = f * fma(f, fma(f, fma(f, Z * Z * Z * Z / 24.0, Z * Z * Z / 6.0), Z * Z / 2.0), Z);
        const double w = shared_at<double>(SamplePlaces<float>::TABLE)[n & (SAMPLE_STEPS - 1)];
        const double y = fma(w, p, w);
        return __hiloint2double(__double2hiint(y) + ((n >> 8) << 20), __double2loint(y));
    }
};

struct SampleLimits {
    int k;              // NONE: off
    double p;           // >= 1: off
    uint32_t key;       // min-p as a bound on the key; LOWEST: off
};

// Where the kept prefix ends: entries with a larger key are kept; of those with this key the first `ties` by index, or, if
// `listed`, those up to `index`.
struct SampleCut {
    uint32_t key;
    int ties, index, count;
    bool listed;
};

// inclusive prefix sums over a warp
__device__ __forceinline__ double warp_scan(double x, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// A lane's 32 entries of a chunk, from `offset` of shared memory on: the sum of their weights, the sum and number of those
// above `above`.  Four entries at a time, side by side, in a body that is small enough for the instruction cache.
template <typename T>
__device__ __forceinline__ void dense_sums(int offset, const SampleWeight& weigh, float above, double& m_out, double& all_out, int& n_out) {
    double m = 0.0, all = 0.0;
    int n = 0;
#pragma unroll 1
    for (int h = 0; h < 8; ++h) {
        float l[4];
        if (sizeof(T) == 2) {
            const uint2 q = *shared_at<uint2>(offset + (h >> 1) * 512 + (h & 1) * 8);
            l[0] = __uint_as_float(q.x << 16); l[1] = __uint_as_float(q.x & 0xFFFF0000u);
            l[2] = __uint_as_float(q.y << 16); l[3] = __uint_as_float(q.y & 0xFFFF0000u);
        } else {
            const float4 q = *shared_at<float4>(offset + h * 512);
            l[0] = q.x; l[1] = q.y; l[2] = q.z; l[3] = q.w;
        }
        double w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = weigh(l[e]);
        all += (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool up = l[e] > above;
            w[e] = up ? w[e] : 0.0;
            n += up ? 1 : 0;
        }
        m += (w[0] + w[1]) + (w[2] + w[3]);
    }
    m_out = m;
    all_out = all;
    n_out = n;
}

// One row, seen by one CTA of its cluster.
template <typename T> struct SampleRow {
    using K = Key<T>;
    static constexpr int VEC = ChunkRegs<T>::VEC, NVEC = ChunkRegs<T>::NVEC;
    using Places = SamplePlaces<T>;
    Slice<T> s;
    uint32_t rank, ranks;
    int V, nch, mis, tid, lane, warp, first_chunk, data_at;
    float c32, top;                 // scale, largest logit
    double rT, Z;
    SampleWeight weight;
    bool exact;                     // Z is
    int at;                         // copies to use next

    __device__ __forceinline__ SampleRecord* record() const { return shared_at<SampleRecord>(Places::RECORD); }
    __device__ __forceinline__ double* part() const { return shared_at<double>(Places::part(nch)); }
    __device__ __forceinline__ int* ties() const { return shared_at<int>(Places::ties(nch)); }
    __device__ __forceinline__ double* mass() const { return shared_at<double>(Places::mass(nch)); }
    __device__ __forceinline__ float* group_max() const { return shared_at<float>(Places::group_max(nch)); }
    __device__ __forceinline__ SampleEntry* list() const { return shared_at<SampleEntry>(Places::LIST); }
    __device__ __forceinline__ SampleSorted* sorted() const { return shared_at<SampleSorted>(Places::SORTED); }
    __device__ __forceinline__ SampleFound* found() const { return shared_at<SampleFound>(Places::FOUND); }     // for the peers
    __device__ __forceinline__ double (*scan() const)[2] { return reinterpret_cast<double (*)[2]>(shared_at<double>(Places::SCAN)); }
    __device__ __forceinline__ int* ints() const { return shared_at<int>(Places::INTS); }
    __device__ __forceinline__ const unsigned char* chunk(int c) const { return shared_at<unsigned char>(data_at + c * CHUNK * (int)sizeof(T)); }

    // Vector j of the lane in chunk c (ChunkRegs' order): entries behind the row are -inf; entry e of it lies at place(o + e) of
    // the chunk's memory, o = (j * 32 + lane) * VEC.
    __device__ __forceinline__ int place(int o) const { return o < mis ? o + CHUNK : o; }
    __device__ __forceinline__ uint4 vec(int c, int j) const {
        const unsigned char* p = chunk(c);
        const int o = (j * 32 + lane) * VEC, v0 = s.begin + c * CHUNK, end = V + mis;
        uint4 q = *reinterpret_cast<const uint4*>(p + o * (int)sizeof(T));
        if (mis == 0 && v0 + CHUNK <= end) return q;        // (the same for the warp)
        const uint32_t none = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
        if (v0 + o >= end) q = make_uint4(none, none, none, none);
        if (mis && o == 0) {
            uint4 n = make_uint4(none, none, none, none);
            if (v0 + CHUNK < end) n = *reinterpret_cast<const uint4*>(p + CHUNK * (int)sizeof(T));
            ChunkRegs<T> r;
            uint32_t* w = reinterpret_cast<uint32_t*>(&r);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
            splice_granule(r, n, mis);
            q = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return q;
    }
    // The lane's entries of chunk c with low <= entry <= high: bit j * VEC + e.
    __device__ __forceinline__ uint32_t hits(int c, float low, float high) const {
        const bool any = group_max()[c * 32 + lane] >= low;
        if (!__any_sync(0xffffffffu, any)) return 0u;
        const bool open = !(high < top);
        uint32_t m = 0u;
#pragma unroll
        for (int j = 0; j < NVEC; ++j) m |= granule_between(vec(c, j), low, high, open, (const T*)nullptr) << (j * VEC);
        return m;
    }
    // f(logit, index in the vocabulary) for each of them
    template <typename F> __device__ __forceinline__ void for_hits(int c, uint32_t m, F&& f) const {
        const unsigned char* data = chunk(c);
        while (m) {
            const int b = __ffs((int)m) - 1;
            m &= m - 1u;
            const int p = place((b / VEC * 32 + lane) * VEC + b % VEC);
            f(entry_value(data, p, (const T*)nullptr), (first_chunk + c) * CHUNK + p - mis);
        }
        __syncwarp();
    }

    // x = (top - l) log2(e) / T, monotone in l
    __device__ __forceinline__ float distance(float l, float off) const {
        return offset_ok(off) ? fmaxf(0.0f, fmaf(-l, c32, off)) : l == top ? 0.0f : CUDART_INF_F;
    }

    __device__ __forceinline__ uint32_t* bins(int i) const { return shared_at<uint32_t>(Places::BINS) + (at * 2 + i) * SAMPLE_BINS; }
    // inclusive prefix sums of two doubles per thread over the CTA, and the totals; contains two barriers
    __device__ __forceinline__ void scan_pair(double& x, double& y, double& all_x, double& all_y) const {
        x = warp_scan(x, lane);
        y = warp_scan(y, lane);
        if (lane == 31) scan()[warp][0] = x, scan()[warp][1] = y;
        __syncthreads();
        double bx = 0.0, by = 0.0;
        all_x = all_y = 0.0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const double tx = scan()[w][0], ty = scan()[w][1];
            if (w < warp) bx += tx, by += ty;
            all_x += tx;
            all_y += ty;
        }
        __syncthreads();
        x += bx;
        y += by;
    }
    // the smallest of the threads' values, seen by all; two barriers
    __device__ __forceinline__ int smallest(int v) const {
        v = __reduce_min_sync(0xffffffffu, v);
        int* part = reinterpret_cast<int*>(scan());
        if (lane == 0) part[warp] = v;
        __syncthreads();
        int r = part[0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) r = min(r, part[w]);
        __syncthreads();
        return r;
    }

    __device__ __forceinline__ void smallest_pair(int a, int b, int& min_a, int& min_b) const {
        a = __reduce_min_sync(0xffffffffu, a);
        b = __reduce_min_sync(0xffffffffu, b);
        int2* part = reinterpret_cast<int2*>(scan());
        if (lane == 0) part[warp] = make_int2(a, b);
        __syncthreads();
        int2 r = part[0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) {
            const int2 o = part[w];
            r.x = min(r.x, o.x);
            r.y = min(r.y, o.y);
        }
        __syncthreads();
        min_a = r.x;
        min_b = r.y;
    }
    // exclusive prefix sum of a number per thread over the CTA; two barriers
    __device__ __forceinline__ int scan_before(int n) const {
        int x = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        int* part = reinterpret_cast<int*>(scan());
        if (lane == 31) part[warp] = x;
        __syncthreads();
        int base = 0;
#pragma unroll
        for (int w = 0; w < WARPS - 1; ++w) base += w < warp ? part[w] : 0;
        __syncthreads();
        return base + x - n;
    }

    // The barrier at the end of a pass.  `clear`: the bins of the copy that comes next are cleared.
    __device__ __forceinline__ int end_pass() {
        cluster_sync();
        const int t = at;
        at ^= 1;
        uint32_t* next = bins(0);
        for (int i = tid; i < 2 * SAMPLE_BINS; i += THREADS) next[i] = 0u;
        return t;
    }
    // this thread's bins 2 tid and 2 tid + 1 of copy t, of the whole cluster
    __device__ __forceinline__ uint2 gather(int t, int i) const {
        const uint32_t* mine = shared_at<uint32_t>(Places::BINS) + (t * 2 + i) * SAMPLE_BINS + 2 * tid;
        uint2 v[SAMPLE_CLUSTER];
#pragma unroll
        for (uint32_t r = 0; r < SAMPLE_CLUSTER; ++r) v[r] = r < ranks ? peer_load2(peer_addr(mine, r)) : make_uint2(0u, 0u);
        uint2 sum = v[0];
#pragma unroll
        for (uint32_t r = 1; r < SAMPLE_CLUSTER; ++r) sum.x += v[r].x, sum.y += v[r].y;
        return sum;
    }
    // what the CTAs found in the pass of copy t: a lane asks one of them
    __device__ __forceinline__ uint2 numbers(int t) const {
        return lane < (int)ranks ? peer_load2(peer_addr(&found()[t].n_above, (uint32_t)lane)) : make_uint2(0u, 0u);
    }
    __device__ __forceinline__ int number_above(int t) const { return (int)__reduce_add_sync(0xffffffffu, numbers(t).x); }
    __device__ __forceinline__ void take_total(int t) {
        Z = warp_sum(lane < (int)ranks ? peer_load_f64(peer_addr(&found()[t].total, (uint32_t)lane)) : 0.0);
        exact = true;
    }
    // a chunk's results to every CTA (by a warp)
    __device__ __forceinline__ void publish(int c, double m, int n) const {
        const int i = at * nch + first_chunk + c;
        if (lane < (int)ranks) {
            peer_store(peer_addr(part() + i, lane), m);
            peer_store(peer_addr(ties() + i, lane), (uint32_t)n);
        }
    }
    // masses of copy t added to the row's, or taken as the row's; and their sum
    __device__ __forceinline__ double put_together(int t, bool add) {
        double m = 0.0;
        for (int c = tid; c < nch; c += THREADS) {
            const double x = part()[t * nch + c] + (add ? mass()[c] : 0.0);
            mass()[c] = x;
            m += x;
        }
        double none = 0.0, all, unused;
        scan_pair(m, none, all, unused);
        return all;
    }

    // the first n entries of the list into the chunks' masses, in the list's order
    __device__ __forceinline__ void add_listed(int n) const {
        for (int c = tid; c < nch; c += THREADS) {
            double x = 0.0;
#pragma unroll 4
            for (int i = 0; i < n; ++i) x += sorted()[i].index / CHUNK == c ? sorted()[i].weight : 0.0;
            mass()[c] += x;
        }
        __syncthreads();
    }

    // All weights of the slice in double precision: the mass and number of entries above key `ktop`, per chunk to everyone;
    // bins of the keys in [klow, ktop] (shift -1: none); the total.
    __device__ __forceinline__ int exact_pass_body(uint32_t ktop, uint32_t klow, int shift, bool masses) {
        const float above = K::value(ktop), low = K::value(klow);
        const SampleWeight weigh = weight;
        double sum_above = 0.0, sum_all = 0.0;
        int n_above = 0;
        uint32_t *counts = bins(0), *shares = bins(1);
        for (int c = warp; c < s.chunks; c += WARPS) {
            // (where the weight's cut is the lowest logit there is -- the largest is, or the temperature is 1e35 and more --, -inf would
            // weigh what that does)
            const bool plain = mis == 0 && s.begin + (c + 1) * CHUNK <= V && weigh.cut > K::value(K::LOWEST);
            double m = 0.0, all = 0.0;
            int n = 0;
            const uint32_t inside = shift >= 0 ? hits(c, low, above) : 0u;
            if (plain) {
                dense_sums<T>(data_at + c * CHUNK * (int)sizeof(T) + lane * 16, weigh, above, m, all, n);
            } else {
#pragma unroll 1
                for (int j = 0; j < NVEC; ++j) {
                    float l[VEC];
                    unpack_granule(vec(c, j), l, (const T*)nullptr);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const double w = l[e] > -CUDART_INF_F ? weigh(l[e]) : 0.0;
                        all += w;
                        if (l[e] > above) m += w, ++n;
                    }
                }
            }
            for_hits(c, inside, [&](float l, int) { count_in_bin(l, ktop, shift, masses, counts, shares); });
            m = warp_sum(m);
            all = warp_sum(all);
            sum_above += m;
            sum_all += all;
            n_above += n;
            publish(c, m, 0);
        }
        n_above = __reduce_add_sync(0xffffffffu, n_above);
        if (lane == 0) scan()[warp][0] = sum_above, scan()[warp][1] = sum_all, ints()[warp] = n_above;
        __syncthreads();
        if (tid == 0) {
            SampleFound f{};
            for (int w = 0; w < WARPS; ++w) f.above += scan()[w][0], f.total += scan()[w][1], f.n_above += ints()[w];
            found()[at] = f;
        }
        return end_pass();
    }
    __device__ __forceinline__ void count_in_bin(float l, uint32_t ktop, int shift, bool masses, uint32_t* counts, uint32_t* shares) const {
        const uint32_t b = (ktop - K::of(l)) >> shift;
        if (b >= (uint32_t)SAMPLE_BINS) return;         // (not reached: l lies between the ends)
        atomicAdd(&counts[b], 1u);
        if (shift > 0 && masses) {          // a share of the bin's largest weight, in steps of 2^-12, rounded up
            const float most = K::value(ktop - (b << shift));
            atomicAdd(&shares[b], (uint32_t)fminf(4096.0f, ceilf(ex2_approx((l - most) * c32) * 4096.0f)));
        }
    }
    // bins of the keys in [klow, ktop]
    __device__ __forceinline__ int count_pass(uint32_t ktop, uint32_t klow, int shift, bool masses) {
        const float low = K::value(klow), high = K::value(ktop);
        uint32_t *counts = bins(0), *shares = bins(1);
        for (int c = warp; c < s.chunks; c += WARPS)
            for_hits(c, hits(c, low, high), [&](float l, int) { count_in_bin(l, ktop, shift, masses, counts, shares); });
        return end_pass();
    }
    // Exact masses of the entries with khi < key <= ktop per chunk, to everyone, and per chunk the number of those with klo <= key
    // <= khi; or, `listed`, those themselves in this CTA's list.  ktop >= khi >= klo.
    __device__ __forceinline__ int mass_pass(uint32_t ktop, uint32_t khi, uint32_t klo, bool listed) {
        const float low = K::value(klo), split = K::value(khi), high = K::value(ktop);
        if (listed) {
            if (tid == 0) found()[at].listed = 0;
            __syncthreads();
        }
        for (int c = warp; c < s.chunks; c += WARPS) {
            const uint32_t h = hits(c, low, high);
            double m = 0.0;
            int n = 0;
            const auto one = [&](float l, int index) {
                if (l > split) {
                    m += weight(l);
                } else {
                    ++n;
                    if (listed) {
                        const int i = atomicAdd(&found()[at].listed, 1);
                        if (i < SAMPLE_LIST) list()[at * SAMPLE_LIST + i] = SampleEntry{K::of(l), index};
                    }
                }
            };
            if (!listed && __reduce_max_sync(0xffffffffu, (unsigned)__popc(h)) > SAMPLE_DENSE_HITS) {
#pragma unroll 1
                for (int j = 0; j < NVEC; ++j) {
                    float l[VEC];
                    unpack_granule(vec(c, j), l, (const T*)nullptr);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const double w = weight(l[e]);
                        if (l[e] > split) m += l[e] <= high ? w : 0.0;
                        else if (l[e] >= low) ++n;
                    }
                }
            } else {
                for_hits(c, h, one);
            }
            publish(c, warp_sum(m), (int)__reduce_add_sync(0xffffffffu, (unsigned)n));
        }
        return end_pass();
    }
    __device__ __forceinline__ int exact_pass(uint32_t ktop, uint32_t klow, int shift, bool masses);
    // Z from double-precision weights.  May come while the results of the pass before are still needed: the pass behind it uses
    // the same copy as this one, behind a barrier of its own.
    __device__ __forceinline__ void exact_total() {
        const int t = exact_pass(K::LOWEST, K::LOWEST, -1, false);
        take_total(t);
        cluster_sync();
        at = t;
    }
};

// A call of its own, on a copy of the row's state: three places make it, and its unrolled exponentials are half of the kernel.
template <typename T> __device__ __noinline__ int exact_pass_call(SampleRow<T>* row, uint32_t ktop, uint32_t klow, int shift, bool masses) {
    SampleRow<T> mine = *row;
    return mine.exact_pass_body(ktop, klow, shift, masses);
}
template <typename T>
__device__ __forceinline__ int SampleRow<T>::exact_pass(uint32_t ktop, uint32_t klow, int shift, bool masses) {
    SampleRow<T> copy = *this;
    const int t = exact_pass_call(&copy, ktop, klow, shift, masses);
    at = t ^ 1;
    return t;
}

// The end of the prefix among `count` entries of weight w at each of the thread's two places, in order; `before` and
// `mass_before` of them lie ahead.
struct SampleEnd {
    int place;          // of the first entry that is not kept; NONE: all are
    int keep, count;    // how many of its place are; kept in all
    bool reached;       // with all of the entries kept, a limit is reached, and the prefix ends here at the latest
};
// Where the mass decides, with Z as it is known: made exact where the outcome depends on its error.
template <typename T>
__device__ __forceinline__ SampleEnd end_of_prefix(SampleRow<T>& row, const SampleLimits& lim, const uint32_t count[2], const double w[2],
                                                   long long before, double mass_before) {
    double n = (double)count[0] + (double)count[1], m = (double)count[0] * w[0] + (double)count[1] * w[1], n_all, m_all;
    const double n_here = n, m_here = m;
    row.scan_pair(n, m, n_all, m_all);
    const double mass = mass_before + m_all;
    for (;;) {
        const double g = row.exact || lim.p >= 1.0 ? 0.0 : GUARD_Z, pz = lim.p * row.Z;
        // with pz at the lower and at the upper end of its error
        int first[2] = {NONE, NONE}, kept_here[2] = {0, 0}, kept_n[2] = {0, 0};
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const double at = side ? pz * (1.0 + g) : pz * (1.0 - g);
            double nb = (double)before + n - n_here, mb = mass_before + m - m_here;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                double keep = (double)count[i];
                keep = fmin(keep, fmax(0.0, (double)lim.k - nb));
                if (lim.p < 1.0 && count[i] && mb + (double)count[i] * w[i] >= at)
                    keep = fmin(keep, mb >= at ? 0.0 : w[i] > 0.0 ? ceil((at - mb) / w[i]) : keep);
                if (nb == 0.0 && count[i]) keep = fmax(keep, 1.0);      // the first entry is kept whatever the limits
                if (count[i] && keep < (double)count[i] && first[side] == NONE) {
                    first[side] = 2 * row.tid + i;
                    kept_here[side] = (int)keep;
                    kept_n[side] = (int)(nb + keep);
                }
                nb += (double)count[i];
                mb += (double)count[i] * w[i];
            }
        }
        SampleEnd e[2];
        row.smallest_pair(first[0], first[1], e[0].place, e[1].place);
#pragma unroll
        for (int side = 0; side < 2; ++side)
            if (first[side] != NONE && first[side] == e[side].place) row.ints()[2 * side] = kept_here[side], row.ints()[2 * side + 1] = kept_n[side];
        __syncthreads();
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const bool all = e[side].place == NONE;
            e[side].keep = all ? 0 : row.ints()[2 * side];
            e[side].count = all ? (int)((double)before + n_all) : row.ints()[2 * side + 1];
        }
        __syncthreads();
        e[0].reached = e[0].count >= lim.k || (lim.p < 1.0 && mass >= pz);
        if (g == 0.0 || (e[0].place == e[1].place && e[0].keep == e[1].keep && (e[0].place != NONE || fabs(mass - pz) > g * pz))) return e[0];
        row.exact_total();
    }
}

// Where to look for the end of the prefix: its last key lies in [klow, ktop].
struct SampleBracket {
    uint32_t ktop, klow;
    bool sure;          // else a guess from a sample, with many entries above ktop
};
// From the largest entry of each group of 32: k of them, or the share p of the mass, at or above a value bound the prefix to it.
// A prefix of more entries than that is bracketed by a sample of one entry in 32: by its counts for top-k, for top-p by the mass
// that it finds below a value, each within four and a half standard deviations and a few entries.
template <typename T>
__device__ __forceinline__ SampleBracket bracket(SampleRow<T>& row, const SampleLimits& lim, uint32_t floor_key) {
    using K = Key<T>;
    constexpr float STEPS = 16.0f;          // bins per factor of two
    const float off = __fmul_rn(row.top, row.c32);
    uint32_t *groups = row.bins(0), *samples = row.bins(1);
    for (int c = row.warp; c < row.s.chunks; c += WARPS) {
        const float g = row.group_max()[c * 32 + row.lane];
        if (g > -CUDART_INF_F) {
            const float x = row.distance(g, off) * STEPS;
            if (x < (float)SAMPLE_BINS) atomicAdd(&groups[(int)x], 1u);
        }
        const int e = row.lane * 32 + ((row.lane * 7 + c * 11) & 31);
        if ((row.first_chunk + c) * CHUNK + e < row.V) {
            const float l = entry_value(row.chunk(c), e + row.mis, (const T*)nullptr);
            if (l > -CUDART_INF_F) atomicAdd(&samples[(int)fminf(row.distance(l, off) * STEPS, (float)(SAMPLE_BINS - 1))], 1u);
        }
    }
    const int t = row.end_pass();
    const uint2 g = row.gather(t, 0);
    double w[2], n = (double)g.x + (double)g.y, n_all, m_all;
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = (double)exp2f(-(float)(2 * row.tid + i + 1) / STEPS);        // at least
    double m = (double)g.x * w[0] + (double)g.y * w[1];
    row.scan_pair(n, m, n_all, m_all);
    const double want = lim.p * row.Z * (1.0 + 1e-4);
    int first = NONE;
    if (n >= (double)lim.k || (lim.p < 1.0 && m >= want)) first = 2 * row.tid + 1;
    if (n - (double)g.y >= (double)lim.k || (lim.p < 1.0 && m - (double)g.y * w[1] >= want)) first = 2 * row.tid;
    first = row.smallest(first);
    // a key that the entries within x of the top reach, down by more than the roundings of x and of the division
    const auto key_at = [&](double x) {
        const double low = (double)row.top - (x * (1.0 + 1e-5) + 1e-4) / (double)row.c32 - fabs((double)row.top) * 1e-6;
        return low > -3.3e38 ? max(K::of(__double2float_rd(low)), floor_key) : floor_key;
    };
    SampleBracket b;
    b.ktop = K::of(row.top);
    b.sure = true;
    if (first != NONE) {
        b.klow = min(key_at((double)(first + 1) / STEPS), b.ktop);
        return b;
    }
    // the sample: numbers at or above the end of bin i, mass and its variance below it
    const uint2 q = row.gather(t, 1);
    double s = (double)q.x + (double)q.y, s_all, f = 0.0, f_all, v_all, v;
    const double mid = exp2(0.5 / (double)STEPS);
    s = (double)q.x + (double)q.y;
    f = ((double)q.x * w[0] + (double)q.y * w[1]) * mid;
    v = ((double)q.x * w[0] * w[0] + (double)q.y * w[1] * w[1]) * mid * mid;
    double unused = 0.0, unused_all;
    const double f_here = f, v_here = v, s_here = s;
    row.scan_pair(s, f, s_all, f_all);
    row.scan_pair(v, unused, v_all, unused_all);
    double sb = s - s_here, fb = f - f_here, vb = v - v_here;
    int low = NONE, high = -1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const double cnt = i ? (double)q.y : (double)q.x;
        sb += cnt;
        fb += cnt * w[i] * mid;
        vb += cnt * w[i] * w[i] * mid * mid;
        const int bin = 2 * row.tid + i;
        if (bin == SAMPLE_BINS - 1) break;              // (open)
        const double dev = 4.5 * sqrt(sb) + 6.0, tail = 32.0 * (f_all - fb), spread = 32.0 * (4.5 * sqrt(fmax(0.0, v_all - vb)) + 6.0 * w[i]);
        const double rest = (1.0 - lim.p) * row.Z;
        const bool not_yet = 32.0 * (sb + dev) < (double)lim.k && (lim.p >= 1.0 || tail * 0.99 - spread > rest);
        const bool surely = 32.0 * (sb - dev) >= (double)lim.k || (lim.p < 1.0 && tail * 1.01 + spread <= rest);
        if (surely && low == NONE) low = bin;
        if (not_yet) high = bin;
    }
    low = row.smallest(low);
    high = -row.smallest(-high);        // (not_yet holds up to one bin and no further, by and large)
    b.klow = low != NONE ? min(key_at((double)(low + 1) / STEPS), b.ktop) : floor_key;
    if (high >= 0 && (low == NONE || high < low)) {
        const double value = (double)row.top - (double)(high + 1) / (double)STEPS / (double)row.c32;
        const uint32_t k = value > -3.3e38 ? K::of(__double2float_rd(value)) : floor_key;
        if (k >= b.klow && k < b.ktop) {
            b.ktop = k;
            b.sure = false;
        }
    }
    if (low != NONE) b.sure = false;
    return b;
}

// The cut; row.mass() holds the chunk masses of the kept entries with a larger key afterwards, copy `t` of the ties the number
// of entries with the cut's key per chunk (not listed) (those of a list are in the masses).
template <typename T>
__device__ __forceinline__ SampleCut find_cut(SampleRow<T>& row, const SampleLimits& lim, int& ties_at) {
    using K = Key<T>;
    const bool by_mass = lim.p < 1.0;
    uint32_t ktop = K::of(row.top), klow = lim.key;
    long long before = 0;
    double mass_before = 0.0;
    if (lim.k == NONE && !by_mass) {            // min-p alone: the end is known
        ties_at = row.mass_pass(ktop, klow, klow, false);
        row.put_together(ties_at, false);
        int n = 0;
        // the entries above the bound are counted by their own pass over the slice
        for (int c = row.warp; c < row.s.chunks; c += WARPS) n += __popc(row.hits(c, K::value(klow), row.top));
        n = (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
        if (row.lane == 0) row.ints()[row.warp] = n;
        __syncthreads();
        if (row.tid == 0) {
            int all = 0;
            for (int w = 0; w < WARPS; ++w) all += row.ints()[w];
            row.found()[row.at].n_above = all;
        }
        const int t = row.end_pass();
        return SampleCut{klow, NONE, 0, row.number_above(t), false};
    }
    SampleBracket b = bracket(row, lim, klow);
    uint32_t floor_key = klow;              // no entry of the prefix lies below
    ktop = b.ktop;
    klow = b.klow;
    for (int c = row.tid; c < row.nch; c += THREADS) row.mass()[c] = 0.0;
    const auto whole_range = [&]() {        // the bracket was wrong
        ktop = K::of(row.top);
        klow = floor_key;
        before = 0;
        mass_before = 0.0;
        b.sure = true;
        for (int c = row.tid; c < row.nch; c += THREADS) row.mass()[c] = 0.0;
        __syncthreads();
    };
    // What lies above `key` is kept, and in the masses already; nothing has that key, and no pass counted ties.
    const auto above_only = [&](uint32_t key) { return SampleCut{key, 0, -1, (int)before, true}; };
    // Each turn leaves one bin of the range, leaves out one at least, or is the only one that takes back the bracket.
    for (int turn = 0; turn < MAX_TURNS; ++turn) {
        if (lower_end<T>(klow) > upper_end<T>(ktop)) return above_only(ktop);      // (nothing is left: all that lies above is kept)
        klow = lower_end<T>(klow);
        ktop = upper_end<T>(ktop);
        int shift = 0;
        while (((ktop - klow) >> shift) >= (uint32_t)SAMPLE_BINS) ++shift;
        int t;
        if (!b.sure && turn == 0) {
            t = row.exact_pass(ktop, klow, shift, by_mass);
            row.take_total(t);
            mass_before = row.put_together(t, false);
            before = row.number_above(t);
        } else {
            t = row.count_pass(ktop, klow, shift, by_mass);
        }
        const uint2 c2 = row.gather(t, 0);
        uint2 m2 = make_uint2(0u, 0u);
        if (by_mass && shift > 0) m2 = row.gather(t, 1);
        if (before >= lim.k || (by_mass && row.exact && before > 0 && mass_before >= lim.p * row.Z)) {
            whole_range();          // (the prefix ends above)
            continue;
        }
        const uint32_t count[2] = {c2.x, c2.y};
        double w[2];
        if (shift == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = count[i] ? row.weight(K::value(ktop - (uint32_t)(2 * row.tid + i))) : 0.0;
            const SampleEnd e = end_of_prefix(row, lim, count, w, before, mass_before);
            if (e.place == NONE && !e.reached && klow != floor_key) {
                whole_range();
                continue;
            }
            const uint32_t key = e.place == NONE ? klow : ktop - (uint32_t)e.place;
            ties_at = row.mass_pass(ktop, key, key, false);
            row.put_together(ties_at, true);
            return SampleCut{key, e.place == NONE ? NONE : e.keep, 0, e.count, false};
        }
        // the bin in which the prefix ends, by the masses of the bins
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t bin = (uint32_t)(2 * row.tid + i);
            w[i] = by_mass && count[i] ? (double)(i ? m2.y : m2.x) * (1.0 / 4096.0) * row.weight(K::value(ktop - (bin << shift))) : 0.0;
        }
        double n = (double)count[0] + (double)count[1], m = w[0] + w[1], n_all, m_all;
        const double n_here = n, m_here = m;
        row.scan_pair(n, m, n_all, m_all);
        double nb = (double)before + n - n_here, mb = mass_before + m - m_here;
        const double nb_first = nb;
        int first = NONE, by_count = NONE, last = NONE;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (count[i]) {
                const int bin = 2 * row.tid + i;
                const bool full = nb + (double)count[i] >= (double)lim.k;
                if (full && by_count == NONE) by_count = bin;
                if ((full || (by_mass && mb + w[i] >= lim.p * row.Z)) && first == NONE) first = bin;
                last = -bin;
            }
            nb += (double)count[i];
            mb += w[i];
        }
        by_count = row.smallest(by_count);
        first = row.smallest(first);
        const bool all = first == NONE;
        if (all) {                      // no limit is reached, by the masses of the bins: the last bin that holds any
            if (klow != floor_key) {
                whole_range();
                continue;
            }
            first = row.smallest(last);
            if (first == NONE) return above_only(klow);
            first = -first;
        }
        if (row.tid == first / 2) {
            const uint32_t skip = first & 1 ? count[0] : 0u;
            row.ints()[0] = (int)nb_first + (int)skip;
            row.ints()[1] = (int)(first & 1 ? count[1] : count[0]);
        }
        __syncthreads();
        const int upto = row.ints()[0], in_bin = row.ints()[1];
        __syncthreads();
        const uint32_t hi_bin = ktop - ((uint32_t)first << shift);
        const uint32_t hi = upper_end<T>(hi_bin), lo = lower_end<T>(hi_bin - klow >= (1u << shift) ? hi_bin - (1u << shift) + 1u : klow);
        if (all) floor_key = klow = lo;
        const bool listed = sizeof(T) == 4 && in_bin <= SAMPLE_LIST;
        t = row.mass_pass(ktop, hi, lo, listed);
        // (sums over the row of what the pass found, without touching the row's masses yet)
        double part = 0.0, none = 0.0, above, unused;
        for (int c = row.tid; c < row.nch; c += THREADS) part += row.part()[t * row.nch + c];
        row.scan_pair(part, none, above, unused);
        above += mass_before;
        if (by_mass && !row.exact && above >= lim.p * row.Z * (1.0 - GUARD_Z) && above <= lim.p * row.Z * (1.0 + GUARD_Z)) {
            row.exact_total();          // (uses the other copy)
        }
        if (by_mass && above >= lim.p * row.Z && hi < ktop) {       // the prefix ends before this bin
            klow = hi + 1u;
            continue;
        }
        if (!listed) {
            for (int c = row.tid; c < row.nch; c += THREADS) row.mass()[c] += row.part()[t * row.nch + c];
            __syncthreads();
            mass_before = above;
            before = upto;
            // does the mass end in it?  Else only what lies behind it is left, and it counts with what lies ahead
            if (by_mass && first != by_count && lo > klow) {
                const uint32_t under = upper_end<T>(lo - 1u);
                const int t2 = row.mass_pass(hi, under, under, false);
                double in = 0.0, none2 = 0.0, all, unused2;
                for (int c = row.tid; c < row.nch; c += THREADS) in += row.part()[t2 * row.nch + c];
                row.scan_pair(in, none2, all, unused2);
                if (!row.exact && fabs(above + all - lim.p * row.Z) <= GUARD_Z * lim.p * row.Z) {
                    // (t2's copy is the other one of the exact pass's)
                    row.exact_total();
                }
                if (above + all < lim.p * row.Z) {
                    for (int c = row.tid; c < row.nch; c += THREADS) row.mass()[c] += row.part()[t2 * row.nch + c];
                    __syncthreads();
                    mass_before = above + all;
                    before = upto + in_bin;
                    ktop = lo - 1u;
                    continue;
                }
            }
            ktop = hi;
            klow = lo;
            continue;
        }
        // put the bin's entries in order: a thread per entry
        const int n_lane = (int)row.numbers(t).y;
        int offset = 0, mine = 0, from = -1;
        for (uint32_t r = 0; r < row.ranks; ++r) {
            const int n_r = __shfl_sync(0xffffffffu, n_lane, (int)r);
            if (row.tid >= offset && row.tid < offset + n_r) from = (int)r, mine = row.tid - offset;
            offset += n_r;
        }
        SampleEntry e{0u, 0};
        if (from >= 0) {
            const uint2 x = peer_load2(peer_addr(&row.list()[t * SAMPLE_LIST + mine], (uint32_t)from));
            e = SampleEntry{x.x, (int)x.y};
        }
        SampleEntry* unsorted = reinterpret_cast<SampleEntry*>(row.bins(1));        // (cleared again below)
        if (from >= 0) unsorted[row.tid] = e;
        __syncthreads();
        int place = 0;
        for (int i = 0; i < in_bin; ++i) {
            const SampleEntry o = unsorted[i];
            place += o.key > e.key || (o.key == e.key && o.index < e.index) ? 1 : 0;
        }
        if (from >= 0) row.sorted()[place] = SampleSorted{row.weight(K::value(e.key)), e.key, e.index};
        __syncthreads();
        reinterpret_cast<uint2*>(unsorted)[row.tid] = make_uint2(0u, 0u);
        __syncthreads();
        uint32_t one[2];
        double we[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            one[i] = 2 * row.tid + i < in_bin ? 1u : 0u;
            we[i] = one[i] ? row.sorted()[2 * row.tid + i].weight : 0.0;
        }
        const SampleEnd end_at = end_of_prefix(row, lim, one, we, (long long)upto, above);
        const int end = end_at.place, n_kept = end_at.count;
        if (end == NONE && !end_at.reached) {
            if (lo > klow) {            // all of the bin is kept, and more: what it holds counts with what lies ahead
                double sum = we[0] + we[1], none2 = 0.0, all, unused2;
                row.scan_pair(sum, none2, all, unused2);
                row.put_together(t, true);
                row.add_listed(in_bin);
                mass_before = above + all;
                before = upto + in_bin;
                ktop = lo - 1u;
                continue;
            }
            if (klow != floor_key) {
                whole_range();
                continue;
            }
        }
        row.put_together(t, true);
        const int list_kept = end == NONE ? in_bin : end;         // (one entry a place: those ahead of `end` are kept)
        row.add_listed(list_kept);
        const SampleSorted stop = row.sorted()[max(list_kept - 1, 0)];
        if (list_kept == 0) return SampleCut{hi, 0, -1, n_kept, true};
        return SampleCut{stop.key, 0, stop.index, n_kept, true};
    }
    return SampleCut{klow, 0, -1, -1, true};        // (not reached)
}

// One cluster per row.  Bound: a chain of seven exchanges at most, each a pass over the slice, a cluster's barrier and one or two
// scans of the CTA (1 to 2 us), while few CTAs share an SM; where all weights are taken in double precision, that pass (8 of 20 us
// a row of 262144).  256 rows of 128256 bf16 with mixed limits: 117 to 125 us by their limits, 0.54 TB/s; without limits 256 rows of 151936: 43 us,
// 1.8 TB/s.  LIMITS: some row may be truncated; without, the kernel is a third as large and keeps three CTAs
// an SM where the other has two (256 x 151936: 46 us against 52).
template <typename T, bool LIMITS>
__global__ void __launch_bounds__(THREADS, LIMITS ? 2 : 3) sample_kernel(SampleArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint64_t bars[MAX_SLICE_TILES];
    __shared__ float part_max[WARPS];
    __shared__ unsigned shared_bad[WARPS];
    using K = Key<T>;
    using Places = SamplePlaces<T>;
    SampleRow<T> row;
    row.V = a.V;
    row.nch = a.nch;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(row.ranks));
    row.rank = cluster_rank();
    row.tid = threadIdx.x; row.lane = threadIdx.x & 31; row.warp = threadIdx.x >> 5;
    row.at = 0;
    row.exact = false;
    row.data_at = Places::data(a.nch, a.slice_chunks);
    const int tid = row.tid, lane = row.lane, warp = row.warp;
    const long long r = blockIdx.x / row.ranks;
    const int b = (int)(r / a.R);
    cluster_arrive();
    shared_at<double>(Places::TABLE)[tid] = exp2((double)tid / SAMPLE_STEPS);
    static_assert(SAMPLE_STEPS == THREADS, "a step per thread");
    for (int i = tid; i < 4 * SAMPLE_BINS; i += THREADS) shared_at<uint32_t>(Places::BINS)[i] = 0u;
    row.s.init(smem + row.data_at, bars);
    __syncthreads();
    grid_dependency_sync();

    const StagedRow<T> in(reinterpret_cast<const T*>(a.logits) + r * a.row_stride, a.V);
    row.mis = in.mis;
    row.first_chunk = (int)row.rank * a.slice_chunks;
    row.s.stage(in, row.rank, a.slice_chunks, true);
    const float temperature = a.temperature[b];
    const int k = LIMITS && a.top_k ? a.top_k[b] : 0;
    const float p = LIMITS && a.top_p ? a.top_p[b] : 1.0f, m = LIMITS && a.min_p ? a.min_p[b] : 0.0f;
    row.c32 = temp_scale(temperature);
    row.rT = 1.0 / (double)temperature;
    unsigned bad = temp_ok(temperature) && row.c32 < CUDART_INF_F ? 0u : ST_TEMPERATURE;
    if (k < 0 || !(p > 0.0f) || !(m >= 0.0f && m <= 1.0f)) bad |= ST_RANGE;
    const bool limited = LIMITS && ((k > 0 && k < a.V) || p < 1.0f || m > 0.0f);

    // statistics of the chunks, to every CTA of the cluster
    cluster_wait();
    for (int c = warp; c < row.s.chunks; c += WARPS) {
        // (one outcome for the warp: each CTA of the cluster is told by another lane, and all have to give the row up, or none)
        const int late = __reduce_max_sync(0xffffffffu, row.s.wait(c, in.mis != 0, a.wait_limit_ns));
        ChunkRegs<T> x;
        load_staged_shifted(x, row.chunk(c), row.s.begin + c * CHUNK, in.end, in.mis, lane);
        const float g = x.lane_max_plain();
        row.group_max()[c * 32 + lane] = g;
        const float top = warp_max_redux(g);
        const float sum = warp_sum(lane_weight_sum(x, top, row.c32, top > -CUDART_INF_F ? __fmul_rn(top, row.c32) : 0.0f));
        int finite = 0;
        if (!limited && a.count) {
            uint32_t f = 0u;
#pragma unroll
            for (int i = 0; i < 32; ++i) f += x.value(i) > -CUDART_INF_F ? 1u : 0u;
            finite = (int)__reduce_add_sync(0xffffffffu, f);
        }
        if (late != WAIT_OK) finite = -1;
        // (a lane per CTA and word)
        for (int i = lane; i < 4 * (int)row.ranks; i += 32)
            peer_store(peer_addr(reinterpret_cast<uint32_t*>(row.record() + row.first_chunk + c) + (i & 3), i >> 2),
                       (i & 3) == 0 ? __float_as_uint(top) : (i & 3) == 1 ? __float_as_uint(sum) : (uint32_t)finite);
    }
    cluster_sync();

    float top = -CUDART_INF_F;
    for (int c = tid; c < a.nch; c += THREADS) {
        const SampleRecord x = row.record()[c];
        if (x.finite < 0) bad |= ST_INTERNAL;
        else if (x.top == CUDART_INF_F || x.sum != x.sum) bad |= ST_LOGIT;
        top = fmaxf(top, x.top);
    }
    top = warp_max_redux(top);
    bad = __reduce_or_sync(0xffffffffu, bad);
    if (lane == 0) part_max[warp] = top, shared_bad[warp] = bad;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        top = fmaxf(top, part_max[w]);
        bad |= shared_bad[w];
    }
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
    row.weight.init(top, row.rT);
    // fp32-accumulated chunk masses on the scale of the exact ones
    double z = 0.0, finite = 0.0, all_finite;
    for (int c = tid; c < a.nch; c += THREADS) {
        const SampleRecord x = row.record()[c];
        const double mass = (double)x.sum * reference_factor(x.top, top, row.c32, row.rT);
        row.mass()[c] = mass;
        z += mass;
        finite += (double)x.finite;
    }
    row.scan_pair(z, finite, row.Z, all_finite);

    SampleCut cut{K::LOWEST, NONE, 0, (int)all_finite, false};
    int ties_at = 0;
    if (limited) {
        SampleLimits lim;
        lim.k = k > 0 && k < a.V ? k : NONE;
        lim.p = (double)p;
        lim.key = K::LOWEST;
        if (m > 0.0f) {
            // the lowest key whose weight reaches min_p, compared by their logarithms (exp would round weights next to 1 to 1): the
            // threads ask the keys around top + T ln min_p, and where that is not among them (next to the lowest values, or next to
            // zero, where many values are one in their difference to top) evenly spaced keys of what is left
            const double log_m = log((double)m), at = (double)top + log_m / row.rT;
            const uint32_t about = at > -3.3e38 ? K::of((float)at) : K::LOWEST, most = K::of(top);
            const uint32_t from = max(K::LOWEST, min(about, most) - min(min(about, most), (uint32_t)THREADS / 2));
            const auto first_of = [&](uint32_t begin, uint32_t step) {      // (`most` reaches it)
                const unsigned long long key = min(begin + (unsigned long long)step * tid, (unsigned long long)most);
                return row.smallest(((double)K::value((uint32_t)key) - (double)top) * row.rT >= log_m ? tid : NONE);
            };
            int first = first_of(from, 1u);
            uint32_t low = from + (uint32_t)first, high = low;              // it lies between these
            if (first == NONE) low = from + THREADS, high = most;
            else if (first == 0) low = K::LOWEST, high = from;
            while (low < high) {
                const uint32_t step = (high - low) / THREADS + 1u;
                first = first_of(low, step);
                const uint32_t reaches = first == NONE ? high : min(high, low + (uint32_t)first * step);
                if (first != 0) low += (first == NONE ? (uint32_t)THREADS - 1u : (uint32_t)first - 1u) * step + 1u;
                high = reaches;
            }
            lim.key = lower_end<T>(high);
        }
        cut = find_cut<T>(row, lim, ties_at);
        if (cut.count < 0 && tid == 0) atomicOr(a.status, ST_INTERNAL);
        // A CTA's shared memory may be read by its peers for as long as it runs, and the last pass, whichever it was, is followed by such
        // reads: all of them lie ahead of this arrival (for rows without limits, which may take one more pass, of the one below), and no
        // CTA ends before every CTA has arrived.
        cluster_arrive();
    }

    // level 1: a thread per stretch of chunks
    const float u0 = a.u[2 * r], u1 = a.u[2 * r + 1];
    const int stretch = (a.nch + THREADS - 1) / THREADS, c0 = min(tid * stretch, a.nch), c1 = min(c0 + stretch, a.nch);
    const bool by_ties = limited && !cut.listed;
    if (by_ties) {              // the cut's own entries into the chunks' masses
        const double cut_weight = row.weight(K::value(cut.key));
        const int* ties = row.ties() + ties_at * a.nch;
        int n = 0;
        for (int c = c0; c < c1; ++c) n += ties[c];
        int before = row.scan_before(n);
        for (int c = c0; c < c1; ++c) {
            const int t = ties[c], kept = max(0, min(t, cut.ties - before));
            row.mass()[c] += (double)kept * cut_weight;
            row.ties()[(ties_at ^ 1) * a.nch + c] = kept;
            before += t;
        }
    }
    double W;
    int chunk;
    for (;;) {
        double mine = 0.0, none = 0.0, unused;
        for (int c = c0; c < c1; ++c) mine += row.mass()[c];
        double upto = mine;
        row.scan_pair(upto, none, W, unused);
        upto -= mine;
        const double target = (double)u0 * W, guard = limited || row.exact ? 0.0 : GUARD_Z * W;
        int first = NONE, last = NONE, close = 0;
        for (int c = c0; c < c1; ++c) {
            const double x = row.mass()[c];
            upto += x;
            if (x > 0.0) {
                if (upto > target && first == NONE) first = c;
                last = -c;
            }
            if (guard > 0.0 && fabs(upto - target) <= guard) close = 1;
        }
        if (guard > 0.0 && __syncthreads_or(close)) {           // (rows without limits)
            const uint32_t lowest = K::LOWEST - 1u;     // every finite entry lies above
            const int t = row.exact_pass(lowest, lowest, -1, false);
            row.take_total(t);
            row.put_together(t, false);
            continue;
        }
        chunk = row.smallest(first);
        if (chunk == NONE) chunk = -row.smallest(last);         // (the last rounding)
        break;
    }
    const bool asked = limited || row.exact;        // (a row without limits that took no more passes has read nothing since the last barrier)
    if (!limited && row.exact) cluster_arrive();
    if (row.exact && row.rank == 0 && tid == 0) atomicAdd(a.slow_rows, 1ull);

    // level 2: by the CTA that holds the chunk
    const int local = chunk - row.first_chunk;
    if (local < 0 || local >= row.s.chunks) {
        if (asked) cluster_wait();
        return;
    }
    const int chunk_ties = by_ties ? row.ties()[(ties_at ^ 1) * a.nch + chunk] : 0;
    float l[4];
    bool keep[4], tie[4];
    int n_tie = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int v = chunk * CHUNK + 4 * tid + i;
        l[i] = v < a.V ? entry_value(row.chunk(local), in.mis + 4 * tid + i, (const T*)nullptr) : -CUDART_INF_F;
        const uint32_t key = K::of(l[i]);
        tie[i] = limited && key == cut.key && l[i] > -CUDART_INF_F;
        keep[i] = l[i] > -CUDART_INF_F && (!limited || key > cut.key || (tie[i] && cut.listed && v <= cut.index));
        n_tie += tie[i] ? 1 : 0;
    }
    if (by_ties) {
        int before = row.scan_before(n_tie);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (tie[i]) keep[i] = before++ < chunk_ties;
    }
    double w[4], sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = keep[i] ? row.weight(l[i]) : 0.0;
        sum += w[i];
    }
    double upto = sum, none = 0.0, total, unused;
    row.scan_pair(upto, none, total, unused);
    upto -= sum;
    const double target = (double)u1 * total;
    int first = NONE, last = NONE;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        upto += w[i];
        if (w[i] > 0.0) {
            if (upto > target && first == NONE) first = 4 * tid + i;
            last = -(4 * tid + i);
        }
    }
    first = row.smallest(first);
    if (first == NONE) first = -row.smallest(last);
    if (tid == first / 4) {
        double wi = 0.0, li = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * tid + i == first) wi = w[i], li = (double)l[i];
        a.token[r] = chunk * CHUNK + first;
        if (a.prob) a.prob[r] = (float)(wi / W);
        if (a.logprob) a.logprob[r] = (float)((li - (double)top) * row.rT - log(row.Z));
        if (a.count) a.count[r] = cut.count;
    }
    __syncwarp();
    if (asked) cluster_wait();
}

inline int sample_smem(int slice_chunks, int nch, int elem) {
    return elem == 2 ? SamplePlaces<__nv_bfloat16>::total(nch, slice_chunks) : SamplePlaces<float>::total(nch, slice_chunks);
}

}  // namespace picospec
