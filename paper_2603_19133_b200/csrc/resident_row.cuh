// Rows of logits held in the shared memory of a thread-block cluster.  Work that has to look at a row several times (a
// softmax and its gradient, a selection and a draw) reads it from HBM once: every CTA of the cluster stages a slice of
// the row by bulk copies, all of them issued at once, and the CTAs exchange their sums through distributed shared memory.
#pragma once
#include "stream_pipeline.cuh"

namespace picospec {

constexpr int MAX_CLUSTER = 16;                 // (beyond 8 a kernel has to opt in)
constexpr int MAX_SLICE_TILES = 16;

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// every thread of every CTA of the cluster; writes to distributed shared memory before it are visible behind it
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The barrier in two halves, for the start of a kernel: a CTA's shared memory may be accessed by its peers only once it
// runs.  (cluster_wait comes before the first access.)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// the address of this CTA's shared-memory word `p` in the CTA of rank `rank`
__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void peer_store(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void peer_store(uint32_t addr, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
}
__device__ __forceinline__ void peer_store4(uint32_t addr, uint4 v) {
    asm volatile("st.shared::cluster.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint2 peer_load2(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ double peer_load_f64(uint32_t addr) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}

// One CTA's part of a row: `chunks` chunks of 1024 virtual entries (StagedRow) from entry `begin` on.  Tiles are of eight
// chunks, one per warp, each with a barrier of its own, so that a warp starts on a tile as soon as it has landed.
template <typename T> struct Slice {
    const unsigned char* data;      // shared memory
    uint64_t* bars;                 // [MAX_SLICE_TILES]
    int begin, end;                 // virtual entries of the slice
    int chunks, tiles;
    // The barriers, before anything is known of the row.  Called by every thread; a barrier of the CTA has to follow.
    __device__ __forceinline__ void init(unsigned char* smem, uint64_t* barriers) {
        data = smem;
        bars = barriers;
        if (threadIdx.x < MAX_SLICE_TILES) {
            mbar_init(&bars[threadIdx.x], 1);
            mbar_init_fence();
        }
    }
    // `shifted`: the slice is of whole vocabulary chunks, which begin StagedRow::mis entries behind the virtual ones, so
    // one more granule is staged behind the last.
    __device__ __forceinline__ void locate(const StagedRow<T>& row, uint32_t rank, int slice_chunks, bool shifted) {
        const int last = shifted ? row.end - row.mis : row.end;        // (vocabulary chunks end with the vocabulary)
        begin = min((int)rank * slice_chunks * CHUNK, row.end);
        chunks = max(0, min(slice_chunks, (last + CHUNK - 1) / CHUNK - (int)rank * slice_chunks));
        end = min(begin + chunks * CHUNK, row.end);
        tiles = (slice_chunks + TILE_CHUNKS - 1) / TILE_CHUNKS;        // (also those that the row does not reach: their barriers complete with the others')
    }
    // One tile's copies, by one thread; they land behind the tile's barrier.
    __device__ __forceinline__ void issue(const StagedRow<T>& row, uint32_t rank, int slice_chunks, bool shifted, int t) const {
        constexpr int CHUNK_GRAINS = CHUNK / StagedRow<T>::GRAIN, TILE = TILE_CHUNKS * CHUNK_GRAINS;
        const int first = t * TILE, behind = shifted && row.mis ? 1 : 0;
        const int count = t + 1 < tiles ? TILE : slice_chunks * CHUNK_GRAINS - first + behind;
        stage_tile<T>(const_cast<unsigned char*>(data) + (size_t)first * 16, row, (int)rank * slice_chunks * CHUNK_GRAINS + first, count, &bars[t],
                      l2_evict_first_policy());
        mbar_arrive(&bars[t]);
    }
    // All of them, by the first threads.
    __device__ __forceinline__ void stage(const StagedRow<T>& row, uint32_t rank, int slice_chunks, bool shifted) {
        locate(row, rank, slice_chunks, shifted);
        if ((int)threadIdx.x < tiles) issue(row, rank, slice_chunks, shifted, (int)threadIdx.x);
    }
    // Wait until chunk c has landed (and, `shifted`, the granule behind it): a WAIT_* outcome.
    __device__ __forceinline__ int wait(int c, bool shifted, unsigned long long limit, uint32_t parity = 0u) const {
        const int t = c / TILE_CHUNKS;
        int outcome = mbar_wait_twice(&bars[t], parity, limit);
        if (shifted && (c + 1) % TILE_CHUNKS == 0 && t + 1 < tiles) outcome = max(outcome, mbar_wait_twice(&bars[t + 1], parity, limit));
        return outcome;
    }
    __device__ __forceinline__ const unsigned char* chunk(int c) const { return data + (size_t)c * CHUNK * sizeof(T); }
};

__device__ __forceinline__ float entry_value(const unsigned char* data, int i, const __nv_bfloat16*) {
    return __uint_as_float((uint32_t)reinterpret_cast<const unsigned short*>(data)[i] << 16);
}
__device__ __forceinline__ float entry_value(const unsigned char* data, int i, const float*) {
    return reinterpret_cast<const float*>(data)[i];
}

// the entries of one granule
__device__ __forceinline__ void unpack_granule(uint4 q, float* l, const __nv_bfloat16*) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        l[2 * i] = __uint_as_float(w[i] << 16);
        l[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack_granule(uint4 q, float* l, const float*) {
    l[0] = __uint_as_float(q.x); l[1] = __uint_as_float(q.y); l[2] = __uint_as_float(q.z); l[3] = __uint_as_float(q.w);
}

// off = fp32(ref * c32) may miss ref * c32 by 2^-25 of itself, which the streaming terms carry as a factor until
// stream_scale() takes it back: up to 2^30 that is a factor of 2^32, which fp32 holds.  Beyond (a chunk masked with
// the type's lowest value, say) neighbouring fp32 values are 64 and more powers of two apart in weight: an entry counts 1 at
// the reference and 0 anywhere else.
__device__ __forceinline__ bool offset_ok(float off) { return fabsf(off) < 1073741824.0f; }
// sum over the lane's 32 entries of exp((l - ref) / T), up to the factor that stream_scale() gives; off = ref * c32 rounded
template <typename T> __device__ __forceinline__ float lane_weight_sum(const ChunkRegs<T>& r, float ref, float c32, float off) {
    if (offset_ok(off)) return lane_exp_sum2(r, c32, off);
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += r.value(k) != r.value(k) ? r.value(k) : r.value(k) == ref ? 1.0f : 0.0f;
    return s;
}
__device__ __forceinline__ f32x2 fmul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ double stream_scale(float ref, float c32) {
    return offset_ok(__fmul_rn(ref, c32)) ? stream_sum_scale(ref, c32) : 1.0;
}

// loads that stay where they are written
__device__ __forceinline__ int load_now(const int* p) {
    int v;
    asm volatile("ld.global.nc.s32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float load_now(const float* p) {
    float v;
    asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
// sums over a warp, side by side
__device__ __forceinline__ void warp_sums(double& a, double& b, double& c, double& d) {
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) {
        const double x = __shfl_xor_sync(0xffffffffu, a, i), y = __shfl_xor_sync(0xffffffffu, b, i);
        const double z = __shfl_xor_sync(0xffffffffu, c, i), w = __shfl_xor_sync(0xffffffffu, d, i);
        a += x; b += y; c += z; d += w;
    }
}
// exp(x) and stream_scale() to 2^-22 and 2^-24 of the exponent, for what fp32 sums are multiplied by
__device__ __forceinline__ float exp_near(double x) { return ex2_approx((float)(x * 1.4426950408889634074)); }
__device__ __forceinline__ float stream_scale_near(float ref, float c32) {
    const float off = __fmul_rn(ref, c32);
    return offset_ok(off) ? ex2_approx((float)((double)off - (double)ref * (double)c32)) : 1.0f;
}
// What brings a streaming sum relative to `ref` onto the scale of exp((l - top) / T): stream_scale(), and ref against top; to 2^-22.
__device__ __forceinline__ double reference_factor(float ref, float top, float c32, double rT) {
    if (!(ref > -CUDART_INF_F)) return 0.0;
    const float off = __fmul_rn(ref, c32);
    const double x = ((double)ref - (double)top) * rT;
    return (double)exp_near(offset_ok(off) ? fma((double)off - (double)ref * (double)c32, 0.69314718055994530942, x) : x);
}

// How a launch deals rows to clusters: CTAs per row and chunks per CTA.
struct RowDeal {
    int cluster, slice_chunks;      // cluster 0: the row does not fit
};
constexpr long long ROW_MAX_BYTES = 1376256;    // mirrors picospec.h
// Few rows are bound by latency: a row is spread over as many CTAs as leave each warp a chunk.  Many rows are bound by
// HBM: `resident` bytes of slice per CTA let several CTAs of an SM load and compute in turn.  Rows of more than 8 such slices
// take `large` bytes of slice, with up to `most` CTAs.
// `shifted` slices are of whole vocabulary chunks; others take in what lies before the row in its first granule, 7 entries at most.
inline RowDeal deal_rows(long long rows, int V, int elem, int num_sms, int resident, int large, int most, bool shifted) {
    const int nch = (int)(((long long)V + (shifted ? 0 : 8) + CHUNK - 1) / CHUNK);
    const long long bytes = (long long)nch * CHUNK * elem;
    RowDeal d{0, 0};
    if (bytes > ROW_MAX_BYTES) return d;
    d.cluster = (int)((bytes + resident - 1) / resident);
    if (d.cluster > 8) d.cluster = (int)((bytes + large - 1) / large);
    if (d.cluster > most) d.cluster = most;
    while (d.cluster < 8 && rows * (d.cluster + 1) <= num_sms && nch > d.cluster * TILE_CHUNKS) ++d.cluster;
    d.slice_chunks = (nch + d.cluster - 1) / d.cluster;
    return d;
}

}  // namespace picospec
