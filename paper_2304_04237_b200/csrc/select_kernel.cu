// The blocks of keys that each block of queries is to see: the `top` with the largest score
//   score(r, s) = sum_d (sum of q over block r)_d (mean of k over block s)_d
// head by head, the largest first, equal scores in the order of their indexes, a NaN counted as -inf.
//
// Sums, products and comparisons are fp64, so that rounding does not decide which of two neighbours in rank comes first.
// Two launches: the blocks' sums and means (bound by reading q and k once), then scores and ranks from those, which stay in L2.
// 64 x 56 x 56, 2 heads, bf16, 4 of 64 blocks of 7 x 7: 23.7 us, of 7.9 for reading q and k.  Pooling (16 us by itself, L2 cold) is bound by the conversions to
// fp64 (59 % of the pipe that makes them), ranking (14) by the latency of one maximum after the other.
#include "operators.cuh"

namespace slide_attn {

namespace sparse {

constexpr int kPoolThreads = 256;

template <typename T> __device__ __forceinline__ void widen(const uint4& r, double (&v)[16 / sizeof(T)]);
template <> __device__ __forceinline__ void widen<float>(const uint4& r, double (&v)[4]) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
}
template <> __device__ __forceinline__ void widen<__nv_bfloat16>(const uint4& r, double (&v)[8]) {
    v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y);
    v[4] = bf16_lo(r.z); v[5] = bf16_hi(r.z); v[6] = bf16_lo(r.w); v[7] = bf16_hi(r.w);
}

// A thread keeps to a 16-byte column of one block and takes every `parts`-th of its pixels; neighbouring threads have neighbouring columns, then
// neighbouring blocks, so that a warp reads whole lines.  Parts are joined through shared memory, in their order.  blockIdx.y: q or k.
// pooled: [q or k][B][heads][blocks][d]
template <typename T>
__global__ void __launch_bounds__(kPoolThreads) pool_kernel(const Geometry g, Divisor by_columns, int d, long long images, int parts, const T* q, const T* k,
                                                            double* pooled)
{
    constexpr int V = 16 / sizeof(T);
    __shared__ double part_sums[kPoolThreads][V + 1];
    grid_dependency_wait();
    const int C = g.heads * d, columns = C / V, units = kPoolThreads / parts;
    const int part = (int)threadIdx.x / units, own = (int)threadIdx.x - part * units;
    const long long at = (long long)blockIdx.x * units + own;          // (image, block, column)
    const bool there = at < images * g.blocks * columns;
    unsigned column = there ? (unsigned)at : 0u;
    unsigned r = by_columns.divide(column);
    const unsigned b = g.by_blocks.divide(r);
    const Block block = block_of(g, (int)r);
    const int size = block.size();
    double sum[V] = {};
    if (there) {
        const unsigned char* src = reinterpret_cast<const unsigned char*>((blockIdx.y ? k : q) + (size_t)b * (unsigned)(g.H * g.W) * (unsigned)C) + column * 16;
#pragma unroll 8
        for (int i = part; i < size; i += parts) {
            double v[V];
            widen<T>(*reinterpret_cast<const uint4*>(src + (size_t)(unsigned)pixel_of(g, block, i) * (unsigned)(C * (int)sizeof(T))), v);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += v[e];
        }
    }
    if (parts > 1) {
#pragma unroll
        for (int e = 0; e < V; ++e) part_sums[threadIdx.x][e] = sum[e];
        __syncthreads();
        for (int p = 1; p < parts; ++p)
            if (part == 0)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += part_sums[p * units + own][e];
    }
    if (part || !there) return;
    const unsigned channel = column * V, h = channel / (unsigned)d;
    double* out = pooled + ((((size_t)blockIdx.y * images + b) * g.heads + h) * g.blocks + r) * d + (channel - h * d);
#pragma unroll
    for (int e = 0; e < V; e += 2) {
        const double2 v = blockIdx.y ? make_double2(sum[e] / (double)size, sum[e + 1] / (double)size) : make_double2(sum[e], sum[e + 1]);
        *reinterpret_cast<double2*>(out + e) = v;
    }
}

constexpr int kRankRows = 8;              // rows of scores of a CTA, one to a warp when they are ranked
constexpr int kRankThreads = 32 * kRankRows, kRankColumns = 64;

// The order of doubles as that of unsigned integers.  0 is below every score.
__device__ __forceinline__ unsigned long long order_of(double x) {
    if (x != x) x = -INFINITY;
    const long long bits = __double_as_longlong(x + 0.0);          // -0 as +0
    return bits < 0 ? ~(unsigned long long)bits : (unsigned long long)bits | 0x8000000000000000ull;
}

// Eight rows of one image's and head's scores, the keys' means in tiles of 64 through shared memory (rows padded against bank conflicts), then
// the largest, again and again.
template <int D>
__global__ void __launch_bounds__(kRankThreads) rank_kernel(const Geometry g, long long images, const double* pooled, int* idx)
{
    extern __shared__ __align__(16) unsigned char smem[];
    double* rows = reinterpret_cast<double*>(smem);                                       // [kRankRows][D]
    double* tile = rows + kRankRows * D;                                                  // [kRankColumns][D + 1]
    unsigned long long* order = reinterpret_cast<unsigned long long*>(tile + kRankColumns * (D + 1));     // [kRankRows][blocks]
    grid_dependency_wait();
    const int groups = (g.blocks + kRankRows - 1) / kRankRows;
    const size_t plane = blockIdx.x / (unsigned)groups;             // image and head
    const int r0 = (int)(blockIdx.x - (unsigned)plane * (unsigned)groups) * kRankRows, n = min(kRankRows, g.blocks - r0);
    const double* qs = pooled + (plane * g.blocks + r0) * D;
    const double* ks = pooled + ((size_t)images * g.heads + plane) * g.blocks * D;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int i = threadIdx.x; i < n * D; i += kRankThreads) rows[i] = qs[i];
    for (int s0 = 0; s0 < g.blocks; s0 += kRankColumns) {
        const int count = min(kRankColumns, g.blocks - s0);
#pragma unroll
        for (int i = threadIdx.x; i < kRankColumns * D; i += kRankThreads)
            if (i < count * D) tile[i / D * (D + 1) + i % D] = ks[(size_t)s0 * D + i];
        __syncthreads();
        double x = 0.0, y = 0.0;                                    // columns lane and lane + 32 of the warp's row
#pragma unroll 8
        for (int c = 0; c < D; ++c) {
            const double qc = rows[warp * D + c];
            x = fma(qc, tile[lane * (D + 1) + c], x);
            y = fma(qc, tile[(lane + 32) * (D + 1) + c], y);
        }
        if (warp < n) {
            if (lane < count) order[warp * g.blocks + s0 + lane] = order_of(x);
            if (lane + 32 < count) order[warp * g.blocks + s0 + lane + 32] = order_of(y);
        }
        __syncthreads();
    }
    if (warp >= n) return;
    unsigned long long* mine = order + warp * g.blocks;
    int* out = idx + (plane * g.blocks + r0 + warp) * g.top;
    for (int t = 0; t < g.top; ++t) {
        unsigned long long best = 0;
        int at = 0;
        for (int s = lane; s < g.blocks; s += 32)
            if (mine[s] > best) { best = mine[s]; at = s; }
        const unsigned high = __reduce_max_sync(0xffffffffu, (unsigned)(best >> 32));
        const unsigned low = __reduce_max_sync(0xffffffffu, (unsigned)(best >> 32) == high ? (unsigned)best : 0u);
        const bool is = best == ((unsigned long long)high << 32 | low);
        const int chosen = (int)__reduce_min_sync(0xffffffffu, is ? (unsigned)at : 0xffffffffu);
        if (lane == 0) { out[t] = chosen; mine[chosen] = 0; }
        __syncwarp();
    }
}

template <int D>
cudaError_t launch_rank(const Geometry& g, long long B, const double* pooled, int* idx, cudaStream_t stream) {
    constexpr int kFixed = (kRankRows * D + kRankColumns * (D + 1)) * 8, kMost = kFixed + kRankRows * kMaxBlocks * 8;
    static std::atomic<bool> ready[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(rank_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev].store(true, std::memory_order_release);
    }
    const long long groups = (g.blocks + kRankRows - 1) / kRankRows;
    return launch_chained(rank_kernel<D>, dim3((unsigned)(B * g.heads * groups)), kRankThreads, (size_t)(kFixed + kRankRows * g.blocks * 8), stream, g, B,
                          pooled, idx);
}

}  // namespace sparse

cudaError_t launch_select(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const void* q, const void* k, double* pooled,
                          int* idx, int sms, cudaStream_t stream) {
    using namespace sparse;
    g.complete();
    // Columns are shared among up to 16 threads until an SM has 512 threads (q's and k's), as long as each keeps eight pixels.
    const int columns = g.heads * head_dim * (dtype == SLIDE_ATTN_BF16 ? 2 : 4) / 16;
    const long long units = B * g.blocks * columns;
    int parts = 1;
    while (parts < 16 && 2 * units * parts < 512LL * sms && parts * 8 < g.bh * g.bw) parts *= 2;
    const dim3 grid((unsigned)((units * parts + kPoolThreads - 1) / kPoolThreads), 2);
    const Divisor by_columns = Divisor::of(columns);
    cudaError_t e = dtype == SLIDE_ATTN_BF16
                        ? launch_chained(pool_kernel<__nv_bfloat16>, grid, kPoolThreads, 0, stream, g, by_columns, head_dim, B, parts,
                                         static_cast<const __nv_bfloat16*>(q), static_cast<const __nv_bfloat16*>(k), pooled)
                        : launch_chained(pool_kernel<float>, grid, kPoolThreads, 0, stream, g, by_columns, head_dim, B, parts, static_cast<const float*>(q),
                                         static_cast<const float*>(k), pooled);
    if (e != cudaSuccess) return e;
    if (head_dim == 16) return launch_rank<16>(g, B, pooled, idx, stream);
    if (head_dim == 32) return launch_rank<32>(g, B, pooled, idx, stream);
    return launch_rank<64>(g, B, pooled, idx, stream);
}

}  // namespace slide_attn
