// The blocks of keys that each block of queries is to see: the `top` with the largest score
//   score(r, s) = sum_d (sum of q over block r)_d (mean of k over block s)_d
// head by head, the largest first, equal scores in the order of their indexes, a NaN counted as -inf.
//
// Sums, products and comparisons are fp64, so that rounding does not decide which of two neighbours in rank comes first.
// Two launches: the blocks' sums and means (bound by reading q and k once), then scores and ranks from those, which stay in L2.
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

// A CTA pools one block of q (blockIdx.y = 0) or k: a thread keeps to a 16-byte column of the pixels and takes every so many of them.
// pooled: [q or k][B][heads][blocks][d]
template <typename T>
__global__ void __launch_bounds__(kPoolThreads) pool_kernel(const Geometry g, int d, long long images, const T* q, const T* k, double* pooled)
{
    constexpr int V = 16 / sizeof(T);
    __shared__ double part[kPoolThreads][V];
    grid_dependency_wait();
    const int C = g.heads * d, columns = C / V;
    const int r = blockIdx.x % g.blocks;
    const size_t b = blockIdx.x / g.blocks;
    const Block own = block_of(g, r);
    const int size = own.size();
    const unsigned char* src = reinterpret_cast<const unsigned char*>((blockIdx.y ? k : q) + b * g.H * g.W * C);
    for (int first = 0; first < columns; first += kPoolThreads) {
        const int here = min(columns - first, kPoolThreads), rows = kPoolThreads / here;
        const int column = threadIdx.x % here, row = threadIdx.x / here;
        double sum[V] = {};
        if (row < rows) {
#pragma unroll 4
            for (int i = row; i < size; i += rows) {
                double v[V];
                widen<T>(*reinterpret_cast<const uint4*>(src + ((size_t)pixel_of(g, own, i) * columns + first + column) * 16), v);
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += v[e];
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) part[threadIdx.x][e] = sum[e];
        __syncthreads();
        for (int c = threadIdx.x; c < here * V; c += kPoolThreads) {
            double s = 0.0;
            for (int i = 0; i < rows; ++i) s += part[i * here + c / V][c % V];
            const int channel = first * V + c, h = channel / d;
            pooled[((((size_t)blockIdx.y * images + b) * g.heads + h) * g.blocks + r) * d + channel - h * d] = blockIdx.y ? s / (double)size : s;
        }
        __syncthreads();
    }
}

constexpr int kRankRows = 8;              // rows of scores of a CTA, one to a warp when they are ranked
constexpr int kRankThreads = 32 * kRankRows;

// The order of doubles as that of unsigned integers.  0 is below every score.
__device__ __forceinline__ unsigned long long order_of(double x) {
    if (x != x) x = -INFINITY;
    const long long bits = __double_as_longlong(x + 0.0);          // -0 as +0
    return bits < 0 ? ~(unsigned long long)bits : (unsigned long long)bits | 0x8000000000000000ull;
}

template <int D>
__global__ void __launch_bounds__(kRankThreads) rank_kernel(const Geometry g, long long images, const double* pooled, int* idx)
{
    extern __shared__ __align__(16) unsigned char smem[];
    double* rows = reinterpret_cast<double*>(smem);                                       // [kRankRows][D]
    unsigned long long* order = reinterpret_cast<unsigned long long*>(rows + kRankRows * D);      // [kRankRows][blocks]
    grid_dependency_wait();
    const int groups = (g.blocks + kRankRows - 1) / kRankRows;
    const size_t plane = blockIdx.x / groups;                       // image and head
    const int r0 = (int)(blockIdx.x % groups) * kRankRows, n = min(kRankRows, g.blocks - r0);
    const double* qs = pooled + (plane * g.blocks + r0) * D;
    const double* ks = pooled + ((size_t)images * g.heads + plane) * g.blocks * D;
    for (int i = threadIdx.x; i < n * D; i += kRankThreads) rows[i] = qs[i];
    __syncthreads();
    for (int s = threadIdx.x; s < g.blocks; s += kRankThreads) {
        double sum[kRankRows] = {};
#pragma unroll 4
        for (int c = 0; c < D; ++c) {
            const double kc = ks[(size_t)s * D + c];
#pragma unroll
            for (int i = 0; i < kRankRows; ++i) sum[i] = fma(rows[i * D + c], kc, sum[i]);
        }
        for (int i = 0; i < n; ++i) order[i * g.blocks + s] = order_of(sum[i]);
    }
    __syncthreads();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
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
    constexpr int kMost = kRankRows * (kMaxBlocks + D) * 8;
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(rank_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    const long long groups = (g.blocks + kRankRows - 1) / kRankRows;
    return launch_chained(rank_kernel<D>, dim3((unsigned)(B * g.heads * groups)), kRankThreads, (size_t)kRankRows * (g.blocks + D) * 8, stream, g, B,
                          pooled, idx);
}

}  // namespace sparse

cudaError_t launch_select(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const void* q, const void* k, double* pooled,
                          int* idx, cudaStream_t stream) {
    using namespace sparse;
    g.complete();
    const dim3 grid((unsigned)(B * g.blocks), 2);
    cudaError_t e = dtype == SLIDE_ATTN_BF16
                        ? launch_chained(pool_kernel<__nv_bfloat16>, grid, kPoolThreads, 0, stream, g, head_dim, B, static_cast<const __nv_bfloat16*>(q),
                                         static_cast<const __nv_bfloat16*>(k), pooled)
                        : launch_chained(pool_kernel<float>, grid, kPoolThreads, 0, stream, g, head_dim, B, static_cast<const float*>(q),
                                         static_cast<const float*>(k), pooled);
    if (e != cudaSuccess) return e;
    if (head_dim == 16) return launch_rank<16>(g, B, pooled, idx, stream);
    if (head_dim == 32) return launch_rank<32>(g, B, pooled, idx, stream);
    return launch_rank<64>(g, B, pooled, idx, stream);
}

}  // namespace slide_attn
