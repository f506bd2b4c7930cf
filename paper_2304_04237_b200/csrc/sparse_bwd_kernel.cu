// Block-sparse attention, backward.  With P the softmax weights (computed again from the stored logarithms of the sums) and
// delta = sum_d dout out of each query:
//
//   dS = P (dout v^T - delta),   dq = dS k / sqrt(d),   dk = dS^T q / sqrt(d),   dv = P^T dout
//
// Two launches: queries (dq, over the blocks of their list; also writes delta) and keys (dk and dv, over the blocks of queries whose
// lists name the key's block, found by going through the image's lists in their order).  Neither adds to memory that another CTA
// writes, so results do not depend on which CTA runs first.
#include "operators.cuh"

namespace slide_attn {

namespace sparse {

template <typename T, int D> constexpr int kBackwardTile = D == 64 ? 32 : 64;       // rows of a tile
constexpr int kListed = 1024;                                                       // entries that the keys' kernel lists at a time
constexpr int kScan = 4 * kThreads;                                                 // entries of the image's lists that it looks at in one go

// exp2 of a score less the logarithm of its row's sum.  A row that has none (no keys, or none but -inf) has no weights.
__device__ __forceinline__ float log2_of_sum(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

template <typename T> __device__ __forceinline__ float dot_piece(const T* a, const T* b);
template <> __device__ __forceinline__ float dot_piece<float>(const float* a, const float* b) {
    const float4 x = *reinterpret_cast<const float4*>(a), y = *reinterpret_cast<const float4*>(b);
    return fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, x.w * y.w)));
}
template <> __device__ __forceinline__ float dot_piece<__nv_bfloat16>(const __nv_bfloat16* a, const __nv_bfloat16* b) {
    const uint4 x = *reinterpret_cast<const uint4*>(a), y = *reinterpret_cast<const uint4*>(b);
    const uint32_t p[4] = {x.x, x.y, x.z, x.w}, q[4] = {y.x, y.y, y.z, y.w};
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(bf16_lo(p[i]), bf16_lo(q[i]), fmaf(bf16_hi(p[i]), bf16_hi(q[i]), s));
    return s;
}

template <typename T, int D> constexpr size_t queries_smem() {
    return (size_t)Tile<T, D>::kRowBytes * (2 * kRows + 4 * kBackwardTile<T, D>) + kMaxTop * sizeof(Entry) + kRows * sizeof(float);
}
template <typename T, int D> constexpr size_t keys_smem() {
    return (size_t)Tile<T, D>::kRowBytes * (2 * kRows + 4 * kBackwardTile<T, D>) + kListed * sizeof(Entry) + 4 * kBackwardTile<T, D> * sizeof(float);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
sparse_queries_kernel(const Geometry g, const T* q, const T* k, const T* v, const int* idx, const T* out, const float* lse, const T* dout, T* dq,
                      float* delta)
{
    using L = Tile<T, D>;
    constexpr int N = kBackwardTile<T, D>, NT = N / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int listed;
    const uint32_t tile_q = smem_u32(smem), tile_g = tile_q + kRows * L::kRowBytes, tiles = tile_g + kRows * L::kRowBytes;
    constexpr uint32_t kStage = 2 * N * L::kRowBytes;
    Entry* list = reinterpret_cast<Entry*>(smem + (size_t)(2 * kRows + 4 * N) * L::kRowBytes);
    float* own_delta = reinterpret_cast<float*>(list + kMaxTop);

    unsigned u = blockIdx.x;
    const int h = u % g.heads; u /= g.heads;
    const int part = u % g.tiles; u /= g.tiles;
    const int r = u % g.blocks;
    const size_t b = u / g.blocks;
    const Block own = block_of(g, r);
    const int rows = own.size() - part * kRows;
    const size_t stride = (size_t)g.heads * D;
    const size_t plane = b * g.H * g.W * stride + (size_t)h * D;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    grid_dependency_wait();
    if (rows <= 0) return;
    copy_rows<T, D, kRows>(tile_q, tile_g, q + plane, dout + plane, stride, rows,
                           [&](int row) { return pixel_of(g, own, part * kRows + row); });
    copies_commit();
    {
        // delta: two threads a row
        const int row = threadIdx.x / 2;
        float s = 0.0f;
        size_t pixel = 0;
        if (row < rows) {
            pixel = pixel_of(g, own, part * kRows + row);
            const size_t at = plane + pixel * stride;
            constexpr int kPiece = 16 / sizeof(T);
#pragma unroll
            for (int i = 0; i < L::kPieces / 2; ++i) {
                const int e = (i * 2 + (threadIdx.x & 1)) * kPiece;
                s += dot_piece<T>(dout + at + e, out + at + e);
            }
        }
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        if (!(threadIdx.x & 1)) {
            own_delta[row] = s;
            if (row < rows) delta[(b * g.H * g.W + pixel) * g.heads + h] = s;
        }
    }
    if (warp == 0) {
        const int total = read_list(g, idx + ((b * g.heads + h) * g.blocks + r) * g.top, list, lane);
        if (lane == 0) listed = total;
    }
    __syncthreads();
    const int keys = listed, steps = (keys + N - 1) / N;
    Cursor cursor;
    auto fetch = [&](int step) {
        const uint32_t at = tiles + (step & 1) * kStage;
        copy_rows<T, D, N>(at, at + N * L::kRowBytes, k + plane, v + plane, stride, keys - step * N,
                           [&](int row) { return cursor.pixel(g, list, step * N + row); });
        copies_commit();
    };
    if (steps > 0) fetch(0);

    const bool busy = warp * 16 < rows;
    constexpr float scale = root<D>();
    typename L::Rows rows_q, rows_g;
    float dqs[D / 8][4] = {};
    float sum[2], del[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int row = warp * 16 + half * 8 + (lane >> 2);
        sum[half] = INFINITY;
        if (row < rows) sum[half] = log2_of_sum(lse[(b * g.H * g.W + pixel_of(g, own, part * kRows + row)) * g.heads + h]);
        del[half] = own_delta[row];
    }
    for (int step = 0; step < steps; ++step) {
        copies_wait_all();
        __syncthreads();
        if (step + 1 < steps) fetch(step + 1);
        if (!busy) continue;
        if (step == 0) { rows_q.load(tile_q, warp * 16, lane); rows_g.load(tile_g, warp * 16, lane); }
        const uint32_t at = tiles + (step & 1) * kStage;
        const int used = min(N, keys - step * N);
        float s[NT][4], dp[NT][4];
        L::template scores<NT>(rows_q, at, lane, used, s);
        L::template scores<NT>(rows_g, at + N * L::kRowBytes, lane, used, dp);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = n * 8 + 2 * (lane & 3) + (e & 1) < used ? fast_exp2(fmaf(s[n][e], scale * kLog2e, -sum[e >> 1])) : 0.0f;
                s[n][e] = p * (dp[n][e] - del[e >> 1]);
            }
        L::template gather<NT>(s, at, lane, used, dqs);
    }
    if (!busy) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int row = warp * 16 + half * 8 + (lane >> 2);
        if (row >= rows) continue;
        T* dst = dq + plane + (size_t)pixel_of(g, own, part * kRows + row) * stride + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < D / 8; ++n) store2(dst + n * 8, dqs[n][2 * half] * scale, dqs[n][2 * half + 1] * scale);
    }
}

__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
sparse_keys_kernel(const Geometry g, const T* q, const T* k, const T* v, const int* idx, const float* lse, const float* delta, const T* dout, T* dk, T* dv)
{
    using L = Tile<T, D>;
    constexpr int N = kBackwardTile<T, D>, NT = N / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int warp_sums[kThreads / 32];
    const uint32_t tile_k = smem_u32(smem), tile_v = tile_k + kRows * L::kRowBytes, tiles = tile_v + kRows * L::kRowBytes;
    constexpr uint32_t kStage = 2 * N * L::kRowBytes;     // queries, then gradients of the output
    Entry* list = reinterpret_cast<Entry*>(smem + (size_t)(2 * kRows + 4 * N) * L::kRowBytes);
    const float* columns = reinterpret_cast<const float*>(list + kListed);      // of each stage: logarithms of the sums, then delta
    const uint32_t columns_at = smem_u32(columns);

    unsigned u = blockIdx.x;
    const int h = u % g.heads; u /= g.heads;
    const int part = u % g.tiles; u /= g.tiles;
    const int r = u % g.blocks;
    const size_t b = u / g.blocks;
    const Block own = block_of(g, r);
    const int rows = own.size() - part * kRows;
    const size_t stride = (size_t)g.heads * D;
    const size_t plane = b * g.H * g.W * stride + (size_t)h * D;
    const size_t row_plane = b * g.H * g.W * g.heads + h;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    grid_dependency_wait();
    if (rows <= 0) return;
    copy_rows<T, D, kRows>(tile_k, tile_v, k + plane, v + plane, stride, rows,
                           [&](int row) { return pixel_of(g, own, part * kRows + row); });
    copies_commit();

    const bool busy = warp * 16 < rows;
    constexpr float scale = root<D>();
    typename L::Rows rows_k, rows_v;
    bool loaded = false;
    float dks[D / 8][4] = {}, dvs[D / 8][4] = {};
    const int* lists = idx + (b * g.heads + h) * (size_t)g.blocks * g.top;
    const int entries = g.blocks * g.top;
    int seen = 0;
    while (seen < entries) {
        // the next blocks of queries that see this block, in an order that the lists alone decide
        int n = 0, total = 0;
        while (seen < entries && n + kScan <= kListed) {
            int mine[4], own_rows = 0, own_count = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = seen + e * kThreads + (int)threadIdx.x;
                mine[e] = i < entries && lists[i] == r ? i / g.top : -1;
                if (mine[e] >= 0) { own_rows += block_of(g, mine[e]).size(); ++own_count; }
            }
            int sum = own_count << 20 | own_rows;            // at most 512 blocks of 1024 rows
            const int own_sum = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int x = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += x;
            }
            if (lane == 31) warp_sums[warp] = sum;
            __syncthreads();
            int before = sum - own_sum, all = 0;
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) {
                if (w < warp) before += warp_sums[w];
                all += warp_sums[w];
            }
            int slot = n + (before >> 20), start = total + (before & 0xFFFFF);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (mine[e] >= 0) {
                    list[slot++] = {mine[e], start};
                    start += block_of(g, mine[e]).size();
                }
            n += all >> 20;
            total += all & 0xFFFFF;
            seen += kScan;
            __syncthreads();
        }
        const int steps = (total + N - 1) / N;
        Cursor cursor;
        auto fetch = [&](int step) {
            const uint32_t at = tiles + (step & 1) * kStage;
            constexpr int kPer = kThreads / N;
            copy_rows<T, D, N>(at, at + N * L::kRowBytes, q + plane, dout + plane, stride, total - step * N, [&](int row) {
                const int pixel = cursor.pixel(g, list, step * N + row);
                const uint32_t c = columns_at + (uint32_t)(((step & 1) * 2 * N + row) * 4);
                if (threadIdx.x % kPer == 0) copy4(c, lse + row_plane + (size_t)pixel * g.heads, true);
                else if (threadIdx.x % kPer == 1) copy4(c + N * 4, delta + row_plane + (size_t)pixel * g.heads, true);
                return pixel;
            });
            copies_commit();
        };
        if (steps > 0) fetch(0);
        for (int step = 0; step < steps; ++step) {
            copies_wait_all();
            __syncthreads();
            if (step + 1 < steps) fetch(step + 1);
            if (!busy) continue;
            if (!loaded) { rows_k.load(tile_k, warp * 16, lane); rows_v.load(tile_v, warp * 16, lane); loaded = true; }
            const uint32_t at = tiles + (step & 1) * kStage;
            const float* col = columns + (step & 1) * 2 * N;
            const int used = min(N, total - step * N);
            float s[NT][4], dp[NT][4];
            L::template scores<NT>(rows_k, at, lane, used, s);
#pragma unroll
            for (int n8 = 0; n8 < NT; ++n8)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = n8 * 8 + 2 * (lane & 3) + (e & 1);
                    s[n8][e] = c < used ? fast_exp2(fmaf(s[n8][e], scale * kLog2e, -log2_of_sum(col[c]))) : 0.0f;
                }
            L::template gather<NT>(s, at + N * L::kRowBytes, lane, used, dvs);
            L::template scores<NT>(rows_v, at + N * L::kRowBytes, lane, used, dp);
#pragma unroll
            for (int n8 = 0; n8 < NT; ++n8)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = n8 * 8 + 2 * (lane & 3) + (e & 1);
                    s[n8][e] = c < used ? s[n8][e] * (dp[n8][e] - col[N + c]) : 0.0f;
                }
            L::template gather<NT>(s, at, lane, used, dks);
        }
        __syncthreads();                                     // the list and the tiles are free again
    }
    copies_wait_all();                                       // a block that nobody sees never waited for its own rows
    if (!busy) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int row = warp * 16 + half * 8 + (lane >> 2);
        if (row >= rows) continue;
        const size_t at = plane + (size_t)pixel_of(g, own, part * kRows + row) * stride + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
            store2(dk + at + n * 8, dks[n][2 * half] * scale, dks[n][2 * half + 1] * scale);
            store2(dv + at + n * 8, dvs[n][2 * half], dvs[n][2 * half + 1]);
        }
    }
}

template <typename T, int D>
cudaError_t launch_backward(const Geometry& g, long long B, const BackwardMaps& m, float* delta, cudaStream_t stream) {
    constexpr size_t smem_q = queries_smem<T, D>(), smem_k = keys_smem<T, D>();
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(sparse_queries_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_q);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(sparse_keys_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_k);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    const dim3 grid((unsigned)(B * g.blocks * g.tiles * g.heads));
    auto in = [](const void* p) { return static_cast<const T*>(p); };
    auto to = [](void* p) { return static_cast<T*>(p); };
    e = launch_chained(sparse_queries_kernel<T, D>, grid, kThreads, smem_q, stream, g, in(m.q), in(m.k), in(m.v), m.idx, in(m.out), m.lse, in(m.dout),
                       to(m.dq), delta);
    if (e != cudaSuccess) return e;
    return launch_chained(sparse_keys_kernel<T, D>, grid, kThreads, smem_k, stream, g, in(m.q), in(m.k), in(m.v), m.idx, m.lse,
                          static_cast<const float*>(delta), in(m.dout), to(m.dk), to(m.dv));
}

}  // namespace sparse

cudaError_t launch_sparse_backward(const sparse::Geometry& g, long long B, int head_dim, slide_attn_dtype dtype, const sparse::BackwardMaps& m,
                                   float* delta, cudaStream_t stream) {
    using namespace sparse;
    if (dtype == SLIDE_ATTN_BF16) {
        if (head_dim == 16) return launch_backward<__nv_bfloat16, 16>(g, B, m, delta, stream);
        if (head_dim == 32) return launch_backward<__nv_bfloat16, 32>(g, B, m, delta, stream);
        return launch_backward<__nv_bfloat16, 64>(g, B, m, delta, stream);
    }
    if (head_dim == 16) return launch_backward<float, 16>(g, B, m, delta, stream);
    if (head_dim == 32) return launch_backward<float, 32>(g, B, m, delta, stream);
    return launch_backward<float, 64>(g, B, m, delta, stream);
}

}  // namespace slide_attn
