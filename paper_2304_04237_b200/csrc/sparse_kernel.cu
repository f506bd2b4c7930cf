// Block-sparse attention, forward: out = softmax(q k^T / sqrt(d)) v over the pixels of the blocks listed for the query's block, and the
// logarithm of each softmax's sum.
//
// A CTA takes 64 queries of one block and head, four warps of 16 rows; keys and values come in tiles of the list, two in flight.
// Scores, weights and sums stay in registers; the maximum and the sum of a row run along (32 bits; bf16 weights are rounded where they
// become an operand of the second product).
#include "operators.cuh"

namespace slide_attn {

namespace sparse {

template <typename T, int D> constexpr int kForwardKeys = sizeof(T) == 4 && D == 64 ? 32 : 64;      // keys of a tile

template <typename T, int D> constexpr size_t forward_smem() {
    return (size_t)Tile<T, D>::kRowBytes * (kRows + 4 * kForwardKeys<T, D>) + kMaxTop * sizeof(Entry);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) sparse_forward_kernel(const Geometry g, const T* q, const T* k, const T* v, const int* idx, T* out, float* lse)
{
    using L = Tile<T, D>;
    constexpr int N = kForwardKeys<T, D>, NT = N / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int listed;                                // rows of the list
    const uint32_t tile_q = smem_u32(smem), tiles = tile_q + kRows * L::kRowBytes;
    constexpr uint32_t kStage = 2 * N * L::kRowBytes;     // keys, then values
    Entry* list = reinterpret_cast<Entry*>(smem + (size_t)(kRows + 4 * N) * L::kRowBytes);

    unsigned u = blockIdx.x;
    const int h = u % g.heads; u /= g.heads;
    const int part = u % g.tiles; u /= g.tiles;
    const int r = u % g.blocks;
    const size_t b = u / g.blocks;
    const Block own = block_of(g, r);
    const int rows = own.size() - part * kRows;           // of this tile
    const size_t stride = (size_t)g.heads * D;
    const size_t plane = b * g.H * g.W * stride + (size_t)h * D;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    grid_dependency_wait();
    if (rows <= 0) return;
    copy_rows<T, D, kRows>(tile_q, 0, q + plane, static_cast<const T*>(nullptr), stride, rows,
                           [&](int row) { return pixel_of(g, own, part * kRows + row); });
    copies_commit();
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

    typename L::Rows rows_q;
    const bool busy = warp * 16 < rows;
    constexpr float scale = root<D>() * kLog2e;
    float o[D / 8][4] = {};
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {};
    for (int step = 0; step < steps; ++step) {
        copies_wait_all();
        __syncthreads();                                  // everyone's copies have landed, and everyone is done with the tile before
        if (step + 1 < steps) fetch(step + 1);
        if (!busy) continue;
        if (step == 0) rows_q.load(tile_q, warp * 16, lane);
        const uint32_t at = tiles + (step & 1) * kStage;
        const int used = min(N, keys - step * N);
        float s[NT][4];
        L::template scores<NT>(rows_q, at, lane, used, s);
        if (used < N) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n * 8 + 2 * (lane & 3) + (e & 1) >= used) s[n][e] = -INFINITY;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float m = top[half];
#pragma unroll
            for (int n = 0; n < NT; ++n) m = fmaxf(m, fmaxf(s[n][2 * half], s[n][2 * half + 1]));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const float base = m == -INFINITY ? 0.0f : m * scale;       // while all scores are -inf, so are all exponents
            const float fade = fast_exp2(top[half] * scale - base);
            top[half] = m;
            float l = 0.0f;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float w = fast_exp2(fmaf(s[n][2 * half + e], scale, -base));
                    s[n][2 * half + e] = w;
                    l += w;
                }
            sum[half] = sum[half] * fade + l;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) { o[n][2 * half] *= fade; o[n][2 * half + 1] *= fade; }
        }
        L::template gather<NT>(s, at + N * L::kRowBytes, lane, used, o);
    }
    if (!busy) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float l = sum[half];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        const int row = warp * 16 + half * 8 + (lane >> 2);
        if (row >= rows) continue;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;                  // no keys, or none that is not -inf: zeros
        const int pixel = pixel_of(g, own, part * kRows + row);
        T* dst = out + plane + (size_t)pixel * stride + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < D / 8; ++n) store2(dst + n * 8, o[n][2 * half] * inv, o[n][2 * half + 1] * inv);
        if ((lane & 3) == 0)
            lse[(b * g.H * g.W + pixel) * g.heads + h] = l == 0.0f ? -INFINITY : top[half] * (scale * kLn2) + logf(l);
    }
}

template <typename T, int D>
cudaError_t launch_forward(const Geometry& g, long long B, const void* q, const void* k, const void* v, const int* idx, void* out, float* lse,
                           cudaStream_t stream) {
    constexpr size_t smem = forward_smem<T, D>();
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(sparse_forward_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    return launch_chained(sparse_forward_kernel<T, D>, dim3((unsigned)(B * g.blocks * g.tiles * g.heads)), kThreads, smem, stream, g,
                          static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v), idx, static_cast<T*>(out), lse);
}

}  // namespace sparse

cudaError_t launch_sparse_forward(const sparse::Geometry& g, long long B, int head_dim, slide_attn_dtype dtype, const void* q, const void* k,
                                  const void* v, const int* idx, void* out, float* lse, cudaStream_t stream) {
    using namespace sparse;
    if (dtype == SLIDE_ATTN_BF16) {
        if (head_dim == 16) return launch_forward<__nv_bfloat16, 16>(g, B, q, k, v, idx, out, lse, stream);
        if (head_dim == 32) return launch_forward<__nv_bfloat16, 32>(g, B, q, k, v, idx, out, lse, stream);
        return launch_forward<__nv_bfloat16, 64>(g, B, q, k, v, idx, out, lse, stream);
    }
    if (head_dim == 16) return launch_forward<float, 16>(g, B, q, k, v, idx, out, lse, stream);
    if (head_dim == 32) return launch_forward<float, 32>(g, B, q, k, v, idx, out, lse, stream);
    return launch_forward<float, 64>(g, B, q, k, v, idx, out, lse, stream);
}

}  // namespace slide_attn
