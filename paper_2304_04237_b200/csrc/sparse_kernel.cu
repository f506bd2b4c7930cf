// Block-sparse attention, forward: out = softmax(q k^T / sqrt(d)) v over the pixels of the blocks listed for the query's block, and the
// logarithm of each softmax's sum.
//
// A CTA takes 64 queries of one block and head, four warps of 16 rows, then the next (sparse_common.cuh, QueryPipe).  Scores, weights and
// sums stay in registers.  The maximum that a row's exponents are taken from is raised only when a score is more than 2^8 above it, so that
// sums are rescaled in the first tile and hardly ever again.  32 bits throughout; bf16 weights are rounded where they become an operand of
// the second product.
// Products of 16 rows a warp by mma.sync, whose operands and results are in the registers that the softmax works on.  Bound by latency, as a warp's products,
// exponentials and products again wait for one another: 64 x 56 x 56, 2 heads, bf16, 4 blocks of 7 x 7, takes 82.8 us, of 15.7 for its bytes (issue slots
// 45 %, exponentials 36 % of their pipe, tensor pipe 30 %); 2 x 128 x 128, 3 heads, fp32, 8 blocks of 8 x 8, 156.6 us with the choice of the blocks (tensor pipe
// 45 %: six products for one).  (tcgen05 with M = 64, a unit's rows, and accumulators in tensor memory has not been tried.)
//
// Tiles of 32 or 64 keys, us each way (64 x 56 x 56 x 2, 4 blocks of 7 x 7, fp32 8 x 56 x 56 x 3; then 2 x 128 x 128 x 3, 16 blocks of 8 x 8, fp32 8 blocks):
//   bf16, heads of 32: 79.9 / 83.0, then 61.2 / 60.6; heads of 16 (32 x 56 x 56 x 4) 65.6 / 60.2.  64
//   bf16, heads of 64: 125.3 / 143.3, then 101.8 / 100.4; 32 x 28 x 42 x 3, 4 blocks of 8 x 8, 40.0 / 44.2.  32
//   fp32, heads of 32: 61.1 / 73.9, then 134.2 / 151.8; heads of 16 (8 x 56 x 56 x 6) 71.2 / 72.3.  32
// Four stages of copies; three where 64 fp32 values a row leave no room for a fourth beside their planes.  Spills of a few registers: bf16 heads of 32 (20 bytes),
// fp32 heads of 64 (100 bytes); still fewer registers, for one CTA more an SM, were slower.
#include "operators.cuh"

namespace slide_attn {

namespace sparse {

template <typename T, int D> using ForwardPipe = QueryPipe<T, D, sizeof(T) == 4 || D == 64 ? 32 : 64, sizeof(T) == 4 && D == 64 ? 3 : 4, 1>;

template <typename T, int D>
__global__ void __launch_bounds__(kBlock, sizeof(T) == 4 || D == 64 ? 3 : 4)
sparse_forward_kernel(const Geometry g, unsigned units, const T* q, const T* k, const T* v, const int* idx, T* out, float* lse)
{
    using P = ForwardPipe<T, D>;
    using L = Layout<T, D>;
    constexpr int N = P::N, NT = N / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = uniform((int)threadIdx.x / 32), lane = threadIdx.x % 32;
    constexpr float scale = root<D>() * kLog2e;

    grid_dependency_wait();
    P pipe(smem, units);
    if (warp == kThreads / 32) {
        pipe.copy_all(g, q, nullptr, k, v, idx);
        return;
    }

    Unit unit;
    Rows<D, L::kPlanes> rows;
    float o[D / 8][4], sum[2], limit[2];               // limit: the score above which the base is raised
    const pair scales = both(scale);
    pair bases[2];                                     // less the base that exponents are taken from, scaled, twice
    int item = 0, step = 0, keys = 0;
    while (item < pipe.items) {
        const uint32_t at = pipe.next();
        if (step == 0) {
            unit.find(g, pipe.first + item);
            keys = uniform(pipe.rows_of(item));
            pipe.take(at, 0, warp * 16, lane, rows, nullptr);
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i) { sum[i] = 0.0f; limit[i] = -INFINITY; bases[i] = both(0.0f); }
        }
        const bool busy = warp * 16 < unit.rows;
        if (step > 0) {
            const uint32_t tile = pipe.tile(at);
            const int used = min(N, keys - (step - 1) * N);
            if (busy) with_width<NT>(used, [&](auto width, auto partial) {
                constexpr int W = decltype(width)::value;
                float s[W][4];
                scores<D, L::kPlanes, W>(rows, tile, P::kPlane, lane, s);
                if constexpr (decltype(partial)::value) {
#pragma unroll
                    for (int n = W > 2 ? W / 2 : 0; n < W; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (n * 8 + 2 * (lane & 3) + (e & 1) >= used) s[n][e] = -INFINITY;
                }
                float most[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    most[i] = fmaxf(s[0][2 * i], s[0][2 * i + 1]);
#pragma unroll
                    for (int n = 1; n < W; ++n) most[i] = max3(most[i], s[n][2 * i], s[n][2 * i + 1]);
                }
                if (__any_sync(0xffffffffu, most[0] > limit[0] || most[1] > limit[1])) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float m = most[i];
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
                        if (m > limit[i]) {
                            float less, same;
                            split_pair(bases[i], less, same);
                            const float raised = m * scale, fade = limit[i] == -INFINITY ? 0.0f : fast_exp2(-less - raised);
                            bases[i] = both(-raised);
                            limit[i] = m + 8.0f / scale;
                            sum[i] *= fade;
#pragma unroll
                            for (int n = 0; n < D / 8; ++n) { o[n][2 * i] *= fade; o[n][2 * i + 1] *= fade; }
                        }
                    }
                }
                // 16 columns at a time, so that the exponentials of the next go beside the products of these
                pair l[2];
#pragma unroll
                for (int n = 0; n < W; ++n) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float& x = s[n][2 * i];
                        float& y = s[n][2 * i + 1];
                        split_pair(fma2(make_pair(x, y), scales, bases[i]), x, y);
                        x = fast_exp2(x);
                        y = fast_exp2(y);
                        l[i] = n == 0 ? make_pair(x, y) : add2(l[i], make_pair(x, y));
                    }
                    if (n & 1) gather16<D, L::kPlanes>(s[n - 1], s[n], tile + P::kBehind + (n - 1) * 8 * 2 * D, P::kPlane, lane, o);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float l0, l1;
                    split_pair(l[i], l0, l1);
                    sum[i] += l0 + l1;
                }
            });
        }
        pipe.release();
        if (step++ * N < keys) continue;
        if (busy) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float l = sum[i];
                l += __shfl_xor_sync(0xffffffffu, l, 1);
                l += __shfl_xor_sync(0xffffffffu, l, 2);
                const int row = warp * 16 + i * 8 + (lane >> 2);
                if (row < unit.rows) {
                    const float inv = l == 0.0f ? 0.0f : rcp_approx(l);      // no keys, or none that is not -inf: zeros
                    const size_t at_row = (unit.image * (unsigned)(g.H * g.W) + unit.pixel(g, row)) * (unsigned)g.heads + (unsigned)unit.h;
                    T* dst = out + at_row * D + 2 * (lane & 3);
#pragma unroll
                    for (int n = 0; n < D / 8; ++n) store2(dst + n * 8, o[n][2 * i] * inv, o[n][2 * i + 1] * inv);
                    float less, same;
                    split_pair(bases[i], less, same);
                    if ((lane & 3) == 0) lse[at_row] = (log2_approx(l) - less) * kLn2;      // log 0 is -infinity
                }
            }
        }
        step = 0;
        ++item;
    }
}

template <typename T, int D>
cudaError_t launch_forward(const Geometry& g, long long B, const void* q, const void* k, const void* v, const int* idx, void* out, float* lse, int sms,
                           cudaStream_t stream) {
    constexpr size_t smem = ForwardPipe<T, D>::kSmem;
    int ctas = 0;
    const cudaError_t e = resident<sparse_forward_kernel<T, D>, smem>(sms, &ctas);
    if (e != cudaSuccess) return e;
    const unsigned units = (unsigned)(B * g.blocks * g.tiles * g.heads), grid = units < (unsigned)ctas ? units : (unsigned)ctas;
    return launch_chained(sparse_forward_kernel<T, D>, dim3(grid), kBlock, smem, stream, g, units,
                          static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v), idx, static_cast<T*>(out), lse);
}

}  // namespace sparse

cudaError_t launch_sparse_forward(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const void* q, const void* k,
                                  const void* v, const int* idx, void* out, float* lse, int sms, cudaStream_t stream) {
    using namespace sparse;
    g.complete();
    if (dtype == SLIDE_ATTN_BF16) {
        if (head_dim == 16) return launch_forward<__nv_bfloat16, 16>(g, B, q, k, v, idx, out, lse, sms, stream);
        if (head_dim == 32) return launch_forward<__nv_bfloat16, 32>(g, B, q, k, v, idx, out, lse, sms, stream);
        return launch_forward<__nv_bfloat16, 64>(g, B, q, k, v, idx, out, lse, sms, stream);
    }
    if (head_dim == 16) return launch_forward<float, 16>(g, B, q, k, v, idx, out, lse, sms, stream);
    if (head_dim == 32) return launch_forward<float, 32>(g, B, q, k, v, idx, out, lse, sms, stream);
    return launch_forward<float, 64>(g, B, q, k, v, idx, out, lse, sms, stream);
}

}  // namespace slide_attn
