// Block-sparse attention, backward.  With P the softmax weights (computed again from the stored logarithms of the sums) and
// delta = sum_d dout out of each query:
//
//   dS = P (dout v^T - delta),   dq = dS k / sqrt(d),   dk = dS^T q / sqrt(d),   dv = P^T dout
//
// Three launches: each query's logarithm and delta, side by side; queries (dq, over the blocks of their list); keys (dk and dv, over the blocks of
// queries whose lists name the key's block, found by going through the image's lists in their order).  None adds to memory that
// another CTA writes, so results do not depend on which CTA runs first.
#include "operators.cuh"

namespace slide_attn {

namespace sparse {

template <typename T, int D> using BackwardPipe = QueryPipe<T, D, sizeof(T) == 4 ? 32 : 64, sizeof(T) == 4 && D == 64 ? 3 : 4, 2>;

// The logarithm to base 2 of a row's sum.  A row that has none (no keys, or none but -inf) has no weights: exp2 of less infinity.
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

// Less each query's logarithm of the sum (base 2), and less its delta: a query and head by as many neighbouring lanes as it has 16-byte pieces.
template <typename T, int D>
__global__ void __launch_bounds__(256) sparse_rows_kernel(long long n, const T* out, const T* dout, const float* lse, float2* stats)
{
    constexpr int kPiece = 16 / sizeof(T), kLanes = D / kPiece, kEach = 4, kAtOnce = 256 / kLanes;
    grid_dependency_wait();
    const int lane = threadIdx.x % kLanes;
    const long long first = (long long)blockIdx.x * (kAtOnce * kEach) + threadIdx.x / kLanes;
    float s[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long row = first + i * kAtOnce;
        s[i] = row < n ? dot_piece<T>(dout + row * D + lane * kPiece, out + row * D + lane * kPiece) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
#pragma unroll
        for (int o = kLanes / 2; o > 0; o /= 2) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
        const long long row = first + i * kAtOnce;
        if (row < n && lane == 0) stats[row] = make_float2(-log2_of_sum(lse[row]), -s[i]);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kBlock, sizeof(T) == 4 ? D == 64 ? 1 : 3 : D == 64 ? 3 : 4)
sparse_queries_kernel(const Geometry g, unsigned units, const T* q, const T* k, const T* v, const int* idx, const T* dout, const float2* stats, T* dq)
{
    using P = BackwardPipe<T, D>;
    using L = Layout<T, D>;
    constexpr int N = P::N, NT = N / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = uniform((int)threadIdx.x / 32), lane = threadIdx.x % 32;
    constexpr float scale = root<D>();

    grid_dependency_wait();
    grid_launch_dependents();                                // the keys' kernel needs nothing of this one
    P pipe(smem, units);
    if (warp == kThreads / 32) {
        pipe.copy_all(g, q, dout, k, v, idx);
        return;
    }

    Unit unit;
    Rows<D, L::kPlanes> rows_q, rows_g;
    float dqs[D / 8][4];
    const pair scales = make_pair(scale * kLog2e, scale * kLog2e);
    pair sums[2], deltas[2];                                 // less the logarithm, less delta; each twice
    int item = 0, step = 0, keys = 0;
    while (item < pipe.items) {
        const uint32_t at = pipe.next();
        if (step == 0) {
            unit.find(g, pipe.first + item);
            keys = uniform(pipe.rows_of(item));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = warp * 16 + i * 8 + (lane >> 2);
                float2 stat = make_float2(-INFINITY, 0.0f);
                if (row < unit.rows) stat = stats[(unit.image * (unsigned)(g.H * g.W) + unit.pixel(g, row)) * (unsigned)g.heads + (unsigned)unit.h];
                sums[i] = make_pair(stat.x, stat.x);
                deltas[i] = make_pair(stat.y, stat.y);
            }
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) dqs[n][e] = 0.0f;
        }
        const bool busy = warp * 16 < unit.rows;
        if (step < P::kOwnSteps) {
            pipe.take(at, step, warp * 16, lane, rows_q, &rows_g);
        } else {
            const uint32_t tile = pipe.tile(at);
            const int used = min(N, keys - (step - P::kOwnSteps) * N);
            if (busy) with_width<NT>(used, [&](auto width, auto partial) {
                constexpr int W = decltype(width)::value;
#pragma unroll (L::kSplit ? 1 : W / 2)
                for (int n = 0; n < W; n += 2) {             // 16 columns at a time
                    float s[2][4], dp[2][4];
                    const uint32_t at16 = tile + n * 8 * 2 * D;
                    scores16<D, L::kPlanes>(rows_q, at16, P::kPlane, lane, s[0], s[1]);
                    scores16<D, L::kPlanes>(rows_g, at16 + P::kBehind, P::kPlane, lane, dp[0], dp[1]);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float x, y;
                            split_pair(fma2(make_pair(s[j][2 * i], s[j][2 * i + 1]), scales, sums[i]), x, y);
                            x = fast_exp2(x);
                            y = fast_exp2(y);
                            split_pair(mul2(make_pair(x, y), add2(make_pair(dp[j][2 * i], dp[j][2 * i + 1]), deltas[i])), s[j][2 * i], s[j][2 * i + 1]);
                        }
                    if (decltype(partial)::value && (W == 2 || n >= W / 2)) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if ((n + j) * 8 + 2 * (lane & 3) + (e & 1) >= used) s[j][e] = 0.0f;
                    }
                    gather16<D, L::kPlanes>(s[0], s[1], at16, P::kPlane, lane, dqs);
                }
            });
        }
        pipe.release();
        ++step;
        if (step < P::kOwnSteps || (step - P::kOwnSteps) * N < keys) continue;
        if (busy) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = warp * 16 + i * 8 + (lane >> 2);
                if (row < unit.rows) {
                    T* dst = dq + unit.plane(g, D) + (size_t)unit.pixel(g, row) * (unsigned)(g.heads * D) + 2 * (lane & 3);
#pragma unroll
                    for (int n = 0; n < D / 8; ++n) store2(dst + n * 8, dqs[n][2 * i] * scale, dqs[n][2 * i + 1] * scale);
                }
            }
        }
        step = 0;
        ++item;
    }
}

constexpr int kScanEach = 8, kScan = kScanEach * kThreads;      // entries of the image's lists that the keys' kernel looks at in one go
constexpr int kListed = kScan + 512;                            // entries that it lists before it goes through them

template <typename T, int D> struct KeysPlan {
    using L = Layout<T, D>;
    static constexpr int N = BackwardPipe<T, D>::N, S = BackwardPipe<T, D>::S;
    static constexpr uint32_t kTile = N * L::kRowBytes, kStage = 2 * kTile, kOwn = kRows * L::kRowBytes;
    static constexpr uint32_t kPlane = 2 * N * 2 * D, kOwnPlane = kRows * 2 * D, kBehind = L::kSplit ? kPlane / 2 : kTile;
    // fp32: the rows that stay arrive where the stages are, and what stays are their planes
    static constexpr uint32_t kPartsAt = S * kStage, kOwnAt = L::kSplit ? 0 : kPartsAt, kOwnPartsAt = kPartsAt + (L::kSplit ? 3 * kPlane : 0);
    static constexpr uint32_t kListAt = kOwnPartsAt + (L::kSplit ? 6 * kOwnPlane : 2 * kOwn), kStatsAt = kListAt + kListed * sizeof(Entry);
    static constexpr size_t kSmem = kStatsAt + S * N * sizeof(float2);
    static_assert(!L::kSplit || 2 * kOwn <= kPartsAt, "room for the rows that stay");
};

template <typename T, int D>
__global__ void __launch_bounds__(kBlock, sizeof(T) == 4 ? D == 64 ? 1 : 2 : D == 64 ? 2 : 3)
sparse_keys_kernel(const Geometry g, const T* q, const T* k, const T* v, const int* idx, const float2* stats, const T* dout, T* dk, T* dv)
{
    using K = KeysPlan<T, D>;
    using L = Layout<T, D>;
    constexpr int N = K::N, NT = N / 8, S = K::S;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ unsigned warp_sums[kThreads / 32];
    const uint32_t base = smem_u32(smem);
    Entry* list = reinterpret_cast<Entry*>(smem + K::kListAt);
    const float* columns = reinterpret_cast<const float*>(smem + K::kStatsAt);          // of each stage: less the logarithms, then less the deltas
    const int warp = uniform((int)threadIdx.x / 32), lane = threadIdx.x % 32;
    const bool copying = warp == kThreads / 32;
    constexpr float scale = root<D>();

    // No wait here: this kernel starts when every CTA of the queries' kernel has waited for what was launched before the two, and takes nothing
    // from it.  The wait for it is at the end.
    Unit unit;
    unit.find(g, blockIdx.x);
    if (unit.rows <= 0) return;                              // (part 0 of each block has rows)
    const size_t plane = unit.plane(g, D);
    const unsigned pixel_bytes = (unsigned)(g.heads * D * (int)sizeof(T));
    if (copying) {
        unsigned pixels[kRows / 32];
#pragma unroll
        for (int i = 0; i < kRows / 32; ++i) pixels[i] = unit.pixel(g, lane + 32 * i);
        Sender<T, D, kRows>::send(base + K::kOwnAt, base + K::kOwnAt + K::kOwn, k + plane, v + plane, pixel_bytes, pixels, unit.rows, lane);
        copies_commit();
    }
    const bool busy = warp * 16 < unit.rows;
    Rows<D, L::kPlanes> rows_k, rows_v;
    float dks[D / 8][4] = {}, dvs[D / 8][4] = {};
    const pair scales = make_pair(scale * kLog2e, scale * kLog2e);
    const int* lists = idx + unit.list * (unsigned)(g.blocks * g.top);
    const int entries = g.blocks * g.top;
    for (int seen = 0; seen < entries;) {
        // the next blocks of queries that see this block, in an order that the lists alone decide
        const bool start = seen == 0;
        unsigned listed = 0;                                 // blocks << 21 | rows: at most 1536 blocks of 1024
        do {
            int mine[kScanEach];
            unsigned sum = 0;
            if (!copying) {
#pragma unroll
                for (int e = 0; e < kScanEach; ++e) {
                    const int i = seen + e * kThreads + (int)threadIdx.x;
                    mine[e] = i < entries ? lists[i] : -1;
                }
#pragma unroll
                for (int e = 0; e < kScanEach; ++e) {
                    const bool is = mine[e] == unit.r;
                    mine[e] = is ? (int)g.by_top.quotient((unsigned)(seen + e * kThreads) + threadIdx.x) : -1;
                    if (is) sum += (1u << 21) + (unsigned)block_of(g, mine[e]).size();
                }
            }
            unsigned before = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const unsigned x = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += x;
            }
            if (lane == 31 && !copying) warp_sums[warp] = before;
            __syncthreads();
            before += listed - sum;
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) {
                if (w < warp) before += warp_sums[w];
                listed += warp_sums[w];
            }
            if (!copying) {
#pragma unroll
                for (int e = 0; e < kScanEach; ++e)
                    if (mine[e] >= 0) {
                        const Block block = block_of(g, mine[e]);
                        const unsigned place = before >> 21;
                        before += (1u << 21) + (unsigned)block.size();
                        list[place] = Entry::of(g, block, (int)(before & 0x1FFFFFu));
                    }
            }
            seen += kScan;
            if (start && copying) copies_wait<0>();
            __syncthreads();
        } while (seen < entries && (int)(listed >> 21) + kScan <= kListed);
        if (start) {                                         // the rows that stay have arrived
            if (!copying) {
                if constexpr (L::kSplit)
#pragma unroll
                    for (int o = 0; o < 2; ++o) cut_rows<D, kRows>(base + K::kOwnAt + o * K::kOwn, base + K::kOwnPartsAt + o * 3 * K::kOwnPlane);
                rows_k.load(L::kSplit ? base + K::kOwnPartsAt : base + K::kOwnAt, K::kOwnPlane, warp * 16, lane);
                rows_v.load(L::kSplit ? base + K::kOwnPartsAt + 3 * K::kOwnPlane : base + K::kOwnAt + K::kOwn, K::kOwnPlane, warp * 16, lane);
            }
            if constexpr (L::kSplit) __syncthreads();        // the stages are free
        }
        const int total = uniform((int)(listed & 0x1FFFFFu));
        if (copying) {
            Ring<S> ring;
            Cursor cursor;
            cursor.reset(list);
            const float2* from_stats = stats + unit.image * (unsigned)(g.H * g.W) * (unsigned)g.heads + (unsigned)unit.h;
#pragma unroll 1
            for (int done = 0; done < total; done += N) {
                unsigned pixels[N / 32];
#pragma unroll
                for (int i = 0; i < N / 32; ++i) pixels[i] = done + 32 * i + lane < total ? cursor.pixel(g, done + 32 * i + lane) : 0u;
                ring.claim();
                const uint32_t stage = base + (uint32_t)ring.slot * K::kStage, at = base + K::kStatsAt + (uint32_t)(ring.slot * 2 * N * 4);
                Sender<T, D, N>::send(stage, stage + K::kTile, q + plane, dout + plane, pixel_bytes, pixels, total - done, lane);
#pragma unroll
                for (int i = 0; i < N / 32; ++i)
                    if (done + 32 * i + lane < total) {
                        const float* from = reinterpret_cast<const float*>(from_stats + (size_t)pixels[i] * (unsigned)g.heads);
                        copy4(at + (32 * i + lane) * 4, from);
                        copy4(at + (N + 32 * i + lane) * 4, from + 1);
                    }
                ring.commit();
            }
            ring.finish();
        } else {
            int slot = 0;
#pragma unroll 1
            for (int done = 0; done < total; done += N) {
                bar_sync<kBlock>(Ring<S>::full(slot));
                uint32_t tile = base + (uint32_t)slot * K::kStage;
                if constexpr (L::kSplit) {
                    compute_sync();
                    cut_rows<D, 2 * N>(tile, base + K::kPartsAt);
                    compute_sync();
                    tile = base + K::kPartsAt;
                }
                const pair* stat = reinterpret_cast<const pair*>(columns + slot * 2 * N) + (lane & 3);       // of two queries each
                const int used = min(N, total - done);
                if (busy) with_width<NT>(used, [&](auto width, auto partial) {
                    constexpr int W = decltype(width)::value;
#pragma unroll (L::kSplit ? 1 : W / 2)
                    for (int n = 0; n < W; n += 2) {             // 16 columns at a time
                        float s[2][4], dp[2][4];
                        const uint32_t at16 = tile + n * 8 * 2 * D;
                        scores16<D, L::kPlanes>(rows_k, at16, K::kPlane, lane, s[0], s[1]);
                        scores16<D, L::kPlanes>(rows_v, at16 + K::kBehind, K::kPlane, lane, dp[0], dp[1]);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const pair sums = stat[(n + j) * 4], deltas = stat[N / 2 + (n + j) * 4];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                float& x = s[j][2 * i];
                                float& y = s[j][2 * i + 1];
                                split_pair(fma2(make_pair(x, y), scales, sums), x, y);
                                x = fast_exp2(x);
                                y = fast_exp2(y);
                                split_pair(mul2(make_pair(x, y), add2(make_pair(dp[j][2 * i], dp[j][2 * i + 1]), deltas)), dp[j][2 * i], dp[j][2 * i + 1]);
                            }
                        }
                        if (decltype(partial)::value && (W == 2 || n >= W / 2)) {        // (a key that is not finite makes a NaN of rows that hold nothing)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if ((n + j) * 8 + 2 * (lane & 3) + (e & 1) >= used) s[j][e] = dp[j][e] = 0.0f;
                        }
                        gather16<D, L::kPlanes>(s[0], s[1], at16 + K::kBehind, K::kPlane, lane, dvs);
                        gather16<D, L::kPlanes>(dp[0], dp[1], at16, K::kPlane, lane, dks);
                    }
                });
                bar_arrive<kBlock>(Ring<S>::empty(slot));
                slot = Ring<S>::after(slot);
            }
        }
        __syncthreads();                                     // the list is free again
    }
    if (copying) grid_dependency_wait();                     // complete only when the queries' kernel is
    if (copying || !busy) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = warp * 16 + i * 8 + (lane >> 2);
        if (row >= unit.rows) continue;
        const size_t at = plane + (size_t)unit.pixel(g, row) * (unsigned)(g.heads * D) + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
            store2(dk + at + n * 8, dks[n][2 * i] * scale, dks[n][2 * i + 1] * scale);
            store2(dv + at + n * 8, dvs[n][2 * i], dvs[n][2 * i + 1]);
        }
    }
}

template <typename T, int D>
cudaError_t launch_backward(const Geometry& g, long long B, const BackwardMaps& m, float2* stats, int sms, cudaStream_t stream) {
    constexpr size_t smem_q = BackwardPipe<T, D>::kSmem, smem_k = KeysPlan<T, D>::kSmem;
    int ctas = 0, ctas_k = 0;
    cudaError_t e = resident<sparse_queries_kernel<T, D>, smem_q>(sms, &ctas);
    if (e == cudaSuccess) e = resident<sparse_keys_kernel<T, D>, smem_k>(sms, &ctas_k);
    if (e != cudaSuccess) return e;
    const unsigned units = (unsigned)(B * g.blocks * g.tiles * g.heads), grid = units < (unsigned)ctas ? units : (unsigned)ctas;
    const long long n = B * g.H * g.W * g.heads;
    auto in = [](const void* p) { return static_cast<const T*>(p); };
    auto to = [](void* p) { return static_cast<T*>(p); };
    constexpr long long rows = 256 / (D * sizeof(T) / 16) * 4;      // of a block
    e = launch_chained(sparse_rows_kernel<T, D>, dim3((unsigned)((n + rows - 1) / rows)), 256, 0, stream, n, in(m.out), in(m.dout), m.lse, stats);
    if (e != cudaSuccess) return e;
    e = launch_chained(sparse_queries_kernel<T, D>, dim3(grid), kBlock, smem_q, stream, g, units, in(m.q), in(m.k),
                       in(m.v), m.idx, in(m.dout), static_cast<const float2*>(stats), to(m.dq));
    if (e != cudaSuccess) return e;
    return launch_chained(sparse_keys_kernel<T, D>, dim3(units), kBlock, smem_k, stream, g, in(m.q), in(m.k), in(m.v), m.idx,
                          static_cast<const float2*>(stats), in(m.dout), to(m.dk), to(m.dv));
}

}  // namespace sparse

cudaError_t launch_sparse_backward(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const sparse::BackwardMaps& m,
                                   void* workspace, int sms, cudaStream_t stream) {
    using namespace sparse;
    g.complete();
    float2* stats = static_cast<float2*>(workspace);
    if (dtype == SLIDE_ATTN_BF16) {
        if (head_dim == 16) return launch_backward<__nv_bfloat16, 16>(g, B, m, stats, sms, stream);
        if (head_dim == 32) return launch_backward<__nv_bfloat16, 32>(g, B, m, stats, sms, stream);
        return launch_backward<__nv_bfloat16, 64>(g, B, m, stats, sms, stream);
    }
    if (head_dim == 16) return launch_backward<float, 16>(g, B, m, stats, sms, stream);
    if (head_dim == 32) return launch_backward<float, 32>(g, B, m, stats, sms, stream);
    return launch_backward<float, 64>(g, B, m, stats, sms, stream);
}

}  // namespace slide_attn
