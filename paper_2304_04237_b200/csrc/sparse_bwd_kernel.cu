// Block-sparse attention, backward.  With P the softmax weights (computed again from the stored logarithms of the sums) and
// delta = sum_d dout out of each query:
//
//   dS = P (dout v^T - delta),   dq = dS k / sqrt(d),   dk = dS^T q / sqrt(d),   dv = P^T dout
//
// Three launches: each query's logarithm and delta, side by side; queries (dq, over the blocks of their list); keys (dk and dv, over the blocks of
// queries whose lists name the key's block, found by going through the image's lists in their order).  None adds to memory that
// another CTA writes, so results do not depend on which CTA runs first.
// Bound by latency: a warp's products, exponentials and products again wait for one another, and registers allow 12 to 16 such warps an SM.  128 x 128 x 2,
// 3 heads, bf16, lists of 16 blocks of 8 x 8: queries 74 us, keys 104 (tensor pipe 50 and 44 %, issue slots 40 and 33 %); with the forward 231 in all, of 27 for the
// products at the rate of large matrices.
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
__global__ void __launch_bounds__(256) sparse_rows_kernel(long long n, const T* out, const T* dout, const float* lse, float2* stats, unsigned* taken)
{
    constexpr int kPiece = 16 / sizeof(T), kLanes = D / kPiece, kEach = 4, kAtOnce = 256 / kLanes;
    grid_dependency_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *taken = 0;
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

constexpr int kScanEach = 2, kScan = 128 * kScanEach;    // entries of the image's lists that are looked at in one go: four neighbours a lane, again and again
constexpr int kListed = 4 * kScan;                              // entries that a table holds

// Shared memory of the keys' kernel: the pipe's, two tables, of each stage the queries' numbers (less the logarithms, then less the deltas) and a
// word on what the stage holds.
template <typename T, int D> struct KeysPlan {
    using P = BackwardPipe<T, D>;
    static constexpr uint32_t kListAt = (uint32_t)(P::kSmem + 15) / 16 * 16, kStatsAt = kListAt + 2 * kListed * sizeof(Entry);
    static constexpr uint32_t kWordsAt = kStatsAt + P::S * P::N * sizeof(float2);
    static constexpr size_t kSmem = kWordsAt + P::S * sizeof(unsigned);
};
constexpr unsigned kLast = 1u << 16;                            // the unit's last tile; below: its rows

// The blocks of queries that see a block, in the order of the lists, found by a warp.
struct Seers {
    Unit unit;
    Entry* table;
    int seen, n, total;                                         // entries looked at; of the table; their rows
    int4 mine[kScanEach];
    __device__ __forceinline__ void begin(const Geometry& g, unsigned u, Entry* room) {
        unit.find(g, u);
        table = room;
        seen = n = total = 0;
    }
    __device__ __forceinline__ bool room(const Geometry& g) const { return seen < g.blocks * g.top && n + kScan <= kListed; }
    // Entries sent for, and looked at.
    __device__ __forceinline__ void read(const Geometry& g, const int* idx, int lane) {
        const int entries = g.blocks * g.top;
        const int* lists = idx + unit.list * (unsigned)entries;
#pragma unroll
        for (int e = 0; e < kScanEach; ++e) {
            const int i = seen + e * 128 + lane * 4;
            mine[e] = make_int4(-1, -1, -1, -1);
            if (entries % 4 == 0) {
                if (i < entries) mine[e] = *reinterpret_cast<const int4*>(lists + i);
            } else {
                if (i < entries) mine[e].x = lists[i];
                if (i + 1 < entries) mine[e].y = lists[i + 1];
                if (i + 2 < entries) mine[e].z = lists[i + 2];
                if (i + 3 < entries) mine[e].w = lists[i + 3];
            }
        }
    }
    __device__ __forceinline__ void look(const Geometry& g, int lane) {
#pragma unroll
        for (int e = 0; e < kScanEach; ++e) {
            const int4 m = mine[e];
            const bool is[4] = {m.x == unit.r, m.y == unit.r, m.z == unit.r, m.w == unit.r};
            if (!__any_sync(0xffffffffu, is[0] || is[1] || is[2] || is[3])) continue;
            Block block[4] = {};
            unsigned own = 0;                                    // blocks << 24 | rows
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (is[j]) {
                    block[j] = block_of(g, (int)g.by_top.quotient((unsigned)(seen + e * 128 + lane * 4 + j)));
                    own += (1u << 24) + (unsigned)block[j].size();
                }
            unsigned before = own;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const unsigned x = __shfl_up_sync(0xffffffffu, before, d);
                if (lane >= d) before += x;
            }
            const unsigned all = __shfl_sync(0xffffffffu, before, 31);
            before -= own;
            int place = n + (int)(before >> 24), end = total + (int)(before & 0xFFFFFFu);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (is[j]) {
                    end += block[j].size();
                    table[place++] = Entry::of(g, block[j], end);
                }
            n += (int)(all >> 24);
            total += (int)(all & 0xFFFFFFu);
        }
        seen += kScan;
    }
};

// What the copying warp of the keys' kernel does.  Units are taken from a counter, one ahead: how many blocks see a block is known only when the lists have been
// gone through, and a fixed share of the units would leave the CTAs with the sought-after blocks behind.  While a unit's tiles are sent for, the next one's
// lists are gone through, a part beside each tile.
template <typename T, int D>
__device__ __forceinline__ void send_seers(const Geometry& g, unsigned units, unsigned char* smem, const T* q, const T* k, const T* v, const int* idx,
                                           const float2* stats, const T* dout, unsigned* taken) {
    using K = KeysPlan<T, D>;
    using P = BackwardPipe<T, D>;
    constexpr int N = P::N;
    const int lane = threadIdx.x % 32;
    const uint32_t base = smem_u32(smem);
    Entry* tables = reinterpret_cast<Entry*>(smem + K::kListAt);
    unsigned* words = reinterpret_cast<unsigned*>(smem + K::kWordsAt);
    const unsigned pixel_bytes = (unsigned)(g.heads * D * (int)sizeof(T));
    Ring<P::S> ring;
    auto ask = [&]() { return lane == 0 ? atomicAdd(taken, 1u) : 0u; };
    auto take = [&](unsigned asked) {                            // the next unit that has rows
        for (;;) {
            const unsigned u = __shfl_sync(0xffffffffu, asked, 0);
            if (u >= units) return units;
            Unit unit;
            unit.find(g, u);
            if (unit.rows > 0) return u;
            asked = ask();
        }
    };
    Seers next;
    unsigned u = take(ask()), turn = 0;
    if (u < units) next.begin(g, u, tables);
#pragma unroll 1
    while (u < units) {
        const Unit unit = next.unit;
        Entry* const table = next.table;
        const unsigned asked = ask();                            // for the unit after this one, on its way
        // the rows that stay
        const size_t plane = unit.plane(g, D);
        {
            unsigned pixels[kRows / 32];
#pragma unroll
            for (int i = 0; i < kRows / 32; ++i) pixels[i] = unit.pixel(g, lane + 32 * i);
#pragma unroll
            for (int o = 0; o < P::kOwnSteps; ++o) {
                ring.claim();
                const uint32_t stage = base + (uint32_t)ring.slot * P::kStage;
                if (lane == 0) words[ring.slot] = u;
                if constexpr (P::kOwnSteps == 1)
                    Sender<T, D, kRows>::send(stage, stage + P::kOwn, k + plane, v + plane, pixel_bytes, pixels, unit.rows, lane);
                else
                    Sender<T, D, kRows>::send(stage, 0, (o ? v : k) + plane, nullptr, pixel_bytes, pixels, unit.rows, lane);
                ring.commit();
            }
        }
        if (next.room(g)) ring.drain();
        const float2* from_stats = stats + unit.image * (unsigned)(g.H * g.W) * (unsigned)g.heads + (unsigned)unit.h;
        bool last = false, ahead = false;                        // ahead: `next` is the unit after this one
        unsigned u_next = units;
        while (!last) {
            // what is left of this unit's lists, as far as the table goes
            while (next.room(g)) {
                next.read(g, idx, lane);
                next.look(g, lane);
            }
            __syncwarp();
            const int total = next.total;
            const bool whole = next.seen >= g.blocks * g.top;    // no more tables of this unit
            if (whole) {
                u_next = take(asked);
                ahead = u_next < units;
                if (ahead) next.begin(g, u_next, tables + (turn ^= 1u) * kListed);
            }
            const int looks = max((g.blocks * g.top / kScan + 1) * N / max(total, 1), 1);       // at each tile: about all of the lists in all
            Cursor cursor;
            cursor.reset(table);
            int done = 0;
#pragma unroll 1
            do {
                if (done >= total && !whole) break;              // an empty table, and more of them
                const bool look = ahead && next.room(g);
                if (look) next.read(g, idx, lane);               // on its way while this tile is sent for
                unsigned pixels[N / 32];
#pragma unroll
                for (int i = 0; i < N / 32; ++i) pixels[i] = done + 32 * i + lane < total ? cursor.pixel(g, done + 32 * i + lane) : 0u;
                ring.claim();
                last = whole && done + N >= total;
                if (lane == 0) words[ring.slot] = (unsigned)max(min(N, total - done), 0) | (last ? kLast : 0u);
                const uint32_t stage = base + (uint32_t)ring.slot * P::kStage, at = base + K::kStatsAt + (uint32_t)(ring.slot * 2 * N * 4);
                if (total > 0) Sender<T, D, N>::send(stage, stage + P::kTile, q + plane, dout + plane, pixel_bytes, pixels, total - done, lane);
#pragma unroll
                for (int i = 0; i < N / 32; ++i)
                    if (done + 32 * i + lane < total) {
                        const float* from = reinterpret_cast<const float*>(from_stats + (size_t)pixels[i] * (unsigned)g.heads);
                        copy4(at + (32 * i + lane) * 4, from);
                        copy4(at + (N + 32 * i + lane) * 4, from + 1);
                    }
                ring.commit();
                if (look) next.look(g, lane);
#pragma unroll 1
                for (int i = 1; i < looks && ahead && next.room(g); ++i) {
                    next.read(g, idx, lane);
                    next.look(g, lane);
                }
                done += N;
            } while (done < total);
            __syncwarp();                                        // the table is free again
            if (!whole) next.n = next.total = 0;
        }
        u = u_next;
    }
    ring.claim();
    if (lane == 0) words[ring.slot] = units;                     // no more
    ring.commit();
    ring.finish();
}

template <typename T, int D>
__global__ void __launch_bounds__(kBlock, sizeof(T) == 4 ? D == 64 ? 1 : 2 : D == 64 ? 2 : 3)
sparse_keys_kernel(const Geometry g, unsigned units, const T* q, const T* k, const T* v, const int* idx, const float2* stats, const T* dout, T* dk, T* dv,
                   unsigned* taken)
{
    using K = KeysPlan<T, D>;
    using P = BackwardPipe<T, D>;
    using L = Layout<T, D>;
    constexpr int N = P::N, NT = N / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = uniform((int)threadIdx.x / 32), lane = threadIdx.x % 32;
    constexpr float scale = root<D>();

    // No wait here: this kernel starts when every CTA of the queries' kernel has waited for what was launched before the two, and takes nothing
    // from it.  The wait for it is at the end.
    if (warp == kThreads / 32) {
        send_seers<T, D>(g, units, smem, q, k, v, idx, stats, dout, taken);
        grid_dependency_wait();                              // complete only when the queries' kernel is
        return;
    }
    P pipe(smem, units);
    const float* columns = reinterpret_cast<const float*>(smem + K::kStatsAt);          // of each stage: less the logarithms, then less the deltas
    const unsigned* words = reinterpret_cast<const unsigned*>(smem + K::kWordsAt);
    const pair scales = make_pair(scale * kLog2e, scale * kLog2e);
    for (;;) {
        uint32_t own = pipe.next();
        const unsigned u = (unsigned)uniform((int)words[pipe.slot]);
        if (u >= units) {
            pipe.release();
            return;
        }
        Unit unit;
        unit.find(g, u);
        const bool busy = warp * 16 < unit.rows;
        Rows<D, L::kPlanes> rows_k, rows_v;
        float dks[D / 8][4] = {}, dvs[D / 8][4] = {};
#pragma unroll
        for (int o = 0; o < P::kOwnSteps; ++o) {
            if (o) own = pipe.next();
            pipe.take(own, o, warp * 16, lane, rows_k, &rows_v);
            pipe.release();
        }
        for (bool last = false; !last;) {
            const uint32_t at = pipe.next();
            const unsigned word = (unsigned)uniform((int)words[pipe.slot]);
            const int used = (int)(word & (kLast - 1u));
            last = word >= kLast;
            if (used > 0) {
                const uint32_t tile = pipe.tile(at);
                const pair* stat = reinterpret_cast<const pair*>(columns + pipe.slot * 2 * N) + (lane & 3);       // of two queries each
                if (busy) with_width<NT>(used, [&](auto width, auto partial) {
                    constexpr int W = decltype(width)::value;
#pragma unroll (L::kSplit ? 1 : W / 2)
                    for (int n = 0; n < W; n += 2) {             // 16 columns at a time
                        float s[2][4], dp[2][4];
                        const uint32_t at16 = tile + n * 8 * 2 * D;
                        scores16<D, L::kPlanes>(rows_k, at16, P::kPlane, lane, s[0], s[1]);
                        scores16<D, L::kPlanes>(rows_v, at16 + P::kBehind, P::kPlane, lane, dp[0], dp[1]);
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
                        gather16<D, L::kPlanes>(s[0], s[1], at16 + P::kBehind, P::kPlane, lane, dvs);
                        gather16<D, L::kPlanes>(dp[0], dp[1], at16, P::kPlane, lane, dks);
                    }
                });
            }
            pipe.release();
        }
        if (!busy) continue;
        const size_t plane = unit.plane(g, D);
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
}

template <typename T, int D>
cudaError_t launch_backward(const Geometry& g, long long B, const BackwardMaps& m, float2* stats, unsigned* taken, int sms, cudaStream_t stream) {
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
    e = launch_chained(sparse_rows_kernel<T, D>, dim3((unsigned)((n + rows - 1) / rows)), 256, 0, stream, n, in(m.out), in(m.dout), m.lse, stats, taken);
    if (e != cudaSuccess) return e;
    e = launch_chained(sparse_queries_kernel<T, D>, dim3(grid), kBlock, smem_q, stream, g, units, in(m.q), in(m.k),
                       in(m.v), m.idx, in(m.dout), static_cast<const float2*>(stats), to(m.dq));
    if (e != cudaSuccess) return e;
    return launch_chained(sparse_keys_kernel<T, D>, dim3(units < (unsigned)ctas_k ? units : (unsigned)ctas_k), kBlock, smem_k, stream, g, units, in(m.q), in(m.k),
                          in(m.v), m.idx, static_cast<const float2*>(stats), in(m.dout), to(m.dk), to(m.dv), taken);
}

}  // namespace sparse

cudaError_t launch_sparse_backward(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const sparse::BackwardMaps& m,
                                   void* workspace, int sms, cudaStream_t stream) {
    using namespace sparse;
    g.complete();
    float2* stats = static_cast<float2*>(workspace);             // and behind them the counter of the units that are taken
    unsigned* taken = reinterpret_cast<unsigned*>(stats + B * g.H * g.W * g.heads);
    if (dtype == SLIDE_ATTN_BF16) {
        if (head_dim == 16) return launch_backward<__nv_bfloat16, 16>(g, B, m, stats, taken, sms, stream);
        if (head_dim == 32) return launch_backward<__nv_bfloat16, 32>(g, B, m, stats, taken, sms, stream);
        return launch_backward<__nv_bfloat16, 64>(g, B, m, stats, taken, sms, stream);
    }
    if (head_dim == 16) return launch_backward<float, 16>(g, B, m, stats, taken, sms, stream);
    if (head_dim == 32) return launch_backward<float, 32>(g, B, m, stats, taken, sms, stream);
    return launch_backward<float, 64>(g, B, m, stats, taken, sms, stream);
}

}  // namespace slide_attn
