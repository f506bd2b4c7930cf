// Block-sparse attention, backward.  With P the softmax weights (computed again from the stored logarithms of the sums) and
// delta = sum_d dout out of each query:
//
//   dS = P (dout v^T - delta),   dq = dS k / sqrt(d),   dk = dS^T q / sqrt(d),   dv = P^T dout
//
// Three launches: each query's logarithm and delta, side by side, and the lists turned round; queries (dq, over the blocks of their list); keys (dk
// and dv, over the blocks of queries whose lists name the key's block, in the order of the lists).  None adds to memory that
// another CTA writes, so results do not depend on which CTA runs first.
// Bound by latency: a warp's products, exponentials and products again wait for one another, and registers allow 12 to 16 such warps an SM.  128 x 128 x 2,
// 3 heads, bf16, lists of 16 blocks of 8 x 8: queries 80 us, keys 101 by themselves (tensor pipe 46 and 48 %, issue slots 35 and 31 %); with the forward 230 in
// all, of 27 for the products at the rate of large matrices.  fp32 heads of 64 have one CTA an SM, as registers and shared memory allow: 8 x 56 x 56, 3 heads, 4 blocks of
// 7 x 7, 464 us where heads of 32 take 208.
//
// Tiles of 32 or 64 rows, us each way, backward alone (64 x 56 x 56 x 2, 4 blocks of 7 x 7, fp32 8 x 56 x 56 x 3; then 2 x 128 x 128 x 3, 16 blocks of 8 x 8,
// fp32 8 blocks):
//   bf16, heads of 32: 224.9 / 214.7, then 182.4 / 172.2; heads of 64: 397.6 / 373.7, then 317 / 291; heads of 16 (32 x 56 x 56 x 4) 168.8 / 156.3.  64
//   fp32, heads of 32: 207.5 / 233.9, then 456 / 502; heads of 16 (8 x 56 x 56 x 6) 223.8 / 219.7.  32
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

// What the first launch leaves in the workspace.
struct Prepared {
    float2* stats;                   // of each query and head: less its logarithm of the sum (base 2), less its delta
    unsigned* taken;                 // units that the keys' kernel has begun
    int* starts;                     // [B][heads][blocks + 1]: of each block's part of `seers`
    int* seers;                      // [B][heads][blocks top]: the blocks of queries that see a block, in the order of the lists
};
constexpr int kInvertWarps = 8;

// One image's and head's lists turned round, by a CTA: each warp counts the blocks in its part of the lists, and puts them where the counts of the warps and blocks
// ahead say.  counts: [warp][blocks]
__device__ __forceinline__ void invert(const Geometry& g, const int* lists, int* starts, int* seers, int* counts) {
    __shared__ int warp_sums[kInvertWarps];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, entries = g.blocks * g.top;
    const int each = (entries + kInvertWarps * 32 - 1) / (kInvertWarps * 32) * 32, first = warp * each, end = min(entries, first + each);
    int* own = counts + warp * g.blocks;
    for (int i = threadIdx.x; i < kInvertWarps * g.blocks; i += 32 * kInvertWarps) counts[i] = 0;
    __syncthreads();
    // f(first of 128 entries, of each lane's four the block, or -1)
    auto go = [&](auto f) {
        for (int i0 = first; i0 < end; i0 += 128) {
            int id[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = i0 + j * 32 + lane;
                id[j] = i < end ? lists[i] : -1;
                if ((unsigned)id[j] >= (unsigned)g.blocks) id[j] = -1;
            }
            f(i0, id);
        }
    };
    go([&](int, const int (&id)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (id[j] >= 0) atomicAdd(own + id[j], 1);
    });
    __syncthreads();
    // where each block's and, in it, each warp's begin; a thread takes neighbouring blocks
    const int span = (g.blocks + 32 * kInvertWarps - 1) / (32 * kInvertWarps), b0 = min(g.blocks, (int)threadIdx.x * span), b1 = min(g.blocks, b0 + span);
    int sum = 0;
    for (int b = b0; b < b1; ++b)
        for (int w = 0; w < kInvertWarps; ++w) sum += counts[w * g.blocks + b];
    int before = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int x = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += x;
    }
    if (lane == 31) warp_sums[warp] = before;
    __syncthreads();
    before -= sum;
    for (int w = 0; w < warp; ++w) before += warp_sums[w];
    for (int b = b0; b < b1; ++b) {
        starts[b] = before;
        for (int w = 0; w < kInvertWarps; ++w) {
            const int n = counts[w * g.blocks + b];
            counts[w * g.blocks + b] = before;
            before += n;
        }
    }
    if (threadIdx.x == 32 * kInvertWarps - 1) starts[g.blocks] = before;
    __syncthreads();
    go([&](int i0, const int (&id)[4]) {
        unsigned same[4];                                        // the lanes that name the same block
#pragma unroll
        for (int j = 0; j < 4; ++j) same[j] = __match_any_sync(0xffffffffu, id[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = id[j] >= 0 ? own[id[j]] : 0, rank = __popc(same[j] & ((1u << lane) - 1u));
            __syncwarp();
            if (id[j] >= 0) {
                seers[at + rank] = (int)g.by_top.quotient((unsigned)(i0 + j * 32 + lane));
                if (rank == 0) own[id[j]] = at + __popc(same[j]);
            }
            __syncwarp();
        }
    });
}

// The first CTAs turn the lists round, one each of `lists`; the others take a query and head by as many neighbouring lanes as it has 16-byte pieces.
template <typename T, int D>
__global__ void __launch_bounds__(32 * kInvertWarps) sparse_rows_kernel(const Geometry g, unsigned lists, long long n, const int* idx, const T* out,
                                                                        const T* dout, const float* lse, const Prepared to)
{
    constexpr int kPiece = 16 / sizeof(T), kLanes = D / kPiece, kEach = 4, kAtOnce = 256 / kLanes;
    static_assert(kInvertWarps == 8, "256 threads");
    extern __shared__ __align__(128) unsigned char smem[];
    grid_dependency_wait();
    if (blockIdx.x < lists) {
        if (blockIdx.x == 0 && threadIdx.x == 0) *to.taken = 0;
        const size_t entries = (size_t)(g.blocks * g.top);
        invert(g, idx + blockIdx.x * entries, to.starts + (size_t)blockIdx.x * (unsigned)(g.blocks + 1), to.seers + blockIdx.x * entries, reinterpret_cast<int*>(smem));
        return;
    }
    const int lane = threadIdx.x % kLanes;
    const long long first = (long long)(blockIdx.x - lists) * (kAtOnce * kEach) + threadIdx.x / kLanes;
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
        if (row < n && lane == 0) to.stats[row] = make_float2(-log2_of_sum(lse[row]), -s[i]);
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
    grid_launch_dependents();                                // CTAs of the keys' kernel take the places that become free, and wait there
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

constexpr int kListed = 512;                                    // entries that a table holds

// Shared memory of the keys' kernel: the pipe's, two tables, of each stage the queries' numbers (less the logarithms, then less the deltas) and a
// word on what the stage holds.
template <typename T, int D> struct KeysPlan {
    using P = BackwardPipe<T, D>;
    static constexpr uint32_t kListAt = (uint32_t)(P::kSmem + 15) / 16 * 16, kStatsAt = kListAt + 2 * kListed * sizeof(Entry);
    static constexpr uint32_t kWordsAt = kStatsAt + P::S * P::N * sizeof(float2);
    static constexpr size_t kSmem = kWordsAt + P::S * sizeof(unsigned);
};
constexpr unsigned kLast = 1u << 16;                            // the unit's last tile; below: its rows

// The blocks of queries that see a block: a table of some of them, made by a warp, 32 at a time.
struct Seers {
    Unit unit;
    Entry* table;
    const int* from;
    int left, n, total;                                         // left: not in the table yet; n: of the table; total: their rows
    int mine;
    bool reading;
    __device__ __forceinline__ void begin(const Geometry& g, unsigned u, const Prepared& by, Entry* room) {
        unit.find(g, u);
        const int* starts = by.starts + unit.list * (unsigned)(g.blocks + 1) + unit.r;
        const int start = starts[0];
        from = by.seers + unit.list * (unsigned)(g.blocks * g.top) + start;
        left = starts[1] - start;
        table = room;
        n = total = 0;
        reading = false;
    }
    __device__ __forceinline__ bool room() const { return left > 0 && n + 32 <= kListed; }
    // Half of a step: sends for 32 entries, or writes those down that were sent for.
    __device__ __forceinline__ void step(const Geometry& g, int lane) {
        if (!reading) {
            mine = lane < left ? from[lane] : -1;
            reading = true;
            return;
        }
        Block block = {};
        if (mine >= 0) block = block_of(g, mine);
        int end = block.size();
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int x = __shfl_up_sync(0xffffffffu, end, d);
            if (lane >= d) end += x;
        }
        if (mine >= 0) table[n + lane] = Entry::of(g, block, total + end);
        const int taken = min(32, left);
        n += taken;
        left -= taken;
        from += 32;
        total += __shfl_sync(0xffffffffu, end, 31);
        reading = false;
    }
};

// What the copying warp of the keys' kernel does.  Units are taken from a counter, one ahead: some blocks are seen by many more than others, and a fixed share of
// the units would leave the CTAs with these behind.  The next unit's table is made while this one's tiles are sent for.
template <typename T, int D>
__device__ __forceinline__ void send_seers(const Geometry& g, unsigned units, unsigned char* smem, const T* q, const T* k, const T* v, const T* dout,
                                           const Prepared& by) {
    using K = KeysPlan<T, D>;
    using P = BackwardPipe<T, D>;
    constexpr int N = P::N;
    const int lane = threadIdx.x % 32;
    const uint32_t base = smem_u32(smem);
    Entry* tables = reinterpret_cast<Entry*>(smem + K::kListAt);
    unsigned* words = reinterpret_cast<unsigned*>(smem + K::kWordsAt);
    const unsigned pixel_bytes = (unsigned)(g.heads * D * (int)sizeof(T));
    Ring<P::S> ring;
    auto ask = [&]() { return lane == 0 ? atomicAdd(by.taken, 1u) : 0u; };
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
    if (u < units) next.begin(g, u, by, tables);
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
        if (next.room()) ring.drain();
        const float2* from_stats = by.stats + unit.image * (unsigned)(g.H * g.W) * (unsigned)g.heads + (unsigned)unit.h;
        bool last = false, ahead = false;                        // ahead: `next` is the unit after this one
        unsigned u_next = units;
        while (!last) {
            while (next.room()) next.step(g, lane);              // what is left of this unit, as far as the table goes
            __syncwarp();
            const int total = next.total;
            const bool whole = next.left == 0;                   // no more tables of this unit
            if (whole) {
                u_next = take(asked);
                ahead = u_next < units;
                if (ahead) next.begin(g, u_next, by, tables + (turn ^= 1u) * kListed);
            }
            Cursor cursor;
            cursor.reset(table);
            int done = 0;
#pragma unroll 1
            do {
                if (done >= total && !whole) break;              // an empty table, and more of them
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
                if (ahead && next.room()) next.step(g, lane);
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
sparse_keys_kernel(const Geometry g, unsigned units, const T* q, const T* k, const T* v, const T* dout, T* dk, T* dv, const Prepared by)
{
    using K = KeysPlan<T, D>;
    using P = BackwardPipe<T, D>;
    using L = Layout<T, D>;
    constexpr int N = P::N, NT = N / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = uniform((int)threadIdx.x / 32), lane = threadIdx.x % 32;
    constexpr float scale = root<D>();

    // It takes nothing from the queries' kernel, but only a wait of its own makes visible to it what was written before that one.
    grid_dependency_wait();
    if (warp == kThreads / 32) {
        send_seers<T, D>(g, units, smem, q, k, v, dout, by);
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
cudaError_t launch_backward(const Geometry& g, long long B, const BackwardMaps& m, const Prepared& to, int sms, cudaStream_t stream) {
    constexpr size_t smem_q = BackwardPipe<T, D>::kSmem, smem_k = KeysPlan<T, D>::kSmem;
    int ctas = 0, ctas_k = 0;
    cudaError_t e = resident<sparse_queries_kernel<T, D>, smem_q>(sms, &ctas);
    if (e == cudaSuccess) e = resident<sparse_keys_kernel<T, D>, smem_k>(sms, &ctas_k);
    if (e != cudaSuccess) return e;
    const unsigned units = (unsigned)(B * g.blocks * g.tiles * g.heads), grid = units < (unsigned)ctas ? units : (unsigned)ctas;
    const long long n = B * g.H * g.W * g.heads;
    auto in = [](const void* p) { return static_cast<const T*>(p); };
    auto map = [](void* p) { return static_cast<T*>(p); };
    constexpr long long rows = 256 / (D * sizeof(T) / 16) * 4;      // of a block
    const unsigned lists = (unsigned)(B * g.heads);
    e = launch_chained(sparse_rows_kernel<T, D>, dim3((unsigned)(lists + (n + rows - 1) / rows)), 256, kInvertWarps * g.blocks * sizeof(int), stream, g, lists, n, m.idx,
                       in(m.out), in(m.dout), m.lse, to);
    if (e != cudaSuccess) return e;
    e = launch_chained(sparse_queries_kernel<T, D>, dim3(grid), kBlock, smem_q, stream, g, units, in(m.q), in(m.k),
                       in(m.v), m.idx, in(m.dout), static_cast<const float2*>(to.stats), map(m.dq));
    if (e != cudaSuccess) return e;
    return launch_chained(sparse_keys_kernel<T, D>, dim3(units < (unsigned)ctas_k ? units : (unsigned)ctas_k), kBlock, smem_k, stream, g, units, in(m.q), in(m.k),
                          in(m.v), in(m.dout), map(m.dk), map(m.dv), to);
}

}  // namespace sparse

cudaError_t launch_sparse_backward(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const sparse::BackwardMaps& m,
                                   void* workspace, int sms, cudaStream_t stream) {
    using namespace sparse;
    g.complete();
    Prepared to;
    to.stats = static_cast<float2*>(workspace);
    to.taken = reinterpret_cast<unsigned*>(to.stats + B * g.H * g.W * g.heads);
    to.starts = reinterpret_cast<int*>(to.taken) + 1;
    to.seers = to.starts + B * g.heads * (g.blocks + 1);
    if (dtype == SLIDE_ATTN_BF16) {
        if (head_dim == 16) return launch_backward<__nv_bfloat16, 16>(g, B, m, to, sms, stream);
        if (head_dim == 32) return launch_backward<__nv_bfloat16, 32>(g, B, m, to, sms, stream);
        return launch_backward<__nv_bfloat16, 64>(g, B, m, to, sms, stream);
    }
    if (head_dim == 16) return launch_backward<float, 16>(g, B, m, to, sms, stream);
    if (head_dim == 32) return launch_backward<float, 32>(g, B, m, to, sms, stream);
    return launch_backward<float, 64>(g, B, m, to, sms, stream);
}

}  // namespace slide_attn
