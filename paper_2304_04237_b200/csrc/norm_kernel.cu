// Group norm with an activation over channels-last maps [B][P pixels][C], forward and backward.
//
//   m, s2 = mean and variance of an image's group (P pixels x C/groups channels);  rstd = 1 / sqrt(s2 + eps)
//   u = (x - m) rstd,  z = gamma_c u + beta_c,  y = act(z)
//   dz = dy act'(z),  du = gamma_c dz,  dx = rstd (du - mean(du) - u mean(du u)),  dgamma_c = sum dz u,  dbeta_c = sum dz
//
// Bound by memory: x in and y out; x, dy in and dx out.  Two passes that stream over the map: sums of chunks of pixels, then the result, whose
// inputs the second pass finds in L2 (126 MB) as long as they fit.  The chunks are joined by every CTA of the second pass or, where there are many
// groups, by a small launch between the passes.  A thread keeps to one 16-byte column of the pixels, of which a CTA takes whole rows.  Images that
// one CTA can hold in its registers take one launch.
// 64 x 56 x 56 x 96, bf16, 32 groups, forward and backward in turn: 63 us, with SiLU 77, with GELU 93, of 29.5 for the 193 MB that they cannot do without.  Each
// pass reads its maps again, and the activation's special functions and roundings share the issue slots.
// (One pass for all, with an image's pixels kept in the shared memory of a cluster of CTAs that exchange their sums, read every map once,
// but its barriers and low occupancy made 64 x 56 x 56 x 96, bf16, GELU, forward and backward, take 114 us.)
// Sums are fp32 (the weights' over many chunks fp64), in an order that only the shape decides.
#include <atomic>

#include "operators.cuh"
#include "packed.cuh"

namespace slide_attn {

namespace {

constexpr int kTogether = 4;           // 16-byte pieces that a thread works on together (backward: half of them of each map)
constexpr int kForwardCtas = 4, kBackwardCtas = 3;     // of 256 threads on an SM, as registers allow
constexpr int kPair = kTogether / 2;
constexpr int kOnce = 8;               // rounds of an image that one CTA keeps
constexpr long long kSms = 148;        // that chunks are made for: B200's, whatever device is current, so that the workspace and the order of the sums depend on
                                       // the shape alone

struct NormShape {
    int P, C, groups, per_group;       // per_group: channels of a group
    int columns, rows, threads;        // 16-byte columns of a pixel; pixels that a CTA takes at a time (a round)
    int rounds, chunks;                // of a CTA; CTAs of an image
    bool once;                         // forward: a CTA keeps its whole image in registers (kOnce rounds at most), one launch.  Not the same as one
};                                     // chunk: where there are many images, each is one chunk however large it is

struct NormArgs {
    const void* x;
    const float* gamma;
    const float* beta;
    const void* dy;
    void* y;              // forward: y, backward: dx
    float* mean;          // [B][groups], written by the forward and read by the backward
    float* rstd;
    float2* partial;      // [B][groups][chunks]: forward mean and sum of squares about it, backward sums of du and of du u
    float2* joined;       // backward: [B][groups], what a launch between the passes joined; null: the second pass does it
    bool join;            // forward: the second pass joins the chunks
    float* channels;      // backward: [B][chunks][2][C], sums of dz and of dz u; or null
    float eps;
    float* dgamma;        // backward, where there is `channels`: what the second pass's first `weight_ctas` CTAs add up, of `all_chunks` chunks
    float* dbeta;
    unsigned weight_ctas;
    long long all_chunks;
};

// Sixteen bytes of channels as pairs of fp32 values.
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int pairs = 2;
    static __device__ __forceinline__ void get(const uint4& r, pair (&v)[2]) {
        v[0] = make_pair(__uint_as_float(r.x), __uint_as_float(r.y));
        v[1] = make_pair(__uint_as_float(r.z), __uint_as_float(r.w));
    }
    static __device__ __forceinline__ uint4 put(const pair (&v)[2]) {
        float a, b, c, d;
        split_pair(v[0], a, b);
        split_pair(v[1], c, d);
        return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int pairs = 4;
    static __device__ __forceinline__ void get(const uint4& r, pair (&v)[4]) {
        v[0] = make_pair(bf16_lo(r.x), bf16_hi(r.x));
        v[1] = make_pair(bf16_lo(r.y), bf16_hi(r.y));
        v[2] = make_pair(bf16_lo(r.z), bf16_hi(r.z));
        v[3] = make_pair(bf16_lo(r.w), bf16_hi(r.w));
    }
    static __device__ __forceinline__ uint32_t word(pair v) {
        float a, b;
        split_pair(v, a, b);
        return pack_bf16(a, b);
    }
    static __device__ __forceinline__ uint4 put(const pair (&v)[4]) { return make_uint4(word(v[0]), word(v[1]), word(v[2]), word(v[3])); }
};

__device__ __forceinline__ pair exp2_2(pair x) {
    float a, b;
    split_pair(x, a, b);
    return make_pair(fast_exp2(a), fast_exp2(b));
}
__device__ __forceinline__ pair rcp_2(pair x) {
    float a, b;
    split_pair(x, a, b);
    return make_pair(rcp_approx(a), rcp_approx(b));
}

// The normal distribution's integral up to -|z| and the exponential exp(-z^2 / 2) that is in it: with t = 1 / (1 + p |z|) it is that times t q(t), q a polynomial
// fitted up to |z| = 13.5, where the exponential is below fp32's normal numbers.  fp32: degree 7, of the least relative error, 1.3e-7.  bf16: degree 5,
// off by 1.1e-7 or by 1.1e-4 of itself, whichever is less, a 35th of a rounding to bf16 (with fp32's polynomial 64 x 56 x 56 x 96, forward and backward,
// takes 97.2 us instead of 93.8).  The arithmetic adds five or six roundings, and the exponential's argument some z^2 of them, as z's own does.  a: |z|, or a
// large number in an infinity's place, times which nothing is still nothing.
template <typename T> __device__ __forceinline__ pair normal_tail(pair z, pair& a, pair& e) {
    constexpr bool kWide = sizeof(T) == 4;
    constexpr int kTerms = kWide ? 8 : 6;
    constexpr float kFit[8] = {kWide ? 0.119626395f : 0.165674686f, kWide ? 0.120798312f : 0.179397747f, kWide ? 0.0996377915f : 0.0673380196f,
                               kWide ? 0.129468247f : 0.266205519f, kWide ? -0.0553920753f : -0.23595579f, kWide ? 0.208204731f : 0.0573398992f,
                               -0.158274934f, 0.0359314866f};
    float z0, z1;
    split_pair(z, z0, z1);
    a = make_pair(fminf(fabsf(z0), 1e30f), fminf(fabsf(z1), 1e30f));
    const pair t = rcp_2(fma2(a, both(kWide ? 0.3f : 0.4175f), both(1.0f)));
    pair q = both(kFit[kTerms - 1]);
#pragma unroll
    for (int i = kTerms - 2; i >= 0; --i) q = fma2(q, t, both(kFit[i]));
    e = exp2_2(mul2(mul2(z, both(-0.72134752f)), z));
    return mul2(mul2(q, t), e);
}

template <typename T, int Act> __device__ __forceinline__ pair act_value(pair z) {
    if constexpr (Act == SLIDE_ATTN_ACT_SILU) {
        return mul2(z, rcp_2(add2(exp2_2(mul2(z, both(-1.44269504f))), both(1.0f))));
    } else if constexpr (Act == SLIDE_ATTN_ACT_GELU) {
        // z times the integral up to z, which for z > 0 is 1 less the tail: max(z, 0) - |z| tail.  Nothing of the tail is lost for z < 0.
        pair a, e;
        const pair tail = normal_tail<T>(z, a, e);
        float z0, z1;
        split_pair(z, z0, z1);
        return fma2(mul2(a, both(-1.0f)), tail, make_pair(fmaxf(z0, 0.0f), fmaxf(z1, 0.0f)));
    } else {
        return z;
    }
}
template <typename T, int Act> __device__ __forceinline__ pair act_slope(pair z) {
    if constexpr (Act == SLIDE_ATTN_ACT_SILU) {
        const pair g = rcp_2(add2(exp2_2(mul2(z, both(-1.44269504f))), both(1.0f)));
        return mul2(g, fma2(z, fma2(g, both(-1.0f), both(1.0f)), both(1.0f)));    // g (1 + z (1 - g))
    } else if constexpr (Act == SLIDE_ATTN_ACT_GELU) {
        // The integral up to z plus z times the density: for z < 0 tail - |z| density, otherwise 1 less that.
        pair a, e;
        const pair tail = normal_tail<T>(z, a, e), below = fma2(mul2(a, both(-0.39894228f)), e, tail), above = fma2(below, both(-1.0f), both(1.0f));
        float z0, z1, b0, b1, c0, c1;
        split_pair(z, z0, z1);
        split_pair(below, b0, b1);
        split_pair(above, c0, c1);
        return make_pair(z0 < 0.0f ? b0 : c0, z1 < 0.0f ? b1 : c1);
    } else {
        return both(1.0f);
    }
}

// The groups of a column's channels.
template <int V> __device__ __forceinline__ void find_groups(int per_group, int column, int (&group)[V]) {
    int g = column * V / per_group, left = (g + 1) * per_group - column * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        group[e] = g;
        if (--left == 0) { ++g; left = per_group; }
    }
}
// V channels of gamma or beta, or a constant.
template <int V> __device__ __forceinline__ void get_weights(const float* w, int c, float otherwise, pair (&v)[V / 2]) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
        const float4 x = w ? *reinterpret_cast<const float4*>(w + c + e) : make_float4(otherwise, otherwise, otherwise, otherwise);
        v[e / 2] = make_pair(x.x, x.y);
        v[e / 2 + 1] = make_pair(x.z, x.w);
    }
}

// out[i] = sum over rows r < `rows` and columns c < `unit` of in[r][i unit + c], i < n, by `lanes` neighbouring threads each (a power of two up
// to 32), who share the rows or, of a single row, the columns.
__device__ __forceinline__ int lanes_for(int n) {
    int lanes = 32;
    while (lanes > 1 && n * lanes > (int)blockDim.x) lanes /= 2;
    return lanes;
}
__device__ __forceinline__ void sum_cells(const float* in, int rows, int width, int unit, int n, int lanes, float* out) {
    const int lane = threadIdx.x & (lanes - 1), at_once = (int)blockDim.x / lanes;
    for (int first = 0; first < n; first += at_once) {
        const int i = first + (int)threadIdx.x / lanes;
        float s = 0.0f;
        if (i < n) {
            const float* cell = in + i * unit;
            if (rows > 1) {
                if (unit == 1) {
#pragma unroll 4
                    for (int r = lane; r < rows; r += lanes) s += cell[r * width];
                } else {
#pragma unroll 2
                    for (int r = lane; r < rows; r += lanes)
                        for (int c = 0; c < unit; ++c) s += cell[r * width + c];
                }
            } else {
                for (int c = lane; c < unit; c += lanes) s += cell[c];
            }
        }
        for (int o = lanes / 2; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (i < n && lane == 0) out[i] = s;
    }
    __syncthreads();
}
template <int V> __device__ __forceinline__ void leave(float* red, const pair (&v)[V / 2]) {
#pragma unroll
    for (int e = 0; e < V / 4; ++e) {
        float4 x;
        split_pair(v[2 * e], x.x, x.y);
        split_pair(v[2 * e + 1], x.z, x.w);
        reinterpret_cast<float4*>(red)[threadIdx.x * (V / 4) + e] = x;               // [row][channel of the slab]
    }
}

// A thread's part of a chunk.
struct Place {
    int column;
    int mine;                          // its rounds
    int pixels;                        // the chunk's
    unsigned image;
    int chunk;
    size_t start, step;                // bytes to its first piece and from one to the next
    bool active;
};
__device__ __forceinline__ int chunk_pixels(const NormShape& s, int chunk) { return min(s.rows * s.rounds, s.P - chunk * s.rows * s.rounds); }
template <typename T> __device__ __forceinline__ Place find_place(const NormShape& s, unsigned cta = blockIdx.x) {
    Place p;
    p.image = cta / (unsigned)s.chunks;
    p.chunk = (int)(cta - p.image * (unsigned)s.chunks);
    const int row = (int)threadIdx.x / s.columns;
    p.column = (int)threadIdx.x - row * s.columns;
    p.active = row < s.rows;
    p.pixels = chunk_pixels(s, p.chunk);
    p.mine = p.active ? (p.pixels - row + s.rows - 1) / s.rows : 0;
    const size_t row_bytes = (size_t)s.C * sizeof(T);
    p.start = ((size_t)p.image * s.P + (size_t)p.chunk * (s.rows * s.rounds) + row) * row_bytes + (size_t)p.column * 16;
    p.step = s.rows * row_bytes;
    return p;
}

// A thread's pieces of one or two maps on their way through shared memory, a batch of `Batch` rounds at a time, kRing - 1 batches ahead of the
// arithmetic.  A thread reads only what it copied itself, so no barrier is needed; a batch's room is filled again one batch after it was read.
template <int Threads, int Maps, int Batch> struct Stream {
    static constexpr int kRing = 3, kPieces = Maps * Batch;
    static constexpr size_t kSmem = (size_t)Threads * kRing * kPieces * 16;
    unsigned char* ring;
    const unsigned char *x, *g;
    size_t step;
    int left, to, from;
    __device__ __forceinline__ Stream(unsigned char* smem, const unsigned char* src_x, const unsigned char* src_g, const Place& at)
        : ring(smem + threadIdx.x * 16), x(src_x), g(src_g), step(at.step), left(at.mine), to(0), from(0) {
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) send();
    }
    __device__ __forceinline__ unsigned char* piece(int batch, int i) const { return ring + (batch * kPieces + i) * (Threads * 16); }
    __device__ __forceinline__ void send() {
#pragma unroll
        for (int i = 0; i < Batch; ++i)
            if (i < left) {
                copy16(smem_u32(piece(to, i * Maps)), x);
                x += step;
                if constexpr (Maps > 1) {
                    copy16(smem_u32(piece(to, i * Maps + 1)), g);
                    g += step;
                }
            }
        left -= Batch;
        to = to == kRing - 1 ? 0 : to + 1;
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // The next batch has arrived: its pieces, those of a round side by side.
    __device__ __forceinline__ void next(uint4 (&raw)[kPieces]) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
#pragma unroll
        for (int i = 0; i < kPieces; ++i) raw[i] = *reinterpret_cast<const uint4*>(piece(from, i));
        from = from == kRing - 1 ? 0 : from + 1;
        send();
    }
    static __device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    }
};

// An image's group's moments from its chunks', by a warp; deviations from the first chunk's mean, so that nothing large cancels.  (mean, rstd)
__device__ __forceinline__ float2 join_moments(const NormShape& s, const float2* chunks, float eps, int lane) {
    const float per = (float)s.per_group, n = (float)s.P * per;
    const float m0 = chunks[0].x;
    float shift = 0.0f;
    for (int c = lane; c < s.chunks; c += 32) shift += (float)chunk_pixels(s, c) * per * (chunks[c].x - m0);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) shift += __shfl_xor_sync(0xffffffffu, shift, o);
    const float m = m0 + shift / n;
    float m2 = 0.0f;
    for (int c = lane; c < s.chunks; c += 32) {
        const float2 v = chunks[c];
        const float d = v.x - m;
        m2 += fmaf((float)chunk_pixels(s, c) * per * d, d, v.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
    return make_float2(m, 1.0f / sqrtf(m2 / n + eps));
}
// The same of the backward's sums: (quad, shift), of which dx = dz (rstd gamma) + (c quad + shift) with c = x - mean: quad = -rstd^2 mean(du u),
// shift = -rstd mean(du).
__device__ __forceinline__ float2 join_slopes(const NormShape& s, const float2* chunks, float rstd, int lane) {
    float2 t = make_float2(0.0f, 0.0f);
    for (int c = lane; c < s.chunks; c += 32) { t.x += chunks[c].x; t.y += chunks[c].y; }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
        t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
    }
    const float inv = 1.0f / ((float)s.P * (float)s.per_group);
    return make_float2(-rstd * rstd * (t.y * inv), -rstd * (t.x * inv));
}

// First pass, forward: of a chunk, each group's mean and sum of squares about that mean, which loses nothing however far it is from zero: batch by
// batch of a thread's pixels (mean, then squares about it), joined by what the means differ, then over the threads in the same way.
template <typename T>
struct Moments {
    static constexpr int Q = Vec<T>::pairs;
    pair mean[Q] = {}, square[Q] = {};
    float n = 0.0f;
    template <int N> __device__ __forceinline__ void add(const uint4 (&raw)[N], int count) {
        pair sum[Q] = {};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < count) {
                pair v[Q];
                Vec<T>::get(raw[i], v);
#pragma unroll
                for (int e = 0; e < Q; ++e) sum[e] = add2(sum[e], v[e]);
            }
        const float k = (float)count, all = n + k;
        const pair inv = both(-1.0f / k), part = both(k / all), weight = both(n * k / all);
        pair own[Q], own_square[Q] = {};                            // less the batch's mean
#pragma unroll
        for (int e = 0; e < Q; ++e) own[e] = mul2(sum[e], inv);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < count) {
                pair v[Q];
                Vec<T>::get(raw[i], v);
#pragma unroll
                for (int e = 0; e < Q; ++e) {
                    const pair d = add2(v[e], own[e]);
                    own_square[e] = fma2(d, d, own_square[e]);
                }
            }
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            const pair d = fma2(own[e], both(-1.0f), mul2(mean[e], both(-1.0f)));       // the batch's mean less the one so far
            mean[e] = fma2(d, part, mean[e]);
            square[e] = fma2(mul2(d, d), weight, add2(square[e], own_square[e]));
        }
        n = all;
    }
};
// Each group's mean and sum of squares from the threads'; all threads call it.  red: [row][channel]
template <typename T>
__device__ __forceinline__ void join_threads(const NormShape& s, const Place& at, const Moments<T>& m, const int (&group)[2 * Vec<T>::pairs], float* red,
                                             float* means, float* squares) {
    constexpr int Q = Vec<T>::pairs, V = 2 * Q;
    const int lanes = lanes_for(s.groups);
    pair v[Q];
#pragma unroll
    for (int e = 0; e < Q; ++e) v[e] = mul2(m.mean[e], both(m.n));
    if (at.active) leave<V>(red, v);
    __syncthreads();
    sum_cells(red, s.rows, s.C, s.per_group, s.groups, lanes, means);
    const float inv = 1.0f / ((float)at.pixels * (float)s.per_group);
#pragma unroll
    for (int e = 0; e < Q; ++e) {
        const pair d = add2(m.mean[e], make_pair(-means[group[2 * e]] * inv, -means[group[2 * e + 1]] * inv));
        v[e] = fma2(mul2(d, d), both(m.n), m.square[e]);
    }
    if (at.active) leave<V>(red, v);
    __syncthreads();
    for (int g = threadIdx.x; g < s.groups; g += blockDim.x) means[g] *= inv;
    sum_cells(red, s.rows, s.C, s.per_group, s.groups, lanes, squares);
}

template <int Threads, typename T>
__global__ void __launch_bounds__(Threads, kForwardCtas * 256 / Threads) norm_sums_kernel(const NormArgs a, const NormShape s)
{
    constexpr int V = 2 * Vec<T>::pairs;
    extern __shared__ __align__(16) unsigned char smem[];
    using Maps = Stream<Threads, 1, kTogether>;
    float* red = reinterpret_cast<float*>(smem + Maps::kSmem);
    float* means = red + s.threads * V;
    float* squares = means + s.groups;
    const Place at = find_place<T>(s);
    grid_dependency_wait();
    Maps maps(smem, static_cast<const unsigned char*>(a.x) + at.start, nullptr, at);
    Moments<T> m;
#pragma unroll 1
    for (int done = 0; done < at.mine; done += kTogether) {
        uint4 raw[kTogether];
        maps.next(raw);
        m.add(raw, min(at.mine - done, kTogether));
    }
    int group[V];
    find_groups<V>(s.per_group, at.column, group);
    join_threads<T>(s, at, m, group, red, means, squares);
    for (int g = threadIdx.x; g < s.groups; g += blockDim.x)
        a.partial[((size_t)at.image * s.groups + g) * s.chunks + at.chunk] = make_float2(means[g], squares[g]);
}

// Between the passes: a warp an image and group.
template <bool Backward>
__global__ void __launch_bounds__(256) norm_join_kernel(const NormArgs a, const NormShape s, long long n)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const long long i = (long long)blockIdx.x * 8 + threadIdx.x / 32;
    if (i >= n) return;
    const int lane = threadIdx.x % 32;
    if constexpr (Backward) {
        const float2 r = join_slopes(s, a.partial + i * s.chunks, a.rstd[i], lane);
        if (lane == 0) a.joined[i] = r;
    } else {
        const float2 r = join_moments(s, a.partial + i * s.chunks, a.eps, lane);
        if (lane == 0) { a.mean[i] = r.x; a.rstd[i] = r.y; }
    }
}

template <typename T, int Act>
__device__ __forceinline__ uint4 normalised(const uint4& raw, const pair (&mean)[Vec<T>::pairs], const pair (&scale)[Vec<T>::pairs],
                                            const pair (&beta)[Vec<T>::pairs]) {
    pair v[Vec<T>::pairs];
    Vec<T>::get(raw, v);
#pragma unroll
    for (int e = 0; e < Vec<T>::pairs; ++e) v[e] = act_value<T, Act>(fma2(add2(v[e], mean[e]), scale[e], beta[e]));
    return Vec<T>::put(v);
}

template <int Threads, typename T, int Act>
__global__ void __launch_bounds__(Threads, kForwardCtas * 256 / Threads) norm_forward_kernel(const NormArgs a, const NormShape s)
{
    constexpr int Q = Vec<T>::pairs, V = 2 * Q;
    extern __shared__ __align__(16) unsigned char smem[];
    using Maps = Stream<Threads, 1, kTogether>;
    const Place at = find_place<T>(s);
    unsigned char* dst = static_cast<unsigned char*>(a.y) + at.start;
    float2* stats = reinterpret_cast<float2*>(smem + Maps::kSmem);        // mean and rstd
    grid_dependency_wait();
    Maps maps(smem, static_cast<const unsigned char*>(a.x) + at.start, nullptr, at);
    const size_t first = (size_t)at.image * s.groups;
    if (a.join) {
        const int lane = threadIdx.x % 32;
        for (int g = threadIdx.x / 32; g < s.groups; g += Threads / 32) {
            const float2 r = join_moments(s, a.partial + (first + g) * s.chunks, a.eps, lane);
            if (lane) continue;
            stats[g] = r;
            if (at.chunk == 0) { a.mean[first + g] = r.x; a.rstd[first + g] = r.y; }
        }
    } else {
        for (int g = threadIdx.x; g < s.groups; g += Threads) stats[g] = make_float2(a.mean[first + g], a.rstd[first + g]);
    }
    __syncthreads();
    if (!at.active) return;
    pair scale[Q], beta[Q], mean[Q];                                // mean: less it
    get_weights<V>(a.gamma, at.column * V, 1.0f, scale);
    get_weights<V>(a.beta, at.column * V, 0.0f, beta);
    {
        int group[V];
        find_groups<V>(s.per_group, at.column, group);
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            const float2 u = stats[group[2 * e]], v = stats[group[2 * e + 1]];
            mean[e] = make_pair(-u.x, -v.x);
            scale[e] = mul2(scale[e], make_pair(u.y, v.y));
        }
    }
#pragma unroll 1
    for (int done = 0; done < at.mine; done += kTogether) {
        uint4 raw[kTogether];
        maps.next(raw);
#pragma unroll
        for (int i = 0; i < kTogether; ++i)
            if (done + i < at.mine) *reinterpret_cast<uint4*>(dst + i * at.step) = normalised<T, Act>(raw[i], mean, scale, beta);
        dst += kTogether * at.step;
    }
}

// An image of kOnce rounds at most (NormShape::once): all of the forward, from registers.
template <int Threads, typename T, int Act>
__global__ void __launch_bounds__(Threads, 2 * 256 / Threads) norm_forward_once_kernel(const NormArgs a, const NormShape s)
{
    constexpr int Q = Vec<T>::pairs, V = 2 * Q;
    extern __shared__ __align__(16) unsigned char smem[];
    float* red = reinterpret_cast<float*>(smem);
    float* means = red + s.threads * V;
    float* squares = means + s.groups;
    const Place at = find_place<T>(s);
    const unsigned char* src = static_cast<const unsigned char*>(a.x) + at.start;
    unsigned char* dst = static_cast<unsigned char*>(a.y) + at.start;
    grid_dependency_wait();
    uint4 raw[kOnce];
#pragma unroll
    for (int i = 0; i < kOnce; ++i)
        if (i < at.mine) raw[i] = *reinterpret_cast<const uint4*>(src + i * at.step);
    int group[V];
    find_groups<V>(s.per_group, at.column, group);
    pair scale[Q], beta[Q], mean[Q];
    get_weights<V>(a.gamma, at.column * V, 1.0f, scale);
    get_weights<V>(a.beta, at.column * V, 0.0f, beta);
    Moments<T> m;
    if (at.mine > 0) m.add(raw, at.mine);
    join_threads<T>(s, at, m, group, red, means, squares);
    const float inv = 1.0f / ((float)s.P * (float)s.per_group);
    for (int g = threadIdx.x; g < s.groups; g += blockDim.x) {
        const float rstd = 1.0f / sqrtf(squares[g] * inv + a.eps);
        const size_t o = (size_t)at.image * s.groups + g;
        a.mean[o] = means[g];
        a.rstd[o] = rstd;
        squares[g] = rstd;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < Q; ++e) {
        mean[e] = make_pair(-means[group[2 * e]], -means[group[2 * e + 1]]);
        scale[e] = mul2(scale[e], make_pair(squares[group[2 * e]], squares[group[2 * e + 1]]));
    }
#pragma unroll
    for (int i = 0; i < kOnce; ++i)
        if (i < at.mine) *reinterpret_cast<uint4*>(dst + i * at.step) = normalised<T, Act>(raw[i], mean, scale, beta);
}

// First pass, backward: of a chunk, each channel's sums of dz and dz u, and each group's of du and du u.
template <int Threads, typename T, int Act>
__global__ void __launch_bounds__(Threads, kBackwardCtas * 256 / Threads) norm_slopes_kernel(const NormArgs a, const NormShape s)
{
    constexpr int Q = Vec<T>::pairs, V = 2 * Q;
    extern __shared__ __align__(16) unsigned char smem[];
    using Maps = Stream<Threads, 2, kPair>;
    float* red = reinterpret_cast<float*>(smem + Maps::kSmem);      // [row][channel]; later two values a channel
    float* channel = red + max(s.threads * V, 2 * s.C);             // sums of dz, then of dz u
    float* local = channel + 2 * s.C;                               // the groups'
    const Place at = find_place<T>(s);
    grid_dependency_wait();
    Maps maps(smem, static_cast<const unsigned char*>(a.x) + at.start, static_cast<const unsigned char*>(a.dy) + at.start, at);
    pair mean[Q], scale[Q], beta[Q], s1[Q] = {}, s2[Q] = {};
    const float* means = a.mean + (size_t)at.image * s.groups;
    const float* rstds = a.rstd + (size_t)at.image * s.groups;
    {
        int group[V];
        find_groups<V>(s.per_group, at.column, group);
        get_weights<V>(a.gamma, at.column * V, 1.0f, scale);
        get_weights<V>(a.beta, at.column * V, 0.0f, beta);
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            mean[e] = make_pair(-means[group[2 * e]], -means[group[2 * e + 1]]);
            scale[e] = mul2(scale[e], make_pair(rstds[group[2 * e]], rstds[group[2 * e + 1]]));
        }
    }
#pragma unroll 1
    for (int done = 0; done < at.mine; done += kPair) {
        uint4 raw[2 * kPair];
        maps.next(raw);
#pragma unroll
        for (int i = 0; i < kPair; ++i)
            if (done + i < at.mine) {
                pair c[Q], dz[Q];
                Vec<T>::get(raw[2 * i], c);
                Vec<T>::get(raw[2 * i + 1], dz);
#pragma unroll
                for (int e = 0; e < Q; ++e) {
                    c[e] = add2(c[e], mean[e]);
                    if constexpr (Act != SLIDE_ATTN_ACT_NONE) dz[e] = mul2(dz[e], act_slope<T, Act>(fma2(c[e], scale[e], beta[e])));
                    s1[e] = add2(s1[e], dz[e]);
                    s2[e] = fma2(dz[e], c[e], s2[e]);
                }
            }
    }
    const int lanes = lanes_for(s.C);
    if (at.active) leave<V>(red, s1);
    __syncthreads();
    sum_cells(red, s.rows, s.C, 1, s.C, lanes, channel);
    if (at.active) leave<V>(red, s2);
    __syncthreads();
    sum_cells(red, s.rows, s.C, 1, s.C, lanes, channel + s.C);
    float* out = a.channels ? a.channels + ((size_t)at.image * s.chunks + at.chunk) * 2 * s.C : nullptr;
    for (int i = threadIdx.x; i < 2 * s.C; i += blockDim.x) {
        const int c = i < s.C ? i : i - s.C;
        const float v = i < s.C ? channel[i] : channel[i] * rstds[c / s.per_group];
        if (out) out[i] = v;
        red[i] = v * (a.gamma ? a.gamma[c] : 1.0f);
    }
    __syncthreads();
    sum_cells(red, 1, 0, s.per_group, 2 * s.groups, lanes_for(2 * s.groups), local);
    for (int g = threadIdx.x; g < s.groups; g += blockDim.x)
        a.partial[((size_t)at.image * s.groups + g) * s.chunks + at.chunk] = make_float2(local[g], local[s.groups + g]);
}

// dbeta and dgamma: the chunks' sums, added up in their order.  32 of the 2 C columns a CTA, a row a warp at a time.  There may be a hundred thousand
// chunks (images of a few pixels): 32 of a warp's at a time in fp32, those sums in fp64, so that the error does not grow with their number.
// part: [warp][32]
template <int Threads>
__device__ __forceinline__ void sum_weights(const NormArgs& a, int C, double (*part)[32]) {
    constexpr int kRowsAtOnce = Threads / 32, kRun = 32;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
    double sum = 0.0;
    if (c < 2 * C) {
        const float* from = a.channels + c;
        for (long long r0 = warp; r0 < a.all_chunks; r0 += kRun * kRowsAtOnce) {
            const long long end = min(a.all_chunks, r0 + kRun * kRowsAtOnce);
            float run = 0.0f;
#pragma unroll 8
            for (long long r = r0; r < end; r += kRowsAtOnce) run += from[(size_t)r * 2 * C];
            sum += run;
        }
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < 2 * C) {
#pragma unroll
        for (int i = 1; i < kRowsAtOnce; ++i) sum += part[i][lane];
        (c < C ? a.dbeta : a.dgamma)[c < C ? c : c - C] = (float)sum;
    }
}

// Second pass, backward.  Its first CTAs add up the weights' gradients beside it, which need nothing of it: 64 x 56 x 56 x 96, bf16, GELU, forward and backward
// 93.4 us, some 4 more with a launch of their own behind it.
template <int Threads, typename T, int Act>
__global__ void __launch_bounds__(Threads, kBackwardCtas * 256 / Threads) norm_backward_kernel(const NormArgs a, const NormShape s)
{
    constexpr int Q = Vec<T>::pairs, V = 2 * Q;
    extern __shared__ __align__(16) unsigned char smem[];
    using Maps = Stream<Threads, 2, kPair>;
    grid_dependency_wait();
    if (blockIdx.x < a.weight_ctas) {
        sum_weights<Threads>(a, s.C, reinterpret_cast<double (*)[32]>(smem));
        return;
    }
    const Place at = find_place<T>(s, blockIdx.x - a.weight_ctas);
    unsigned char* dst = static_cast<unsigned char*>(a.y) + at.start;
    Maps maps(smem, static_cast<const unsigned char*>(a.x) + at.start, static_cast<const unsigned char*>(a.dy) + at.start, at);
    float2* stats = reinterpret_cast<float2*>(smem + Maps::kSmem);        // quad and shift
    const size_t first = (size_t)at.image * s.groups;
    if (!a.joined) {
        const int lane = threadIdx.x % 32;
        for (int g = threadIdx.x / 32; g < s.groups; g += Threads / 32) {
            const float2 r = join_slopes(s, a.partial + (first + g) * s.chunks, a.rstd[first + g], lane);
            if (lane == 0) stats[g] = r;
        }
    } else {
        for (int g = threadIdx.x; g < s.groups; g += Threads) stats[g] = a.joined[first + g];
    }
    __syncthreads();
    if (!at.active) return;
    pair mean[Q], scale[Q], beta[Q], quad[Q], shift[Q];
    get_weights<V>(a.gamma, at.column * V, 1.0f, scale);
    get_weights<V>(a.beta, at.column * V, 0.0f, beta);
    {
        int group[V];
        find_groups<V>(s.per_group, at.column, group);
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            const int i = group[2 * e], j = group[2 * e + 1];
            mean[e] = make_pair(-a.mean[first + i], -a.mean[first + j]);
            scale[e] = mul2(scale[e], make_pair(a.rstd[first + i], a.rstd[first + j]));
            quad[e] = make_pair(stats[i].x, stats[j].x);
            shift[e] = make_pair(stats[i].y, stats[j].y);
        }
    }
#pragma unroll 1
    for (int done = 0; done < at.mine; done += kPair) {
        uint4 raw[2 * kPair];
        maps.next(raw);
#pragma unroll
        for (int i = 0; i < kPair; ++i)
            if (done + i < at.mine) {
                pair c[Q], dz[Q];
                Vec<T>::get(raw[2 * i], c);
                Vec<T>::get(raw[2 * i + 1], dz);
#pragma unroll
                for (int e = 0; e < Q; ++e) {
                    c[e] = add2(c[e], mean[e]);
                    if constexpr (Act != SLIDE_ATTN_ACT_NONE) dz[e] = mul2(dz[e], act_slope<T, Act>(fma2(c[e], scale[e], beta[e])));
                    dz[e] = fma2(dz[e], scale[e], fma2(c[e], quad[e], shift[e]));
                }
                *reinterpret_cast<uint4*>(dst + i * at.step) = Vec<T>::put(dz);
            }
        dst += kPair * at.step;
    }
}

unsigned weight_ctas_of(int C) { return (2 * (unsigned)C + 31) / 32; }

// False where a pixel has too many columns for a CTA, or the call too many CTAs for a grid.  `maps`: 1 forward, 2 backward.
bool make_shape(long long B, long long P, int C, int groups, int size, int maps, NormShape* out) {
    if (C > 512 * 16 / size) return false;            // more than 512 columns; C is anything so far, and products with it may overflow
    NormShape s = {};
    s.P = (int)P; s.C = C; s.groups = groups; s.per_group = C / groups;
    s.columns = C * size / 16;
    s.threads = s.columns > 256 ? 512 : 256;
    s.rows = s.threads / s.columns;
    if (maps == 1 && P <= (long long)(512 / s.columns) * kOnce) {
        // an image in one CTA's registers
        if (P > (long long)s.rows * kOnce) { s.threads = 512; s.rows = 512 / s.columns; }
        s.rounds = kOnce;
        s.once = true;
    } else {
        // What a thread does once (some hundred instructions) wants many rounds: as many CTAs as kSms SMs hold together, or the images' number.
        const long long all = (P + s.rows - 1) / s.rows, room = kSms * (maps == 1 ? kForwardCtas : kBackwardCtas) * 256 / s.threads;
        const long long each = room / B > 0 ? room / B : 1;
        long long rounds = (all + each - 1) / each;
        if (rounds < kTogether) rounds = kTogether;
        s.rounds = (int)rounds;
    }
    const long long chunks = (P + (long long)s.rows * s.rounds - 1) / ((long long)s.rows * s.rounds);
    if (B > (0x7fffffffLL - weight_ctas_of(C)) / chunks || B > 0x7fffffffLL / groups) return false;
    s.chunks = (int)chunks;
    *out = s;
    return true;
}

// More than 48 KB of shared memory has to be asked for, once on each device and for the most that any call takes (kMostSmem: the backward's first
// pass of 4096 channels in as many groups), so that threads of the host that launch at the same time ask for the same.
constexpr size_t kMostSmem = 192 * 1024;
template <auto Kernel, typename... Args>
cudaError_t launch_with(dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args) {
    static std::atomic<bool> asked[64];
    if (smem > 48 * 1024) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 64 || !asked[dev].load(std::memory_order_acquire)) {
            e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
            if (e != cudaSuccess) return e;
            if (dev < 64) asked[dev].store(true, std::memory_order_release);
        }
    }
    return launch_chained(Kernel, grid, threads, smem, stream, args...);
}

size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }
// Every CTA of the second pass joins the chunks of its image by itself where each of its warps has one group at most, which saves a launch: 128 x 128
// x 96, fp32, SiLU, 8 groups 11.9 us against 12.3, backward 12.9 against 14.6 (no launch gaps counted; launched one by one 14.4 against 16.1, 17.9
// against 19.9).  With 32 groups it would take 17.9 us against 11.1, 17.1 against 15.2.
bool joins_inline(const NormShape& s) { return s.groups <= s.threads / 32; }

// A workspace: partial, joined, channels.
struct NormRoom {
    size_t joined, channels, bytes;
    NormRoom(const NormShape& s, long long B, int maps) {
        joined = s.once ? 0 : align16((size_t)B * s.groups * s.chunks * sizeof(float2));
        channels = joined + (maps == 1 || joins_inline(s) ? 0 : align16((size_t)B * s.groups * sizeof(float2)));
        bytes = channels + (maps == 1 ? 0 : (size_t)B * s.chunks * 2 * s.C * sizeof(float));
    }
};

template <int Threads, typename T, int Act>
cudaError_t forward_as(const NormArgs& a, const NormShape& s, long long B, cudaStream_t stream) {
    const dim3 grid((unsigned)(B * s.chunks));
    constexpr size_t ring = Stream<Threads, 1, kTogether>::kSmem;
    const size_t smem = (size_t)(s.threads * 2 * Vec<T>::pairs + 2 * s.groups) * 4;
    if (s.once) return launch_with<norm_forward_once_kernel<Threads, T, Act>>(grid, Threads, smem, stream, a, s);
    cudaError_t e = launch_with<norm_sums_kernel<Threads, T>>(grid, Threads, ring + smem, stream, a, s);
    if (e == cudaSuccess && !a.join)
        e = launch_chained(norm_join_kernel<false>, dim3((unsigned)((B * s.groups + 7) / 8)), 256, 0, stream, a, s, B * s.groups);
    if (e != cudaSuccess) return e;
    return launch_with<norm_forward_kernel<Threads, T, Act>>(grid, Threads, ring + s.groups * sizeof(float2), stream, a, s);
}
template <typename T, int Act>
cudaError_t forward_with(const NormArgs& a, const NormShape& s, long long B, cudaStream_t stream) {
    return s.threads == 512 ? forward_as<512, T, Act>(a, s, B, stream) : forward_as<256, T, Act>(a, s, B, stream);
}
template <typename T>
cudaError_t forward_of(const NormArgs& a, const NormShape& s, long long B, int act, cudaStream_t stream) {
    switch (act) {
        case SLIDE_ATTN_ACT_SILU: return forward_with<T, SLIDE_ATTN_ACT_SILU>(a, s, B, stream);
        case SLIDE_ATTN_ACT_GELU: return forward_with<T, SLIDE_ATTN_ACT_GELU>(a, s, B, stream);
        default: return forward_with<T, SLIDE_ATTN_ACT_NONE>(a, s, B, stream);
    }
}

template <int Threads, typename T, int Act>
cudaError_t backward_as(const NormArgs& a, const NormShape& s, long long B, cudaStream_t stream) {
    const unsigned grid = (unsigned)(B * s.chunks);
    constexpr size_t ring = Stream<Threads, 2, kPair>::kSmem;
    const int red = s.threads * 2 * Vec<T>::pairs;
    const size_t smem = (size_t)((red > 2 * s.C ? red : 2 * s.C) + 2 * s.C + 2 * s.groups) * 4;
    cudaError_t e = launch_with<norm_slopes_kernel<Threads, T, Act>>(grid, Threads, ring + smem, stream, a, s);
    if (e == cudaSuccess && a.joined)
        e = launch_chained(norm_join_kernel<true>, dim3((unsigned)((B * s.groups + 7) / 8)), 256, 0, stream, a, s, B * s.groups);
    if (e != cudaSuccess) return e;
    return launch_with<norm_backward_kernel<Threads, T, Act>>(grid + a.weight_ctas, Threads, ring + s.groups * sizeof(float2), stream, a, s);
}
template <typename T, int Act>
cudaError_t backward_with(const NormArgs& a, const NormShape& s, long long B, cudaStream_t stream) {
    return s.threads == 512 ? backward_as<512, T, Act>(a, s, B, stream) : backward_as<256, T, Act>(a, s, B, stream);
}
template <typename T>
cudaError_t backward_of(const NormArgs& a, const NormShape& s, long long B, int act, cudaStream_t stream) {
    switch (act) {
        case SLIDE_ATTN_ACT_SILU: return backward_with<T, SLIDE_ATTN_ACT_SILU>(a, s, B, stream);
        case SLIDE_ATTN_ACT_GELU: return backward_with<T, SLIDE_ATTN_ACT_GELU>(a, s, B, stream);
        default: return backward_with<T, SLIDE_ATTN_ACT_NONE>(a, s, B, stream);
    }
}

}  // namespace

bool group_norm_workspace(long long B, long long P, int C, int groups, slide_attn_dtype dtype, int maps, size_t* bytes) {
    NormShape s;
    if (!make_shape(B, P, C, groups, dtype == SLIDE_ATTN_BF16 ? 2 : 4, maps, &s)) return false;
    *bytes = NormRoom(s, B, maps).bytes;
    return true;
}

cudaError_t launch_group_norm_forward(const void* x, const float* gamma, const float* beta, long long B, long long P, int C, int groups, float eps,
                                      slide_attn_activation act, slide_attn_dtype dtype, void* y, float* mean, float* rstd, void* workspace,
                                      cudaStream_t stream) {
    NormShape s;
    if (!make_shape(B, P, C, groups, dtype == SLIDE_ATTN_BF16 ? 2 : 4, 1, &s)) return cudaErrorInvalidValue;
    const NormArgs a = {x, gamma, beta, nullptr, y, mean, rstd, static_cast<float2*>(workspace), nullptr, joins_inline(s), nullptr, eps, nullptr, nullptr, 0, 0};
    return dtype == SLIDE_ATTN_BF16 ? forward_of<__nv_bfloat16>(a, s, B, act, stream) : forward_of<float>(a, s, B, act, stream);
}

cudaError_t launch_group_norm_backward(const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd, const void* dy,
                                       long long B, long long P, int C, int groups, slide_attn_activation act, slide_attn_dtype dtype, void* dx,
                                       float* dgamma, float* dbeta, void* workspace, cudaStream_t stream) {
    NormShape s;
    if (!make_shape(B, P, C, groups, dtype == SLIDE_ATTN_BF16 ? 2 : 4, 2, &s)) return cudaErrorInvalidValue;
    const NormRoom room(s, B, 2);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    float* channels = dgamma ? reinterpret_cast<float*>(ws + room.channels) : nullptr;
    const NormArgs a = {x, gamma, beta, dy, dx, const_cast<float*>(mean), const_cast<float*>(rstd), reinterpret_cast<float2*>(ws),
                        joins_inline(s) ? nullptr : reinterpret_cast<float2*>(ws + room.joined), false, channels, 0.0f, dgamma, dbeta,
                        channels ? weight_ctas_of(C) : 0u, B * s.chunks};
    return dtype == SLIDE_ATTN_BF16 ? backward_of<__nv_bfloat16>(a, s, B, act, stream) : backward_of<float>(a, s, B, act, stream);
}

}  // namespace slide_attn
