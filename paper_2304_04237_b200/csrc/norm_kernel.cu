// Group norm with an activation over channels-last maps [B][P pixels][C], forward and backward.
//
//   m, s2 = mean and variance of an image's group (P pixels x C/groups channels);  rstd = 1 / sqrt(s2 + eps)
//   u = (x - m) rstd,  z = gamma_c u + beta_c,  y = act(z)
//   dz = dy act'(z),  du = gamma_c dz,  dx = rstd (du - mean(du) - u mean(du u)),  dgamma_c = sum dz u,  dbeta_c = sum dz
//
// Bound by memory: x in and y out; x, dy in and dx out.  So each map is read from device memory once: a cluster of up to 16 CTAs
// holds the pixels of one image's slab (whole groups, a multiple of 16 bytes wide) in its shared memory, exchanges the
// sums through distributed shared memory and writes the result from what it holds.  Pixels that do not fit are read a
// second time.  A thread keeps to one 16-byte column of the slab and reads from shared memory only what it copied there itself, so
// the copies need no barrier.  All sums are fp32, in an order that only the shape decides.
#include <cooperative_groups.h>

#include "operators.cuh"
#include "packed.cuh"

namespace cg = cooperative_groups;

namespace slide_attn {

namespace {

constexpr int kMaxCluster = 16;
constexpr int kMaxSmem = 227 * 1024;
constexpr int kMostSms = 160;

// How a call is cut up: slabs of `width` channels, clusters of `cluster` CTAs, of whose pixels `cached` rounds of `rows` stay in shared memory.
struct NormPlan {
    int P, C, groups, per_group;       // per_group: channels of a group
    int width, slabs, cluster, log_cluster;
    int columns, rows, threads;        // 16-byte columns of a slab; pixel rows that a CTA takes at a time
    int cached;
    size_t smem;
    long long blocks;
};

struct NormArgs {
    const void* x;
    const float* gamma;
    const float* beta;
    const void* dy;
    void* y;              // forward: y, backward: dx
    float* mean;          // [B][groups], written by the forward and read by the backward
    float* rstd;
    float* sums;          // backward: [B][C] of dz and, behind them, of dz u
    float eps;
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

// The normal distribution's integral up to z and, from the same exponential, its density.  erfc by M. Abramowitz, I. Stegun, Handbook of
// Mathematical Functions, 7.1.26 (error below 1.5e-7): erfc(x) = t (a1 + t (a2 + ...)) exp(-x^2), t = 1 / (1 + p x), x = |z| / sqrt 2.  An
// infinity gives 0 or 1 and a NaN a NaN.
__device__ __forceinline__ void normal_2(pair z, pair& cdf, pair& density) {
    float z0, z1;
    split_pair(z, z0, z1);
    const pair a = make_pair(fabsf(z0), fabsf(z1));
    const pair t = rcp_2(fma2(a, both(0.3275911f * 0.70710678f), both(1.0f)));
    pair p = fma2(t, both(0.5f * 1.061405429f), both(-0.5f * 1.453152027f));      // half of the polynomial
    p = fma2(p, t, both(0.5f * 1.421413741f));
    p = fma2(p, t, both(-0.5f * 0.284496736f));
    p = fma2(p, t, both(0.5f * 0.254829592f));
    const pair e = exp2_2(mul2(mul2(z, both(-0.72134752f)), z));                 // exp(-z^2 / 2)
    const pair d = fma2(mul2(p, t), mul2(e, both(-1.0f)), both(0.5f));           // 1/2 - integral up to -|z|
    float d0, d1;
    split_pair(d, d0, d1);
    cdf = add2(make_pair(copysignf(d0, z0), copysignf(d1, z1)), both(0.5f));
    density = mul2(e, both(0.39894228f));
}

template <int Act> __device__ __forceinline__ pair act_value(pair z) {
    if constexpr (Act == SLIDE_ATTN_ACT_SILU) {
        return mul2(z, rcp_2(add2(exp2_2(mul2(z, both(-1.44269504f))), both(1.0f))));
    } else if constexpr (Act == SLIDE_ATTN_ACT_GELU) {
        pair cdf, density;
        normal_2(z, cdf, density);
        return mul2(z, cdf);
    } else {
        return z;
    }
}
template <int Act> __device__ __forceinline__ pair act_slope(pair z) {
    if constexpr (Act == SLIDE_ATTN_ACT_SILU) {
        const pair g = rcp_2(add2(exp2_2(mul2(z, both(-1.44269504f))), both(1.0f)));
        return mul2(g, fma2(z, fma2(g, both(-1.0f), both(1.0f)), both(1.0f)));    // g (1 + z (1 - g))
    } else if constexpr (Act == SLIDE_ATTN_ACT_GELU) {
        pair cdf, density;
        normal_2(z, cdf, density);
        return fma2(z, density, cdf);
    } else {
        return both(1.0f);
    }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where a thread works: a 16-byte column of the slab and every `rows`-th of the CTA's pixels.
struct Place {
    int column, first;
    int mine, held;                    // how many pixels, and how many of them in shared memory
    bool active;
};
__device__ __forceinline__ Place find_place(const NormPlan& pl, int pixels) {
    Place p;
    p.active = (int)threadIdx.x < pl.rows * pl.columns;
    p.first = (int)threadIdx.x / pl.columns;
    p.column = (int)threadIdx.x - p.first * pl.columns;
    p.mine = p.active && p.first < pixels ? (pixels - p.first + pl.rows - 1) / pl.rows : 0;
    p.held = min(p.mine, pl.cached);
    return p;
}
// The groups (within the slab) of a column's channels.
template <int V> __device__ __forceinline__ void find_groups(const NormPlan& pl, int column, int (&group)[V]) {
    int g = column * V / pl.per_group, left = (g + 1) * pl.per_group - column * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        group[e] = g;
        if (--left == 0) { ++g; left = pl.per_group; }
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

constexpr int kCopyGroups = 4;         // groups that a thread's copies come in, so that the sums begin with the first
template <int G> __device__ __forceinline__ void wait_for_group() { copies_wait<kCopyGroups - 1 - G>(); }

template <typename T, int Act>
__global__ void __launch_bounds__(512) norm_forward_kernel(const NormArgs a, const NormPlan pl)
{
    constexpr int Q = Vec<T>::pairs, V = 2 * Q;
    extern __shared__ __align__(16) unsigned char smem[];
    cg::cluster_group cluster = cg::this_cluster();
    const int K = pl.cluster, rank = (int)cluster.block_rank();
    const unsigned unit = blockIdx.x / (unsigned)K;
    const size_t b = unit / (unsigned)pl.slabs;
    const int slab = (int)(unit - (unsigned)b * (unsigned)pl.slabs);
    auto cut = [&](int r) { return (int)((long long)pl.P * r >> pl.log_cluster); };      // the first pixel of a CTA
    const int p0 = cut(rank), pixels = cut(rank + 1) - p0;
    const int slab_groups = pl.width / pl.per_group;
    const Place at = find_place(pl, pixels);
    const int active = pl.rows * pl.columns;

    uint4* cache = reinterpret_cast<uint4*>(smem) + threadIdx.x;                     // [round][active thread]
    float* red = reinterpret_cast<float*>(smem + (size_t)pl.cached * active * 16);
    float* local = red + pl.threads * V;              // sums of this CTA's pixels and of the squares about their mean, by group
    float* total = local + 2 * slab_groups;           // mean and rstd of the image
    const size_t row_bytes = (size_t)pl.C * sizeof(T), step = (size_t)pl.rows * row_bytes;
    const size_t start = (b * (size_t)pl.P + (size_t)(p0 + at.first)) * row_bytes + (size_t)slab * pl.width * sizeof(T) + (size_t)at.column * 16;
    const unsigned char* src = static_cast<const unsigned char*>(a.x) + start;

    grid_dependency_wait();
    auto round_of = [&](int group) { return at.held * group / kCopyGroups; };
#pragma unroll
    for (int g = 0; g < kCopyGroups; ++g) {
        for (int i = round_of(g); i < round_of(g + 1); ++i) copy16(smem_u32(cache + i * active), src + i * step);
        copies_end_group();
    }
    int group[V];
    find_groups<V>(pl, at.column, group);

    // the CTA's own mean ...
    pair sum[Q] = {};
    auto add = [&](const uint4& r) {
        pair v[Q];
        Vec<T>::get(r, v);
#pragma unroll
        for (int e = 0; e < Q; ++e) sum[e] = add2(sum[e], v[e]);
    };
    auto add_group = [&](int g) {
        for (int i = round_of(g); i < round_of(g + 1); ++i) add(cache[i * active]);
    };
    wait_for_group<0>(); add_group(0);
    wait_for_group<1>(); add_group(1);
    wait_for_group<2>(); add_group(2);
    wait_for_group<3>(); add_group(3);
#pragma unroll 4
    for (int i = at.held; i < at.mine; ++i) add(*reinterpret_cast<const uint4*>(src + i * step));
    const int lanes = lanes_for(slab_groups);
    auto fold = [&](const pair (&v)[Q], float* out) {
        if (at.active) leave<V>(red, v);
        __syncthreads();
        sum_cells(red, pl.rows, pl.width, pl.per_group, slab_groups, lanes, out);
    };
    fold(sum, local);
    const float inv_own = 1.0f / ((float)pixels * (float)pl.per_group);               // no CTA is without pixels
    // ... and the squares about it, which lose nothing however far the mean is from zero
    pair mean[Q], square[Q] = {};                      // less the mean
#pragma unroll
    for (int e = 0; e < Q; ++e) mean[e] = make_pair(-local[group[2 * e]] * inv_own, -local[group[2 * e + 1]] * inv_own);
    auto add_square = [&](const uint4& r) {
        pair v[Q];
        Vec<T>::get(r, v);
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            const pair d = add2(v[e], mean[e]);
            square[e] = fma2(d, d, square[e]);
        }
    };
#pragma unroll 2
    for (int i = 0; i < at.held; ++i) add_square(cache[i * active]);
#pragma unroll 4
    for (int i = at.held; i < at.mine; ++i) add_square(*reinterpret_cast<const uint4*>(src + i * step));
    fold(square, local + slab_groups);

    // the cluster's: deviations from the first CTA's mean, so that nothing large cancels
    cluster.sync();
    // a lane for each CTA of the cluster (a power of two)
    for (int first = 0; first < slab_groups; first += (int)blockDim.x >> pl.log_cluster) {
        const int g = first + ((int)threadIdx.x >> pl.log_cluster), r = (int)threadIdx.x & (K - 1);
        const bool there = g < slab_groups;
        const float* theirs = cluster.map_shared_rank(local, r);
        const float per = (float)pl.per_group, n = (float)pl.P * per;
        const float own = (float)(cut(r + 1) - cut(r)) * per;
        const float mine = there ? theirs[g] / own : 0.0f;
        const float m0 = __shfl_sync(0xffffffffu, mine, (int)threadIdx.x & 31 & ~(K - 1));
        float shift = own * (mine - m0);
        for (int o = K / 2; o > 0; o /= 2) shift += __shfl_xor_sync(0xffffffffu, shift, o);
        const float m = m0 + shift / n, d = mine - m;
        float m2 = there ? fmaf(own * d, d, theirs[slab_groups + g]) : 0.0f;
        for (int o = K / 2; o > 0; o /= 2) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
        if (there && r == 0) {
            const float rstd = 1.0f / sqrtf(m2 / n + a.eps);
            total[g] = m;
            total[slab_groups + g] = rstd;
            if (rank == 0) {
                const size_t o = b * pl.groups + slab * slab_groups + g;
                a.mean[o] = m;
                a.rstd[o] = rstd;
            }
        }
    }
    cluster.sync();          // `total` is complete, and nobody reads another CTA's shared memory any more
    if (!at.active) return;

    pair scale[Q], beta[Q];
    get_weights<V>(a.gamma, slab * pl.width + at.column * V, 1.0f, scale);
    get_weights<V>(a.beta, slab * pl.width + at.column * V, 0.0f, beta);
#pragma unroll
    for (int e = 0; e < Q; ++e) {
        mean[e] = make_pair(-total[group[2 * e]], -total[group[2 * e + 1]]);
        scale[e] = mul2(scale[e], make_pair(total[slab_groups + group[2 * e]], total[slab_groups + group[2 * e + 1]]));
    }
    unsigned char* dst = static_cast<unsigned char*>(a.y) + start;
    auto apply = [&](const uint4& r) {
        pair v[Q];
        Vec<T>::get(r, v);
#pragma unroll
        for (int e = 0; e < Q; ++e) v[e] = act_value<Act>(fma2(add2(v[e], mean[e]), scale[e], beta[e]));
        return Vec<T>::put(v);
    };
    for (int i = 0; i < at.held; ++i) *reinterpret_cast<uint4*>(dst + i * step) = apply(cache[i * active]);
#pragma unroll 4
    for (int i = at.held; i < at.mine; ++i)
        *reinterpret_cast<uint4*>(dst + i * step) = apply(*reinterpret_cast<const uint4*>(src + i * step));
}

// Shared memory holds x and, in the place of dy, dz in fp32 (bf16: twice the room): act' is not computed twice.
template <typename T, int Act>
__global__ void __launch_bounds__(512) norm_backward_kernel(const NormArgs a, const NormPlan pl)
{
    constexpr int Q = Vec<T>::pairs, V = 2 * Q;
    extern __shared__ __align__(16) unsigned char smem[];
    cg::cluster_group cluster = cg::this_cluster();
    const int K = pl.cluster, rank = (int)cluster.block_rank();
    const unsigned unit = blockIdx.x / (unsigned)K;
    const size_t b = unit / (unsigned)pl.slabs;
    const int slab = (int)(unit - (unsigned)b * (unsigned)pl.slabs);
    auto cut = [&](int r) { return (int)((long long)pl.P * r >> pl.log_cluster); };      // the first pixel of a CTA
    const int p0 = cut(rank), pixels = cut(rank + 1) - p0;
    const int slab_groups = pl.width / pl.per_group;
    const Place at = find_place(pl, pixels);
    const int active = pl.rows * pl.columns;

    uint4* cache_x = reinterpret_cast<uint4*>(smem) + threadIdx.x;
    uint4* cache_g = cache_x + (size_t)pl.cached * active;                            // dy; then dz, of bf16 the first half
    uint4* cache_h = cache_g + (size_t)pl.cached * active;                            // bf16: the second half of dz
    float* red = reinterpret_cast<float*>(smem + (size_t)pl.cached * active * (16 + 4 * V));
    float* channel = red + pl.threads * V;            // sums of dz, then of dz u, by channel: this CTA's
    float* weighted = channel + 2 * pl.width;         // the same times gamma
    float* local = weighted + 2 * pl.width;           // sums of du, then of du u, by group: this CTA's
    float* total = local + 2 * slab_groups;           // their means over the image
    const size_t row_bytes = (size_t)pl.C * sizeof(T), step = (size_t)pl.rows * row_bytes;
    const size_t start = (b * (size_t)pl.P + (size_t)(p0 + at.first)) * row_bytes + (size_t)slab * pl.width * sizeof(T) + (size_t)at.column * 16;
    const unsigned char* src_x = static_cast<const unsigned char*>(a.x) + start;
    const unsigned char* src_g = static_cast<const unsigned char*>(a.dy) + start;

    grid_dependency_wait();
    auto round_of = [&](int group) { return at.held * group / kCopyGroups; };
#pragma unroll
    for (int g = 0; g < kCopyGroups; ++g) {
        for (int i = round_of(g); i < round_of(g + 1); ++i) {
            copy16(smem_u32(cache_x + i * active), src_x + i * step);
            copy16(smem_u32(cache_g + i * active), src_g + i * step);
        }
        copies_end_group();
    }
    int group[V];
    find_groups<V>(pl, at.column, group);
    pair gamma[Q], beta[Q], mean[Q], rstd[Q];          // less the mean
    get_weights<V>(a.gamma, slab * pl.width + at.column * V, 1.0f, gamma);
    get_weights<V>(a.beta, slab * pl.width + at.column * V, 0.0f, beta);
    {
        const float* m = a.mean + b * pl.groups + slab * slab_groups;
        const float* r = a.rstd + b * pl.groups + slab * slab_groups;
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            mean[e] = make_pair(-m[group[2 * e]], -m[group[2 * e + 1]]);
            rstd[e] = make_pair(r[group[2 * e]], r[group[2 * e + 1]]);
        }
    }
    pair s1[Q] = {}, s2[Q] = {};
    // dz of a column of 16 bytes
    auto slopes = [&](const uint4& rx, const uint4& rg, pair (&u)[Q], pair (&dz)[Q]) {
        Vec<T>::get(rx, u);
        Vec<T>::get(rg, dz);
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            u[e] = mul2(add2(u[e], mean[e]), rstd[e]);
            if constexpr (Act != SLIDE_ATTN_ACT_NONE) dz[e] = mul2(dz[e], act_slope<Act>(fma2(u[e], gamma[e], beta[e])));
        }
    };
    auto add = [&](const pair (&u)[Q], const pair (&dz)[Q]) {
#pragma unroll
        for (int e = 0; e < Q; ++e) {
            s1[e] = add2(s1[e], dz[e]);
            s2[e] = fma2(dz[e], u[e], s2[e]);
        }
    };
    auto add_group = [&](int g) {
        for (int i = round_of(g); i < round_of(g + 1); ++i) {
            pair u[Q], dz[Q];
            slopes(cache_x[i * active], cache_g[i * active], u, dz);
            add(u, dz);
            const pair lower[2] = {dz[0], dz[1]};
            cache_g[i * active] = Vec<float>::put(lower);
            if constexpr (Q == 4) {
                const pair upper[2] = {dz[2], dz[3]};
                cache_h[i * active] = Vec<float>::put(upper);
            }
        }
    };
    wait_for_group<0>(); add_group(0);
    wait_for_group<1>(); add_group(1);
    wait_for_group<2>(); add_group(2);
    wait_for_group<3>(); add_group(3);
#pragma unroll 2
    for (int i = at.held; i < at.mine; ++i) {
        pair u[Q], dz[Q];
        slopes(*reinterpret_cast<const uint4*>(src_x + i * step), *reinterpret_cast<const uint4*>(src_g + i * step), u, dz);
        add(u, dz);
    }
    auto fold = [&](const pair (&v)[Q], float* out) {
        if (at.active) leave<V>(red, v);
        __syncthreads();
        sum_cells(red, pl.rows, pl.width, 1, pl.width, lanes_for(pl.width), out);
    };
    fold(s1, channel);
    fold(s2, channel + pl.width);
    for (int c = threadIdx.x; c < 2 * pl.width; c += blockDim.x) {
        const int ch = c < pl.width ? c : c - pl.width;
        weighted[c] = channel[c] * (a.gamma ? a.gamma[slab * pl.width + ch] : 1.0f);
    }
    __syncthreads();
    sum_cells(weighted, 1, 0, pl.per_group, 2 * slab_groups, lanes_for(2 * slab_groups), local);
    cluster.sync();
    // a lane for each CTA of the cluster (a power of two)
    const float inv = 1.0f / ((float)pl.P * (float)pl.per_group);
    for (int first = 0; first < 2 * slab_groups; first += (int)blockDim.x >> pl.log_cluster) {
        const int g = first + ((int)threadIdx.x >> pl.log_cluster), r = (int)threadIdx.x & (K - 1);
        float s = g < 2 * slab_groups ? cluster.map_shared_rank(local, r)[g] : 0.0f;
        for (int o = K / 2; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (g < 2 * slab_groups && r == 0) total[g] = s * inv;
    }
    if (a.sums) {
        const size_t images = gridDim.x / (unsigned)K / (unsigned)pl.slabs;
        for (int c = rank * (int)blockDim.x + (int)threadIdx.x; c < 2 * pl.width; c += K * (int)blockDim.x) {
            float s = 0.0f;
            for (int r = 0; r < K; ++r) s += cluster.map_shared_rank(channel, r)[c];
            const int which = c / pl.width, ch = c - which * pl.width;
            a.sums[(which * images + b) * pl.C + slab * pl.width + ch] = s;
        }
    }
    cluster.sync();
    if (!at.active) return;

    // dx = rstd (gamma dz - m1 - u m2)
    pair m1[Q], m2[Q];                                 // less the means
#pragma unroll
    for (int e = 0; e < Q; ++e) {
        m1[e] = make_pair(-total[group[2 * e]], -total[group[2 * e + 1]]);
        m2[e] = make_pair(-total[slab_groups + group[2 * e]], -total[slab_groups + group[2 * e + 1]]);
    }
    unsigned char* dst = static_cast<unsigned char*>(a.y) + start;
    auto finish = [&](const pair (&u)[Q], pair (&dz)[Q]) {
#pragma unroll
        for (int e = 0; e < Q; ++e) dz[e] = mul2(rstd[e], fma2(u[e], m2[e], fma2(dz[e], gamma[e], m1[e])));
        return Vec<T>::put(dz);
    };
    for (int i = 0; i < at.held; ++i) {
        pair u[Q], dz[Q], half[2];
        Vec<T>::get(cache_x[i * active], u);
#pragma unroll
        for (int e = 0; e < Q; ++e) u[e] = mul2(add2(u[e], mean[e]), rstd[e]);
        Vec<float>::get(cache_g[i * active], half);
        dz[0] = half[0]; dz[1] = half[1];
        if constexpr (Q == 4) {
            Vec<float>::get(cache_h[i * active], half);
            dz[2] = half[0]; dz[3] = half[1];
        }
        *reinterpret_cast<uint4*>(dst + i * step) = finish(u, dz);
    }
#pragma unroll 2
    for (int i = at.held; i < at.mine; ++i) {
        pair u[Q], dz[Q];
        slopes(*reinterpret_cast<const uint4*>(src_x + i * step), *reinterpret_cast<const uint4*>(src_g + i * step), u, dz);
        *reinterpret_cast<uint4*>(dst + i * step) = finish(u, dz);
    }
}

// dbeta and dgamma: the images' sums, added up in the images' order.  32 channels of one of the two a block, eight rows at a time.
__global__ void norm_weight_kernel(const float* sums, long long images, int C, float* dgamma, float* dbeta)
{
    __shared__ float part[8][33];
    grid_dependency_wait();
    const int c = blockIdx.x * 32 + threadIdx.x, which = blockIdx.y;
    float s = 0.0f;
    if (c < C)
#pragma unroll 4
        for (long long b = threadIdx.y; b < images; b += 8) s += sums[((size_t)which * images + b) * C + c];
    part[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && c < C) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[i][threadIdx.x];
        (which ? dgamma : dbeta)[c] = s;
    }
}

long long gcd(long long a, long long b) { return b ? gcd(b, a % b) : a; }

// maps: 1 forward, 2 backward.  False where no slab fits a block, or no grid the call.
bool make_plan(long long B, long long P, int C, int groups, int size, int maps, int num_sms, NormPlan* out) {
    NormPlan p = {};
    const int V = 16 / size;
    p.P = (int)P; p.C = C; p.groups = groups; p.per_group = C / groups;
    const int narrow = (int)((long long)p.per_group / gcd(p.per_group, V) * V);   // the narrowest slab: whole groups and 16-byte columns
    const int most_slabs = C / narrow;
    if (B * most_slabs > 0x7fffffffLL / kMaxCluster) return false;
    const int held = maps == 1 ? size : size + 4;      // bytes that stay of an element
    // A slab as wide as may be reads the longest runs of memory; narrower ones take smaller clusters, give more CTAs and may be held whole.
    // A CTA's share of 72 KB lets three share an SM.
    constexpr long long kShare = 72 * 1024;
    int best_slabs = 0, best_cluster = 0;
    for (int s = 1; s <= most_slabs; ++s) {
        if (most_slabs % s || C / s / V > 512) continue;
        if (best_slabs && C / s * size < 64) break;
        const long long bytes = P * (C / s) * held;
        int K = 1;
        while (K < kMaxCluster && 2 * K <= P && (bytes > K * kShare || (B * s * K < 2 * num_sms && bytes > K * 8 * 1024))) K *= 2;
        best_slabs = s;
        best_cluster = K;
        if (bytes <= K * kShare && K <= 8 && (B * s * K >= 2 * num_sms || bytes <= K * 16 * 1024)) break;
    }
    if (!best_slabs) return false;
    p.slabs = best_slabs; p.width = C / best_slabs; p.cluster = best_cluster;
    while ((1 << p.log_cluster) < p.cluster) ++p.log_cluster;
    p.columns = p.width / V;
    p.threads = p.columns > 256 ? 512 : 256;
    p.rows = p.threads / p.columns;
    const int active = p.rows * p.columns, slab_groups = p.width / p.per_group;
    const long long rounds = ((P + p.cluster - 1) / p.cluster + p.rows - 1) / p.rows;
    const size_t rest = (size_t)p.threads * V * 4 + (size_t)(4 * slab_groups + (maps > 1 ? 4 * p.width : 0)) * 4;
    const long long round_bytes = (long long)active * V * held;
    const long long fit = (long long)(kMaxSmem - 1024 - rest) / round_bytes;
    p.cached = (int)(rounds < fit ? rounds : fit);
    p.smem = (size_t)p.cached * round_bytes + rest;
    p.blocks = B * p.slabs * p.cluster;
    *out = p;
    return true;
}

template <auto Kernel>
cudaError_t launch_clusters(const NormArgs& a, const NormPlan& p, cudaStream_t stream) {
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.blocks);
    cfg.blockDim = dim3((unsigned)p.threads);
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, Kernel, a, p);
}

template <typename T>
cudaError_t forward_of(const NormArgs& a, const NormPlan& p, int act, cudaStream_t stream) {
    switch (act) {
        case SLIDE_ATTN_ACT_SILU: return launch_clusters<norm_forward_kernel<T, SLIDE_ATTN_ACT_SILU>>(a, p, stream);
        case SLIDE_ATTN_ACT_GELU: return launch_clusters<norm_forward_kernel<T, SLIDE_ATTN_ACT_GELU>>(a, p, stream);
        default: return launch_clusters<norm_forward_kernel<T, SLIDE_ATTN_ACT_NONE>>(a, p, stream);
    }
}
template <typename T>
cudaError_t backward_of(const NormArgs& a, const NormPlan& p, int act, cudaStream_t stream) {
    switch (act) {
        case SLIDE_ATTN_ACT_SILU: return launch_clusters<norm_backward_kernel<T, SLIDE_ATTN_ACT_SILU>>(a, p, stream);
        case SLIDE_ATTN_ACT_GELU: return launch_clusters<norm_backward_kernel<T, SLIDE_ATTN_ACT_GELU>>(a, p, stream);
        default: return launch_clusters<norm_backward_kernel<T, SLIDE_ATTN_ACT_NONE>>(a, p, stream);
    }
}

}  // namespace

// One answer for forward and backward: a slab of the width that both settle for has to fit a block, and the grid its first dimension.
bool group_norm_supports(long long B, long long P, int C, int groups, slide_attn_dtype dtype) {
    NormPlan p;
    const int size = dtype == SLIDE_ATTN_BF16 ? 2 : 4;
    return make_plan(B, P, C, groups, size, 1, kMostSms, &p) && make_plan(B, P, C, groups, size, 2, kMostSms, &p);
}

cudaError_t launch_group_norm_forward(const void* x, const float* gamma, const float* beta, long long B, long long P, int C, int groups, float eps,
                                      slide_attn_activation act, slide_attn_dtype dtype, void* y, float* mean, float* rstd, int num_sms,
                                      cudaStream_t stream) {
    NormPlan p;
    if (!make_plan(B, P, C, groups, dtype == SLIDE_ATTN_BF16 ? 2 : 4, 1, num_sms, &p)) return cudaErrorInvalidValue;
    NormArgs a = {x, gamma, beta, nullptr, y, mean, rstd, nullptr, eps};
    return dtype == SLIDE_ATTN_BF16 ? forward_of<__nv_bfloat16>(a, p, act, stream) : forward_of<float>(a, p, act, stream);
}

cudaError_t launch_group_norm_backward(const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd, const void* dy,
                                       long long B, long long P, int C, int groups, slide_attn_activation act, slide_attn_dtype dtype, void* dx,
                                       float* dgamma, float* dbeta, float* sums, int num_sms, cudaStream_t stream) {
    NormPlan p;
    if (!make_plan(B, P, C, groups, dtype == SLIDE_ATTN_BF16 ? 2 : 4, 2, num_sms, &p)) return cudaErrorInvalidValue;
    NormArgs a = {x, gamma, beta, dy, dx, const_cast<float*>(mean), const_cast<float*>(rstd), dgamma ? sums : nullptr, 0.0f};
    cudaError_t e = dtype == SLIDE_ATTN_BF16 ? backward_of<__nv_bfloat16>(a, p, act, stream) : backward_of<float>(a, p, act, stream);
    if (e != cudaSuccess || !dgamma) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((C + 31) / 32), 2);
    cfg.blockDim = dim3(32, 8);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, norm_weight_kernel, (const float*)sums, B, C, dgamma, dbeta);
}

}  // namespace slide_attn
