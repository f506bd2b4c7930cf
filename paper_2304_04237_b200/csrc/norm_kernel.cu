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

namespace cg = cooperative_groups;

namespace slide_attn {

namespace {

constexpr int kMaxCluster = 16;
constexpr int kMaxSmem = 227 * 1024;
constexpr int kMostSms = 160;

// How a call is cut up: slabs of `width` channels, clusters of `cluster` CTAs, of whose pixels `cached` rows stay in shared memory.
struct NormPlan {
    int P, C, groups, per_group;       // per_group: channels of a group
    int width, slabs, cluster;
    int columns, rows, threads;        // 16-byte columns of a slab; pixel rows that a CTA takes at a time
    int cached;                        // rows x this many rounds of pixels stay in shared memory
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

template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[4]) {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[8]) {
        v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y);
        v[4] = bf16_lo(r.z); v[5] = bf16_hi(r.z); v[6] = bf16_lo(r.w); v[7] = bf16_hi(r.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[8]) {
        return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
};

template <int Act> __device__ __forceinline__ float act_value(float z) {
    if constexpr (Act == SLIDE_ATTN_ACT_SILU) return z / (1.0f + __expf(-z));
    else if constexpr (Act == SLIDE_ATTN_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    else return z;
}
template <int Act> __device__ __forceinline__ float act_slope(float z) {
    if constexpr (Act == SLIDE_ATTN_ACT_SILU) {
        const float g = 1.0f / (1.0f + __expf(-z));
        return g * (1.0f + z * (1.0f - g));
    } else if constexpr (Act == SLIDE_ATTN_ACT_GELU) {
        return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * 0.39894228f * __expf(-0.5f * z * z);
    } else {
        return 1.0f;
    }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// out[i] = sum over rows r and unit's columns c of red[r][i * unit + c], i < n, by `lanes` lanes of a warp each (a power of two).
__device__ __forceinline__ void reduce_units(const float* red, int rows, int width, int unit, int n, int lanes, float* out) {
    const int per_round = blockDim.x / lanes, lane = threadIdx.x % lanes;
    const int count = rows * unit;
    for (int first = 0; first < n; first += per_round) {
        const int i = first + threadIdx.x / lanes;
        float s = 0.0f;
        if (i < n) {
            int r = lane / unit, c = lane - r * unit;
            for (int e = lane; e < count; e += lanes) {
                s += red[r * width + i * unit + c];
                c += lanes;
                while (c >= unit) { c -= unit; ++r; }
            }
        }
        for (int o = lanes / 2; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (i < n && lane == 0) out[i] = s;
    }
}
__device__ __forceinline__ int lanes_for(int n) { return n * 32 <= (int)blockDim.x ? 32 : 8; }

// What a thread works on.
struct Place {
    int column, first, step;           // column of 16 bytes; its first pixel within the CTA's, and the step to the next
    int mine, held;                    // how many pixels, and how many of them in shared memory
    bool active;
};

template <int V>
__device__ __forceinline__ Place find_place(const NormPlan& pl, int pixels) {
    Place p;
    p.active = (int)threadIdx.x < pl.rows * pl.columns;
    p.column = threadIdx.x % pl.columns;
    p.first = threadIdx.x / pl.columns;
    p.step = pl.rows;
    p.mine = p.active && p.first < pixels ? (pixels - p.first + pl.rows - 1) / pl.rows : 0;
    p.held = p.mine < pl.cached ? p.mine : pl.cached;
    return p;
}

template <typename T, int Act>
__global__ void __launch_bounds__(512) norm_forward_kernel(const NormArgs a, const NormPlan pl)
{
    constexpr int V = Vec<T>::n;
    extern __shared__ __align__(16) unsigned char smem[];
    cg::cluster_group cluster = cg::this_cluster();
    const int K = pl.cluster, rank = (int)cluster.block_rank();
    const long long unit = blockIdx.x / K;
    const long long b = unit / pl.slabs;
    const int slab = (int)(unit % pl.slabs);
    const long long p0 = (long long)pl.P * rank / K, p1 = (long long)pl.P * (rank + 1) / K;
    const int pixels = (int)(p1 - p0), slab_groups = pl.width / pl.per_group;
    const Place at = find_place<V>(pl, pixels);
    const int active = pl.rows * pl.columns;

    uint4* cache = reinterpret_cast<uint4*>(smem);
    float* red = reinterpret_cast<float*>(smem + (size_t)pl.cached * active * 16);
    float* local = red + pl.threads * V;              // mean and sum of squares of this CTA's pixels, by group
    float* total = local + 2 * slab_groups;           // mean and rstd of the image
    const size_t row_bytes = (size_t)pl.C * sizeof(T);
    const size_t start = ((size_t)b * pl.P + p0 + at.first) * row_bytes + (size_t)slab * pl.width * sizeof(T) + (size_t)at.column * 16;
    const unsigned char* src = static_cast<const unsigned char*>(a.x) + start;
    const size_t step = (size_t)at.step * row_bytes;

    grid_dependency_wait();
    // four groups of copies, so that the sums begin with the first
    constexpr int kGroups = 4;
    int ends[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        ends[g] = at.held * (g + 1) / kGroups;
        for (int i = g ? ends[g - 1] : 0; i < ends[g]; ++i) copy16(smem_u32(cache + i * active + threadIdx.x), src + i * step);
        copies_end_group();
    }
    float gamma[V], beta[V];
    int group[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = at.column * V + e;
        group[e] = c / pl.per_group;
        gamma[e] = a.gamma ? a.gamma[slab * pl.width + c] : 1.0f;
        beta[e] = a.beta ? a.beta[slab * pl.width + c] : 0.0f;
    }

    // the CTA's own mean ...
    float sum[V] = {};
    auto add = [&](const uint4& r) {
        float v[V];
        Vec<T>::get(r, v);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += v[e];
    };
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        if (g == 0) copies_wait<3>(); else if (g == 1) copies_wait<2>(); else if (g == 2) copies_wait<1>(); else copies_wait<0>();
        for (int i = g ? ends[g - 1] : 0; i < ends[g]; ++i) add(cache[i * active + threadIdx.x]);
    }
#pragma unroll 4
    for (int i = at.held; i < at.mine; ++i) add(*reinterpret_cast<const uint4*>(src + i * step));
    const int lanes = lanes_for(slab_groups);
    auto fold = [&](const float (&v)[V], float* out) {
        if (at.active)
#pragma unroll
            for (int e = 0; e < V; ++e) red[threadIdx.x * V + e] = v[e];       // [row][channel of the slab]
        __syncthreads();
        reduce_units(red, pl.rows, pl.width, pl.per_group, slab_groups, lanes, out);
        __syncthreads();
    };
    fold(sum, local);
    const float inv_own = 1.0f / ((float)pixels * (float)pl.per_group);        // no CTA is without pixels
    // ... and the squares about it, which lose nothing however far the mean is from zero
    float mean[V], square[V] = {};
#pragma unroll
    for (int e = 0; e < V; ++e) mean[e] = at.active ? local[group[e]] * inv_own : 0.0f;
    auto add_square = [&](const uint4& r) {
        float v[V];
        Vec<T>::get(r, v);
#pragma unroll
        for (int e = 0; e < V; ++e) { const float d = v[e] - mean[e]; square[e] = fmaf(d, d, square[e]); }
    };
    for (int i = 0; i < at.held; ++i) add_square(cache[i * active + threadIdx.x]);
#pragma unroll 4
    for (int i = at.held; i < at.mine; ++i) add_square(*reinterpret_cast<const uint4*>(src + i * step));
    fold(square, local + slab_groups);

    // the cluster's: deviations from the first CTA's mean, so that nothing large cancels
    cluster.sync();
    for (int g = threadIdx.x; g < slab_groups; g += blockDim.x) {
        const float n = (float)pl.P, m0 = cluster.map_shared_rank(local, 0)[g] / ((float)((long long)pl.P / K) * (float)pl.per_group);
        float shift = 0.0f, m2 = 0.0f;
        for (int r = 0; r < K; ++r) {
            const float own = (float)((long long)pl.P * (r + 1) / K - (long long)pl.P * r / K);
            shift += own * (cluster.map_shared_rank(local, r)[g] / (own * (float)pl.per_group) - m0);
        }
        const float m = m0 + shift / n;
        for (int r = 0; r < K; ++r) {
            const float own = (float)((long long)pl.P * (r + 1) / K - (long long)pl.P * r / K);
            const float* there = cluster.map_shared_rank(local, r);
            const float d = there[g] / (own * (float)pl.per_group) - m;
            m2 += there[slab_groups + g] + own * (float)pl.per_group * d * d;
        }
        const float rstd = 1.0f / sqrtf(m2 / (n * (float)pl.per_group) + a.eps);
        total[g] = m;
        total[slab_groups + g] = rstd;
        if (rank == 0) {
            const size_t o = (size_t)b * pl.groups + slab * slab_groups + g;
            a.mean[o] = m;
            a.rstd[o] = rstd;
        }
    }
    cluster.sync();          // `total` is complete, and nobody reads another CTA's shared memory any more
    if (!at.active) return;

    float scale[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { mean[e] = total[group[e]]; scale[e] = total[slab_groups + group[e]] * gamma[e]; }
    unsigned char* dst = static_cast<unsigned char*>(a.y) + start;
    auto apply = [&](const uint4& r) {
        float v[V];
        Vec<T>::get(r, v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = act_value<Act>(fmaf(v[e] - mean[e], scale[e], beta[e]));
        return Vec<T>::put(v);
    };
    for (int i = 0; i < at.held; ++i) *reinterpret_cast<uint4*>(dst + i * step) = apply(cache[i * active + threadIdx.x]);
#pragma unroll 4
    for (int i = at.held; i < at.mine; ++i)
        *reinterpret_cast<uint4*>(dst + i * step) = apply(*reinterpret_cast<const uint4*>(src + i * step));
}

template <typename T, int Act>
__global__ void __launch_bounds__(512) norm_backward_kernel(const NormArgs a, const NormPlan pl)
{
    constexpr int V = Vec<T>::n;
    extern __shared__ __align__(16) unsigned char smem[];
    cg::cluster_group cluster = cg::this_cluster();
    const int K = pl.cluster, rank = (int)cluster.block_rank();
    const long long unit = blockIdx.x / K;
    const long long b = unit / pl.slabs;
    const int slab = (int)(unit % pl.slabs);
    const long long p0 = (long long)pl.P * rank / K, p1 = (long long)pl.P * (rank + 1) / K;
    const int pixels = (int)(p1 - p0), slab_groups = pl.width / pl.per_group;
    const Place at = find_place<V>(pl, pixels);
    const int active = pl.rows * pl.columns;

    uint4* cache_x = reinterpret_cast<uint4*>(smem);
    uint4* cache_g = cache_x + (size_t)pl.cached * active;
    float* red = reinterpret_cast<float*>(smem + (size_t)pl.cached * active * 32);
    float* channel = red + pl.threads * V;            // sums of dz, then of dz u, by channel: this CTA's
    float* weighted = channel + 2 * pl.width;         // the same times gamma
    float* local = weighted + 2 * pl.width;           // sums of du, then of du u, by group: this CTA's
    float* total = local + 2 * slab_groups;           // their means over the image
    const size_t row_bytes = (size_t)pl.C * sizeof(T);
    const size_t start = ((size_t)b * pl.P + p0 + at.first) * row_bytes + (size_t)slab * pl.width * sizeof(T) + (size_t)at.column * 16;
    const unsigned char* src_x = static_cast<const unsigned char*>(a.x) + start;
    const unsigned char* src_g = static_cast<const unsigned char*>(a.dy) + start;
    const size_t step = (size_t)at.step * row_bytes;

    grid_dependency_wait();
    constexpr int kGroups = 4;
    int ends[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        ends[g] = at.held * (g + 1) / kGroups;
        for (int i = g ? ends[g - 1] : 0; i < ends[g]; ++i) {
            copy16(smem_u32(cache_x + i * active + threadIdx.x), src_x + i * step);
            copy16(smem_u32(cache_g + i * active + threadIdx.x), src_g + i * step);
        }
        copies_end_group();
    }
    float gamma[V], beta[V], mean[V], rstd[V];
    int group[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = at.column * V + e;
        group[e] = c / pl.per_group;
        gamma[e] = a.gamma ? a.gamma[slab * pl.width + c] : 1.0f;
        beta[e] = a.beta ? a.beta[slab * pl.width + c] : 0.0f;
        const size_t o = (size_t)b * pl.groups + slab * slab_groups + group[e];
        mean[e] = a.mean[o];
        rstd[e] = a.rstd[o];
    }
    float s1[V] = {}, s2[V] = {};
    auto add = [&](const uint4& rx, const uint4& rg) {
        float x[V], g[V];
        Vec<T>::get(rx, x);
        Vec<T>::get(rg, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float u = (x[e] - mean[e]) * rstd[e];
            const float dz = g[e] * act_slope<Act>(fmaf(u, gamma[e], beta[e]));
            s1[e] += dz;
            s2[e] = fmaf(dz, u, s2[e]);
        }
    };
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        if (g == 0) copies_wait<3>(); else if (g == 1) copies_wait<2>(); else if (g == 2) copies_wait<1>(); else copies_wait<0>();
        for (int i = g ? ends[g - 1] : 0; i < ends[g]; ++i) add(cache_x[i * active + threadIdx.x], cache_g[i * active + threadIdx.x]);
    }
#pragma unroll 2
    for (int i = at.held; i < at.mine; ++i)
        add(*reinterpret_cast<const uint4*>(src_x + i * step), *reinterpret_cast<const uint4*>(src_g + i * step));
    const int lanes_c = lanes_for(pl.width), lanes_g = lanes_for(slab_groups);
    auto fold = [&](const float (&v)[V], float* out) {
        if (at.active)
#pragma unroll
            for (int e = 0; e < V; ++e) red[threadIdx.x * V + e] = v[e];
        __syncthreads();
        reduce_units(red, pl.rows, pl.width, 1, pl.width, lanes_c, out);
        __syncthreads();
    };
    fold(s1, channel);
    fold(s2, channel + pl.width);
    for (int c = threadIdx.x; c < 2 * pl.width; c += blockDim.x) {
        const int ch = c < pl.width ? c : c - pl.width;
        weighted[c] = channel[c] * (a.gamma ? a.gamma[slab * pl.width + ch] : 1.0f);
    }
    __syncthreads();
    reduce_units(weighted, 1, pl.width, pl.per_group, slab_groups, lanes_g, local);
    reduce_units(weighted + pl.width, 1, pl.width, pl.per_group, slab_groups, lanes_g, local + slab_groups);
    cluster.sync();
    const float inv = 1.0f / ((float)pl.P * (float)pl.per_group);
    for (int g = threadIdx.x; g < 2 * slab_groups; g += blockDim.x) {
        float s = 0.0f;
        for (int r = 0; r < K; ++r) s += cluster.map_shared_rank(local, r)[g];
        total[g] = s * inv;
    }
    if (a.sums) {
        const long long images = (long long)gridDim.x / K / pl.slabs;
        for (int c = rank * (int)blockDim.x + (int)threadIdx.x; c < 2 * pl.width; c += K * (int)blockDim.x) {
            float s = 0.0f;
            for (int r = 0; r < K; ++r) s += cluster.map_shared_rank(channel, r)[c];
            const int which = c / pl.width, ch = c - which * pl.width;
            a.sums[((size_t)which * images + b) * pl.C + slab * pl.width + ch] = s;
        }
    }
    cluster.sync();
    if (!at.active) return;

    float m1[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { m1[e] = total[group[e]]; m2[e] = total[slab_groups + group[e]]; }
    unsigned char* dst = static_cast<unsigned char*>(a.y) + start;
    auto apply = [&](const uint4& rx, const uint4& rg) {
        float x[V], g[V];
        Vec<T>::get(rx, x);
        Vec<T>::get(rg, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float u = (x[e] - mean[e]) * rstd[e];
            const float du = g[e] * act_slope<Act>(fmaf(u, gamma[e], beta[e])) * gamma[e];
            g[e] = rstd[e] * (du - m1[e] - u * m2[e]);
        }
        return Vec<T>::put(g);
    };
    for (int i = 0; i < at.held; ++i)
        *reinterpret_cast<uint4*>(dst + i * step) = apply(cache_x[i * active + threadIdx.x], cache_g[i * active + threadIdx.x]);
#pragma unroll 2
    for (int i = at.held; i < at.mine; ++i)
        *reinterpret_cast<uint4*>(dst + i * step) =
            apply(*reinterpret_cast<const uint4*>(src_x + i * step), *reinterpret_cast<const uint4*>(src_g + i * step));
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

// False where no slab fits a block.
bool make_plan(long long B, long long P, int C, int groups, int size, int maps, int num_sms, NormPlan* out) {
    NormPlan p = {};
    const int V = 16 / size;
    p.P = (int)P; p.C = C; p.groups = groups; p.per_group = C / groups;
    const int narrow = (int)((long long)p.per_group / gcd(p.per_group, V) * V);   // the narrowest slab: whole groups and 16-byte columns
    const int most_slabs = C / narrow;
    constexpr long long kShare = 72 * 1024;            // three CTAs share an SM
    auto bytes = [&](int slabs) { return P * (C / slabs) * size * maps; };
    // Wider slabs read longer runs of memory; narrower ones give more CTAs and may be held whole.
    int slabs = 1;
    for (int s = 1; s <= most_slabs; ++s) {
        if (most_slabs % s) continue;
        const bool fits = C / s / V <= 512;
        if (s > 1 && (slabs > 0 && C / slabs / V <= 512) && (C / s) * size < 64) break;
        slabs = s;
        if (fits && bytes(s) <= kMaxCluster * kShare && (B * s * kMaxCluster >= 2 * num_sms || bytes(s) <= 16 * 1024)) break;
    }
    p.slabs = slabs; p.width = C / slabs;
    p.columns = p.width / V;
    if (p.columns > 512) return false;
    p.threads = p.columns > 256 ? 512 : 256;
    p.rows = p.threads / p.columns;
    int K = 1;
    while (K < kMaxCluster && 2 * K <= P && (bytes(slabs) > K * kShare || (B * slabs * K < 2 * num_sms && bytes(slabs) > K * 8 * 1024))) K *= 2;
    p.cluster = K;
    const int active = p.rows * p.columns;
    const long long most = (P + K - 1) / K;
    const long long rounds = (most + p.rows - 1) / p.rows;
    const int slab_groups = p.width / p.per_group;
    const size_t rest = (size_t)p.threads * 16 / size * 4 + (size_t)(4 * slab_groups + (maps > 1 ? 4 * p.width : 0)) * 4;
    const long long fit = (long long)(kMaxSmem - 1024 - rest) / ((long long)active * 16 * maps);
    p.cached = (int)(rounds < fit ? rounds : fit);
    p.smem = (size_t)p.cached * active * 16 * maps + rest;
    p.blocks = B * slabs * K;
    if (B * most_slabs > 0x7fffffffLL / kMaxCluster) return false;
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
