// Dropout from a counter-based generator: y = residual + (kept ? x / (1 - p) : 0), and its gradient dx = kept ? dy / (1 - p) : 0.
//
// Element e is kept if word e % 4 of Philox4x32 with ten rounds (J. K. Salmon et al., "Parallel random numbers: as easy as 1, 2, 3",
// SC11) at counter (e / 4, offset) under the key (seed) is at least floor(p 2^32), so the mask is never stored: the backward
// computes it again.  In units of images the word of image b decides for all of its elements.
//
// fp32 is bound by memory (3 maps forward, 2 backward): 64 x 56 x 56 x 96, 35.2 and 24.4 us, of 35.3 and 23.6.  In bf16 the generator's products of
// 32 x 32 -> 64 bits, ten for two elements, keep the pipe that makes them (fmaheavy) busy for 73 % of the cycles in which an SM has work, where a thread's loads
// come first and its products then: 64 x 56 x 56 x 96 takes 40.2 us for forward and backward, the memory alone 29.5.  Whole images, 32 x 28 x 42 x 192, fp32,
// p = 0.2: 13.8 us, of 13.2.
// The products with the scale are fp32, and the sum is rounded to the storage type once.
#include "operators.cuh"

namespace slide_attn {

namespace {

struct DropArgs {
    const void* x;
    const void* residual;           // or null
    void* y;
    const unsigned long long* rng;  // seed, offset
    long long n;                    // elements
    long long per_image;
    float scale;
    unsigned threshold;
    int none;                       // images: p = 1, nothing is kept
};

struct Key {
    unsigned k0[10], k1[10], c2, c3;
};

__device__ __forceinline__ void make_key(const unsigned long long* rng, Key& key) {
    const unsigned long long seed = rng[0], offset = rng[1];
    unsigned a = (unsigned)seed, b = (unsigned)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        key.k0[r] = a; key.k1[r] = b;
        a += 0x9E3779B9u; b += 0xBB67AE85u;
    }
    key.c2 = (unsigned)offset; key.c3 = (unsigned)(offset >> 32);
}

__device__ __forceinline__ uint4 words(unsigned long long counter, const Key& key) {
    unsigned a = (unsigned)counter, b = (unsigned)(counter >> 32), c = key.c2, d = key.c3;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long p = (unsigned long long)a * 0xD2511F53u, q = (unsigned long long)c * 0xCD9E8D57u;
        a = (unsigned)(q >> 32) ^ b ^ key.k0[r];
        b = (unsigned)q;
        c = (unsigned)(p >> 32) ^ d ^ key.k1[r];
        d = (unsigned)p;
    }
    return make_uint4(a, b, c, d);
}

__device__ __forceinline__ unsigned word_of(unsigned long long e, const Key& key) {
    const uint4 w = words(e >> 2, key);
    const unsigned lane = (unsigned)e & 3u;
    return lane == 0 ? w.x : lane == 1 ? w.y : lane == 2 ? w.z : w.w;
}

template <typename T> struct Pack;
template <> struct Pack<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[4]) {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct Pack<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[8]) {
        v[0] = bf16_lo(r.x); v[1] = bf16_hi(r.x); v[2] = bf16_lo(r.y); v[3] = bf16_hi(r.y);
        v[4] = bf16_lo(r.z); v[5] = bf16_hi(r.z); v[6] = bf16_lo(r.w); v[7] = bf16_hi(r.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[8]) {
        return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
};

constexpr int kThreads = 256, kEach = 4;         // 16-byte pieces a thread takes

// The value of a dropped element is not added, and not multiplied by zero either: an infinity or a NaN there does not reach the sum.  (A
// predicated instruction; a choice between two results costs one more.)
__device__ __forceinline__ void add_if_kept(float& sum, unsigned word, unsigned threshold, float x, float scale) {
    asm("{\n\t.reg .pred p;\n\t"
        "setp.ge.u32 p, %1, %2;\n\t"
        "@p fma.rn.f32 %0, %3, %4, %0;\n\t}"
        : "+f"(sum) : "r"(word), "r"(threshold), "f"(x), "f"(scale));
}

template <typename T, bool Residual>
__global__ void __launch_bounds__(kThreads, 4) drop_elements_kernel(const DropArgs a)
{
    constexpr int V = Pack<T>::n;
    grid_dependency_wait();
    const long long pieces = a.n / V;
    const long long first = (long long)blockIdx.x * (kThreads * kEach) + threadIdx.x;
    uint4 x[kEach], r[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long v = first + i * kThreads;
        if (v < pieces) {
            x[i] = static_cast<const uint4*>(a.x)[v];
            if constexpr (Residual) r[i] = static_cast<const uint4*>(a.residual)[v];
        }
    }
    Key key;
    make_key(a.rng, key);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long v = first + i * kThreads;
        if (v >= pieces) break;
        float xv[V], rv[V] = {};
        Pack<T>::get(x[i], xv);
        if constexpr (Residual) Pack<T>::get(r[i], rv);
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const uint4 w = words((unsigned long long)v * (V / 4) + q, key);
            const unsigned word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                add_if_kept(rv[q * 4 + e], word[e], a.threshold, xv[q * 4 + e], a.scale);
        }
        static_cast<uint4*>(a.y)[v] = Pack<T>::put(rv);
    }
    // what no 16-byte piece holds
    if (blockIdx.x == 0 && threadIdx.x < a.n - pieces * V) {
        const long long e = pieces * V + threadIdx.x;
        float sum = Residual ? to_float(static_cast<const T*>(a.residual)[e]) : 0.0f;
        add_if_kept(sum, word_of(e, key), a.threshold, to_float(static_cast<const T*>(a.x)[e]), a.scale);
        static_cast<T*>(a.y)[e] = from_float<T>(sum);
    }
}

// Images of whole 16-byte pieces: a block works on one image, and does not read x where that is dropped.
template <typename T, bool Residual>
__global__ void __launch_bounds__(kThreads) drop_images_kernel(const DropArgs a, int blocks_per_image)
{
    constexpr int V = Pack<T>::n;
    grid_dependency_wait();
    const long long image = blockIdx.x / blocks_per_image;
    const long long pieces = a.per_image / V, base = image * pieces;
    const long long first = (long long)(blockIdx.x - image * blocks_per_image) * (kThreads * kEach) + threadIdx.x;
    Key key;
    make_key(a.rng, key);
    const bool kept = word_of(image, key) >= a.threshold && !a.none;
    uint4 x[kEach], r[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long v = first + i * kThreads;
        x[i] = r[i] = make_uint4(0, 0, 0, 0);
        if (v < pieces) {
            if (kept) x[i] = static_cast<const uint4*>(a.x)[base + v];
            if constexpr (Residual) r[i] = static_cast<const uint4*>(a.residual)[base + v];
        }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long v = first + i * kThreads;
        if (v >= pieces) break;
        if (kept) {
            float xv[V], rv[V];
            Pack<T>::get(x[i], xv);
            Pack<T>::get(r[i], rv);
#pragma unroll
            for (int e = 0; e < V; ++e) xv[e] = fmaf(xv[e], a.scale, rv[e]);
            r[i] = Pack<T>::put(xv);
        }
        static_cast<uint4*>(a.y)[base + v] = r[i];
    }
}

// Images that end inside a 16-byte piece: element by element.
template <typename T, bool Residual>
__global__ void __launch_bounds__(kThreads) drop_images_ragged_kernel(const DropArgs a)
{
    grid_dependency_wait();
    Key key;
    make_key(a.rng, key);
    for (long long e = (long long)blockIdx.x * kThreads + threadIdx.x; e < a.n; e += (long long)gridDim.x * kThreads) {
        float sum = Residual ? to_float(static_cast<const T*>(a.residual)[e]) : 0.0f;
        if (!a.none && word_of(e / a.per_image, key) >= a.threshold) sum = fmaf(to_float(static_cast<const T*>(a.x)[e]), a.scale, sum);
        static_cast<T*>(a.y)[e] = from_float<T>(sum);
    }
}

template <typename T, bool Residual>
cudaError_t launch_of(const DropArgs& a, bool images, int num_sms, cudaStream_t stream) {
    constexpr int V = Pack<T>::n;
    constexpr long long kPieces = (long long)kThreads * kEach;
    if (!images && !a.none) {
        const long long blocks = (a.n / V + kPieces - 1) / kPieces;
        return launch_chained(drop_elements_kernel<T, Residual>, dim3((unsigned)(blocks ? blocks : 1)), kThreads, 0, stream, a);
    }
    if (a.per_image % V) {
        const long long blocks = (a.n + kThreads - 1) / kThreads;
        const long long most = 16LL * num_sms;
        return launch_chained(drop_images_ragged_kernel<T, Residual>, dim3((unsigned)(blocks < most ? blocks : most)), kThreads, 0, stream, a);
    }
    const long long per = (a.per_image / V + kPieces - 1) / kPieces;
    return launch_chained(drop_images_kernel<T, Residual>, dim3((unsigned)(per * (a.n / a.per_image))), kThreads, 0, stream, a, (int)per);
}

}  // namespace

// Whether the blocks fit a grid's first dimension: a block takes 4096 (fp32) or 8192 elements, of one image where images are dropped.
bool dropout_supports(long long images, long long per_image, bool whole_images) {
    if (!whole_images) return images * per_image <= (1LL << 40);
    return per_image % 4 != 0 || images <= (1LL << 30) / ((per_image + 4095) / 4096);
}

cudaError_t launch_dropout(const void* x, const void* residual, void* y, long long images, long long per_image, double p, bool whole_images,
                           const unsigned long long* rng, slide_attn_dtype dtype, int num_sms, cudaStream_t stream) {
    DropArgs a = {};
    a.x = x; a.residual = residual; a.y = y; a.rng = rng;
    a.n = images * per_image; a.per_image = per_image;
    a.none = p >= 1.0;                 // no word is enough, which 32 bits cannot say: all is one image that is dropped
    if (a.none) a.per_image = a.n;
    a.threshold = a.none ? 0u : (unsigned)(p * 4294967296.0);
    a.scale = a.none ? 0.0f : (float)(1.0 / (1.0 - p));
    if (dtype == SLIDE_ATTN_BF16)
        return residual ? launch_of<__nv_bfloat16, true>(a, whole_images, num_sms, stream) : launch_of<__nv_bfloat16, false>(a, whole_images, num_sms, stream);
    return residual ? launch_of<float, true>(a, whole_images, num_sms, stream) : launch_of<float, false>(a, whole_images, num_sms, stream);
}

}  // namespace slide_attn
