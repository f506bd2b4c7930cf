// Block-sparse attention: what its forward and its backward kernels share.
//
// The map of an image is cut into blocks of bh x bw pixels (smaller at its right and lower edges); a list of blocks says which pixels a
// block of queries attends to.  A CTA keeps 64 rows (queries of one block, or keys of one block in the gradient of keys and values) and
// takes the pixels of the listed blocks one after the other, packed into tiles without gaps whatever the blocks' sizes: each row of a
// tile is looked up by itself and copied in pieces of 16 bytes.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace slide_attn {
namespace sparse {

constexpr int kThreads = 128;        // four warps of 16 rows
constexpr int kRows = 64;
constexpr int kMaxBlocks = 1024;     // of a map
constexpr int kMaxTop = 64;          // entries of a list
constexpr int kMaxEdge = 32;         // of a block
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct Geometry {
    int H, W, heads;
    int bh, bw;                      // block of pixels
    int across, blocks;              // blocks in a row of the map, and in all
    int top;                         // entries of a list
    int tiles;                       // tiles of 64 rows that a whole block takes
};

struct Block {
    int y0, x0, h, w;
    __device__ __forceinline__ int size() const { return h * w; }
};
__device__ __forceinline__ Block block_of(const Geometry& g, int id) {
    Block b;
    const int by = id / g.across, bx = id - by * g.across;
    b.y0 = by * g.bh; b.x0 = bx * g.bw;
    b.h = min(g.bh, g.H - b.y0); b.w = min(g.bw, g.W - b.x0);
    return b;
}
// Pixel r of a block, row by row.  (r + 1/2) / w is at least 1 / (2 w) >= 1/64 away from a whole number, far more than fp32 loses below 1024.
__device__ __forceinline__ int pixel_of(const Geometry& g, const Block& b, int r) {
    const int y = (int)(((float)r + 0.5f) * __fdividef(1.0f, (float)b.w));
    return (b.y0 + y) * g.W + b.x0 + (r - y * b.w);
}

// What the backward reads and writes.
struct BackwardMaps {
    const void *q, *k, *v;
    const int* idx;
    const void* out;
    const float* lse;
    const void* dout;
    void *dq, *dk, *dv;
};

template <int D> __device__ __forceinline__ constexpr float root() { return D == 16 ? 0.25f : D == 32 ? 0.17677669529663688f : 0.125f; }

// An entry of a list: its block and how many rows come before it.
struct Entry { int id, start; };

// The row of the list that a thread copies next; rows are asked for in rising order.
struct Cursor {
    int at = -1, start = 0, end = 0;
    Block block = {};
    __device__ __forceinline__ int pixel(const Geometry& g, const Entry* list, int j) {
        while (j >= end) {
            ++at;
            block = block_of(g, list[at].id);
            start = list[at].start;
            end = start + block.size();
        }
        return pixel_of(g, block, j - start);
    }
};

// 16 bytes to shared memory, zeros where there is no row.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ void ldmatrix4(uint32_t at, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t at, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x = hi + lo with 11 bits each: what the three products kept of (a_hi + a_lo)(b_hi + b_lo) lose is 2^-22 of it.  Of an infinity or a NaN
// only the product of the upper parts is to have anything: `finite` is hi, or 0 where that is not finite, and lo is 0 there.
struct Parts { uint32_t hi, finite, lo; };
__device__ __forceinline__ Parts split_tf32(float x) {
    Parts p;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(p.hi) : "f"(x));
    const float rest = x - __uint_as_float(p.hi);
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(p.lo) : "f"(rest));
    const bool ok = (p.hi & 0x7F800000u) != 0x7F800000u;
    p.finite = ok ? p.hi : 0u;
    p.lo = ok ? p.lo : 0u;
    return p;
}

// Tiles of rows of D values in shared memory, and the two products with them.  A warp's operand of 16 rows:
//   scores:  s[n-tile] += rows . tile^T       (16 x D times D x N)
//   gather:  o[n-tile] += weights . tile      (16 x N times N x D), the weights in the layout that `scores` leaves
// `used`: rows of the tile that hold something; whole runs of 16 behind them are skipped.
template <typename T, int D> struct Tile;

// bf16: mma.sync m16n8k16.  Rows of 2 D bytes, their 16-byte pieces exchanged by the row so that the eight rows of an ldmatrix fall into
// different banks.
template <int D> struct Tile<__nv_bfloat16, D> {
    static constexpr int kPieces = D / 8;
    static constexpr int kRowBytes = D * 2;
    static __device__ __forceinline__ uint32_t at(int row, int piece) {
        const int turn = kPieces == 8 ? row & 7 : kPieces == 4 ? (row >> 1) & 3 : (row >> 2) & 1;
        return (uint32_t)(row * kRowBytes + ((piece ^ turn) << 4));
    }
    struct Rows {
        uint32_t a[D / 16][4];
        __device__ __forceinline__ void load(uint32_t tile, int row0, int lane) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                ldmatrix4(tile + at(row0 + (lane & 15), 2 * ks + (lane >> 4)), a[ks][0], a[ks][1], a[ks][2], a[ks][3]);
        }
    };
    template <int NT>
    static __device__ __forceinline__ void scores(const Rows& q, uint32_t tile, int lane, int used, float (&s)[NT][4]) {
#pragma unroll
        for (int n = 0; n < NT; n += 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = s[n + 1][e] = 0.0f;
            if (n * 8 < used) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t b0, b1, b2, b3;
                    ldmatrix4(tile + at(n * 8 + (lane & 7) + ((lane >> 4) << 3), 2 * ks + ((lane >> 3) & 1)), b0, b1, b2, b3);
                    mma_bf16(s[n], q.a[ks], b0, b1);
                    mma_bf16(s[n + 1], q.a[ks], b2, b3);
                }
            }
        }
    }
    template <int NT>
    static __device__ __forceinline__ void gather(const float (&w)[NT][4], uint32_t tile, int lane, int used, float (&o)[D / 8][4]) {
#pragma unroll
        for (int ks = 0; ks < NT / 2; ++ks) {
            if (ks * 16 < used) {
                const uint32_t a[4] = {pack_bf16(w[2 * ks][0], w[2 * ks][1]), pack_bf16(w[2 * ks][2], w[2 * ks][3]),
                                       pack_bf16(w[2 * ks + 1][0], w[2 * ks + 1][1]), pack_bf16(w[2 * ks + 1][2], w[2 * ks + 1][3])};
#pragma unroll
                for (int n = 0; n < D / 8; n += 2) {
                    uint32_t b0, b1, b2, b3;
                    ldmatrix4_trans(tile + at(ks * 16 + (lane & 15), n + (lane >> 4)), b0, b1, b2, b3);
                    mma_bf16(o[n], a, b0, b1);
                    mma_bf16(o[n + 1], a, b2, b3);
                }
            }
        }
    }
};

// fp32: mma.sync m16n8k8 with TF32 operands in two parts each and three products.  The tensor core truncates as it adds, so the small
// products go first and a tile's sums start at zero; sums over tiles are fp32 additions.  Rows are padded by 16 bytes, which puts the
// words of every access into different banks.
template <int D> struct Tile<float, D> {
    static constexpr int kPieces = D / 4;
    static constexpr int kStride = D + 4;                // words
    static constexpr int kRowBytes = kStride * 4;
    static __device__ __forceinline__ uint32_t at(int row, int piece) { return (uint32_t)(row * kRowBytes + piece * 16); }
    static __device__ __forceinline__ float word(uint32_t tile, int row, int col) {
        float v;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(tile + (uint32_t)(row * kRowBytes + col * 4)) : "memory");
        return v;
    }
    struct Rows {
        uint32_t tile;
        int row0;
        __device__ __forceinline__ void load(uint32_t t, int r0, int) { tile = t; row0 = r0; }
        __device__ __forceinline__ float value(int ks, int lane, int i) const {
            return word(tile, row0 + (lane >> 2) + (i & 1) * 8, ks * 8 + (lane & 3) + (i >> 1) * 4);
        }
    };
    template <int NT>
    static __device__ __forceinline__ void scores(const Rows& q, uint32_t tile, int lane, int used, float (&s)[NT][4]) {
        const int g = lane >> 2, t = lane & 3;
        float small[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = small[n][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < D / 8; ++ks) {
            uint32_t hi[4], finite[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Parts p = split_tf32(q.value(ks, lane, i));
                hi[i] = p.hi; finite[i] = p.finite; lo[i] = p.lo;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (n * 8 < used) {
                    const Parts a = split_tf32(word(tile, n * 8 + g, ks * 8 + t)), b = split_tf32(word(tile, n * 8 + g, ks * 8 + t + 4));
                    mma_tf32(small[n], lo, a.finite, b.finite);
                    mma_tf32(small[n], finite, a.lo, b.lo);
                    mma_tf32(s[n], hi, a.hi, b.hi);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] += small[n][e];
    }
    // The order of the keys in a product is free: k = t and k = t + 4 of a step are keys 2 t and 2 t + 1, which is where `scores` leaves them.
    template <int NT>
    static __device__ __forceinline__ void gather(const float (&w)[NT][4], uint32_t tile, int lane, int used, float (&o)[D / 8][4]) {
        const int g = lane >> 2, t = lane & 3;
        float sum[D / 8][4], small[D / 8][4];
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[n][e] = small[n][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < NT; ++ks) {
            if (ks * 8 < used) {
                uint32_t hi[4], finite[4], lo[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Parts p = split_tf32(w[ks][(i & 1) * 2 + (i >> 1)]);
                    hi[i] = p.hi; finite[i] = p.finite; lo[i] = p.lo;
                }
#pragma unroll
                for (int n = 0; n < D / 8; ++n) {
                    const Parts a = split_tf32(word(tile, ks * 8 + 2 * t, n * 8 + g)), b = split_tf32(word(tile, ks * 8 + 2 * t + 1, n * 8 + g));
                    mma_tf32(small[n], lo, a.finite, b.finite);
                    mma_tf32(small[n], finite, a.lo, b.lo);
                    mma_tf32(sum[n], hi, a.hi, b.hi);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] += sum[n][e] + small[n][e];
    }
};

// Copies rows [0, N) of a tile: row r is pixel(r) of the head's plane in `a` (and in `b`, into the tile behind), or zeros.
// Threads per row: kThreads / N.
template <typename T, int D, int N, typename Pixel>
__device__ __forceinline__ void copy_rows(uint32_t tile_a, uint32_t tile_b, const T* a, const T* b, size_t pixel_stride, int count, Pixel pixel) {
    using L = Tile<T, D>;
    constexpr int kPer = kThreads / N, kEach = L::kPieces / kPer;
    static_assert(kEach >= 1 && kEach * kPer == L::kPieces, "whole pieces for each thread");
    const int row = threadIdx.x / kPer, part = threadIdx.x % kPer;
    const bool there = row < count;
    const size_t off = there ? (size_t)pixel(row) * pixel_stride : 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int piece = part + i * kPer;
        copy16(tile_a + L::at(row, piece), reinterpret_cast<const unsigned char*>(a + off) + piece * 16, there);
        if (b) copy16(tile_b + L::at(row, piece), reinterpret_cast<const unsigned char*>(b + off) + piece * 16, there);
    }
}

// The list of a block of queries, by one warp: entries that name no block are left out.  Returns the rows of all of them.
__device__ __forceinline__ int read_list(const Geometry& g, const int* mine, Entry* list, int lane) {
    int n = 0, total = 0;
    for (int i0 = 0; i0 < g.top; i0 += 32) {
        const int i = i0 + lane;
        const int id = i < g.top ? mine[i] : -1;
        const bool there = id >= 0 && id < g.blocks;
        const int size = there ? block_of(g, id).size() : 0;
        const unsigned ones = __ballot_sync(0xffffffffu, there);
        int before = size;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int x = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += x;
        }
        if (there) list[n + __popc(ones & ((1u << lane) - 1u))] = {id, total + before - size};
        n += __popc(ones);
        total += __shfl_sync(0xffffffffu, before, 31);
    }
    return total;
}

// Two neighbouring values of a row.
__device__ __forceinline__ void store2(float* at, float x, float y) { *reinterpret_cast<float2*>(at) = make_float2(x, y); }
__device__ __forceinline__ void store2(__nv_bfloat16* at, float x, float y) { *reinterpret_cast<uint32_t*>(at) = pack_bf16(x, y); }

}  // namespace sparse
}  // namespace slide_attn
