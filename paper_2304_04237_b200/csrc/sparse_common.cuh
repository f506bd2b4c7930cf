// Block-sparse attention: what its forward and its backward kernels share.
//
// The map of an image is cut into blocks of bh x bw pixels (smaller at its right and lower edges); a list of blocks says which pixels a
// block of queries attends to.  A CTA keeps 64 rows (queries of one block, or keys of one block in the gradient of keys and values) and
// takes the pixels of the listed blocks one after the other, packed into tiles without gaps whatever the blocks' sizes: each row of a
// tile is looked up by itself and copied in pieces of 16 bytes.  A fifth warp does that for the four that compute, through a ring of stages: the
// looking up would be a third of their instructions.  Warps wait for one another at named barriers only.
//
// bf16: mma.sync m16n8k16 on the tiles as they are.  fp32: every tile is cut into three bf16 planes in shared memory, once for the four
// warps (split.cuh: exact), and a product is six bf16 products, down to 2^-24 of it.
#pragma once
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "packed.cuh"
#include "ptx.cuh"
#include "split.cuh"

namespace slide_attn {
namespace sparse {

constexpr int kThreads = 128;        // four warps of 16 rows ...
constexpr int kBlock = 160;          // ... and one that sends for what they need
constexpr int kRows = 64;
constexpr int kMaxBlocks = 1024;     // of a map
constexpr int kMaxTop = 64;          // entries of a list
constexpr int kMaxEdge = 32;         // of a block
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// Division of numbers below 2^31 by one that is known ahead, by a multiplication (T. Granlund, P. Montgomery, "Division by invariant integers
// using multiplication", PLDI 1994): with l the least such that 2^l >= d and m = floor(2^32 (2^l - d) / d) + 1, n / d = (m n / 2^32 + n) / 2^l.
struct Divisor {
    unsigned d, mul, shift;
    static Divisor of(unsigned d) {
        unsigned l = 0;
        while ((1ull << l) < d) ++l;
        return {d, (unsigned)(((1ull << 32) * ((1ull << l) - d)) / d + 1), l};
    }
    __device__ __forceinline__ unsigned quotient(unsigned n) const { return (__umulhi(mul, n) + n) >> shift; }
    // n / d, and n becomes n % d
    __device__ __forceinline__ unsigned divide(unsigned& n) const {
        const unsigned q = quotient(n);
        n -= q * d;
        return q;
    }
};

struct Geometry {
    int H, W, heads;
    int bh, bw;                      // block of pixels
    int across, blocks;              // blocks in a row of the map, and in all
    int top;                         // entries of a list
    int tiles;                       // tiles of 64 rows that a whole block takes
    Divisor by_heads, by_tiles, by_blocks, by_across, by_top;      // set by complete()
    void complete() {
        by_heads = Divisor::of(heads); by_tiles = Divisor::of(tiles); by_blocks = Divisor::of(blocks);
        by_across = Divisor::of(across); by_top = Divisor::of(top);
    }
};

struct Block {
    int y0, x0, h, w;
    __device__ __forceinline__ int size() const { return h * w; }
};
__device__ __forceinline__ Block block_of(const Geometry& g, int id) {
    Block b;
    unsigned bx = (unsigned)id;
    const unsigned by = g.by_across.divide(bx);
    b.y0 = (int)by * g.bh; b.x0 = (int)bx * g.bw;
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

__device__ __forceinline__ float log2_approx(float x) {         // off by 2^-22 at most
    float d;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Bytes to shared memory; 16 of zeros where there is nothing to copy.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// A value that is the same in all lanes, so that the compiler knows it: branches on it need no reconvergence.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Named barriers of `Count` threads, by whole warps: a wait, or an arrival only.
template <int Count> __device__ __forceinline__ void bar_sync(int id) {
    __syncwarp();
    asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(Count) : "memory");
}
template <int Count> __device__ __forceinline__ void bar_arrive(int id) {
    __syncwarp();
    asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(Count) : "memory");
}
constexpr int kComputeBarrier = 15;  // among the warps that compute
__device__ __forceinline__ void compute_sync() { bar_sync<kThreads>(kComputeBarrier); }

template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix4(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t at, uint32_t (&r)[4]) { split::ldmatrix_x4_trans(at, r[0], r[1], r[2], r[3]); }

__device__ __forceinline__ void sts128(uint32_t at, const uint32_t (&v)[4]) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

// Where row `row`, 16-byte piece `piece` of a plane of bf16 rows of D values lies: pieces are exchanged by the row, so that the eight rows of
// an ldmatrix fall into different banks.
template <int D> __device__ __forceinline__ uint32_t plane_at(int row, int piece) {
    const int turn = D == 64 ? row & 7 : D == 32 ? (row >> 1) & 3 : (row >> 2) & 1;
    return (uint32_t)(row * (2 * D) + ((piece ^ turn) << 4));
}

// A tile of N rows of D values as it arrives, and the planes that the tensor core reads.
template <typename T, int D> struct Layout {
    static constexpr bool kSplit = sizeof(T) == 4;
    static constexpr int kPlanes = kSplit ? 3 : 1;
    static constexpr int kPieces = D * (int)sizeof(T) / 16;      // of a row as it arrives
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static __device__ __forceinline__ uint32_t at(int row, int piece) {
        if constexpr (kSplit) return (uint32_t)(row * kRowBytes + piece * 16);
        else return plane_at<D>(row, piece);
    }
};

// fp32 rows to three planes of N rows, by all threads of a CTA.
template <int D, int N>
__device__ __forceinline__ void cut_rows(uint32_t raw, uint32_t planes) {
    constexpr int kGroups = N * D / 8;                           // of eight values
#pragma unroll
    for (int i = 0; i < (kGroups + kThreads - 1) / kThreads; ++i) {
        const int e = i * kThreads + (int)threadIdx.x;
        if (kGroups % kThreads != 0 && e >= kGroups) break;
        const int row = e / (D / 8), piece = e % (D / 8);
        float2 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = split::lds_f2(raw + (uint32_t)(row * D * 4 + piece * 32 + j * 8));
#pragma unroll
        for (int plane = 0; plane < 3; ++plane) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = split::pack_upper(v[j].x, v[j].y);
                if (plane < 2) v[j] = split::rest2(v[j]);
            }
            sts128(planes + (uint32_t)(plane * N * 2 * D) + plane_at<D>(row, piece), w);
        }
    }
}

// An operand of 16 rows of a warp: in registers (bf16), or where its planes lie.
template <int D, int Planes> struct Rows;
template <int D> struct Rows<D, 1> {
    uint32_t a[D / 16][4];
    __device__ __forceinline__ void load(uint32_t tile, int, int row0, int lane) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) ldmatrix4(tile + plane_at<D>(row0 + (lane & 15), 2 * ks + (lane >> 4)), a[ks]);
    }
};
template <int D> struct Rows<D, 3> {
    uint32_t tile, stride;
    int row0;
    __device__ __forceinline__ void load(uint32_t planes, int plane_bytes, int first, int) { tile = planes; stride = (uint32_t)plane_bytes; row0 = first; }
    __device__ __forceinline__ void get(int ks, int lane, uint32_t (&r)[3][4]) const {
#pragma unroll
        for (int p = 0; p < 3; ++p) ldmatrix4(tile + p * stride + plane_at<D>(row0 + (lane & 15), 2 * ks + (lane >> 4)), r[p]);
    }
};

template <bool First> __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (First) mma_bf16_c(c, a, b0, b1, 0.0f, 0.0f, 0.0f, 0.0f);
    else mma_bf16(c, a, b0, b1);
}

// large (+)= a . b and small (+)= the five products of parts below, for two neighbouring n-tiles.  Operands that are not finite have parts
// that are not numbers: where `large` is not finite it is the result (`settle`).
template <bool First>
__device__ __forceinline__ void products(float (&large0)[4], float (&large1)[4], float (&small0)[4], float (&small1)[4], const uint32_t (&a)[3][4],
                                         const uint32_t (&b)[3][4]) {
    mma<First>(small0, a[2], b[0][0], b[0][1]);
    mma<First>(small1, a[2], b[0][2], b[0][3]);
    mma<First>(large0, a[0], b[0][0], b[0][1]);
    mma<First>(large1, a[0], b[0][2], b[0][3]);
    constexpr int kA[4] = {0, 1, 1, 0}, kB[4] = {2, 1, 0, 1};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mma_bf16(small0, a[kA[i]], b[kB[i]][0], b[kB[i]][1]);
        mma_bf16(small1, a[kA[i]], b[kB[i]][2], b[kB[i]][3]);
    }
}
__device__ __forceinline__ float settle(float large, float small) {
    return (__float_as_uint(large) & 0x7F800000u) == 0x7F800000u ? large : large + small;
}

// Two neighbouring n-tiles, 16 columns, of rows . tile^T; `tile` points at the first of their rows, `stride`: from a plane of the tile to the next.
template <int D, int Planes>
__device__ __forceinline__ void scores16(const Rows<D, Planes>& rows, uint32_t tile, uint32_t stride, int lane, float (&s0)[4], float (&s1)[4]) {
    const int row = (lane & 7) + ((lane >> 4) << 3), piece = (lane >> 3) & 1;
    if constexpr (Planes == 1) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            uint32_t b[4];
            ldmatrix4(tile + plane_at<D>(row, 2 * ks + piece), b);
            if (ks == 0) {
                mma<true>(s0, rows.a[ks], b[0], b[1]);
                mma<true>(s1, rows.a[ks], b[2], b[3]);
            } else {
                mma<false>(s0, rows.a[ks], b[0], b[1]);
                mma<false>(s1, rows.a[ks], b[2], b[3]);
            }
        }
    } else {
        float small0[4], small1[4];
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            uint32_t a[3][4], b[3][4];
            rows.get(ks, lane, a);
#pragma unroll
            for (int p = 0; p < 3; ++p) ldmatrix4(tile + p * stride + plane_at<D>(row, 2 * ks + piece), b[p]);
            if (ks == 0) products<true>(s0, s1, small0, small1, a, b);
            else products<false>(s0, s1, small0, small1, a, b);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s0[e] = settle(s0[e], small0[e]);
            s1[e] = settle(s1[e], small1[e]);
        }
    }
}

// s[n-tile] = rows . tile^T (16 x D times D x 8 NT), step by step over D for all columns.
template <int D, int Planes, int NT>
__device__ __forceinline__ void scores(const Rows<D, Planes>& rows, uint32_t tile, uint32_t stride, int lane, float (&s)[NT][4]) {
    if constexpr (Planes == 1) {
        const int row = (lane & 7) + ((lane >> 4) << 3), piece = (lane >> 3) & 1;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t b[4];
                ldmatrix4(tile + n * 8 * 2 * D + plane_at<D>(row, 2 * ks + piece), b);
                if (ks == 0) {
                    mma<true>(s[n], rows.a[ks], b[0], b[1]);
                    mma<true>(s[n + 1], rows.a[ks], b[2], b[3]);
                } else {
                    mma<false>(s[n], rows.a[ks], b[0], b[1]);
                    mma<false>(s[n + 1], rows.a[ks], b[2], b[3]);
                }
            }
    } else {
#pragma unroll
        for (int n = 0; n < NT; n += 2) scores16<D, 3>(rows, tile + n * 8 * 2 * D, stride, lane, s[n], s[n + 1]);
    }
}

// o[n-tile] += weights . tile for 16 rows of the tile (16 x 16 times 16 x D), the weights as scores16 leaves them; `tile` points at the first of the
// rows.  bf16: the weights (forward, and P and dS backward) are rounded to bf16, half a step of 2^-8 each, because the tensor core takes no wider operand beside bf16
// rows; a second product with what the rounding leaves would double this half of the arithmetic.  Sums are fp32.  Against 64 bits the forward's result is off by
// 2.3e-3 where the rounding of the result alone gives 1.7e-3, the gradients 2.4e-3.  fp32: the tensor core truncates as it adds, so 16 products are added up from zero and the sums in fp32.
template <int D, int Planes>
__device__ __forceinline__ void gather16(const float (&w0)[4], const float (&w1)[4], uint32_t tile, uint32_t stride, int lane, float (&o)[D / 8][4]) {
    if constexpr (Planes == 1) {
        const uint32_t a[4] = {pack_bf16(w0[0], w0[1]), pack_bf16(w0[2], w0[3]), pack_bf16(w1[0], w1[1]), pack_bf16(w1[2], w1[3])};
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
            uint32_t b[4];
            ldmatrix4_trans(tile + plane_at<D>(lane & 15, n + (lane >> 4)), b);
            mma_bf16(o[n], a, b[0], b[1]);
            mma_bf16(o[n + 1], a, b[2], b[3]);
        }
    } else {
        uint32_t a[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 v = i < 2 ? make_float2(w0[2 * (i & 1)], w0[2 * (i & 1) + 1]) : make_float2(w1[2 * (i & 1)], w1[2 * (i & 1) + 1]);
            a[0][i] = split::pack_upper(v.x, v.y);
            v = split::rest2(v);
            a[1][i] = split::pack_upper(v.x, v.y);
            v = split::rest2(v);
            a[2][i] = split::pack_upper(v.x, v.y);
        }
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
            float large[2][4], small[2][4];
            uint32_t b[3][4];
#pragma unroll
            for (int p = 0; p < 3; ++p) ldmatrix4_trans(tile + p * stride + plane_at<D>(lane & 15, n + (lane >> 4)), b[p]);
            products<true>(large[0], large[1], small[0], small[1], a, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[n][e] += settle(large[0][e], small[0][e]);
                o[n + 1][e] += settle(large[1][e], small[1][e]);
            }
        }
    }
}

// Calls f(width in n-tiles of 8, whether some of the columns hold nothing): for a full tile, or with the smallest of its halves, quarters ... that
// holds `used` rows.  Straight code for each, instead of a branch at each step; columns that hold nothing are in the second half (of two
// n-tiles: anywhere).
template <int NT, typename F> __device__ __forceinline__ void with_part(int used, F f) {
    if constexpr (NT > 2) {
        if (used <= NT * 4) return with_part<NT / 2>(used, f);
    }
    f(std::integral_constant<int, NT>{}, std::true_type{});
}
template <int NT, typename F> __device__ __forceinline__ void with_width(int used, F f) {
    if (used == NT * 8) f(std::integral_constant<int, NT>{}, std::false_type{});
    else with_part<NT>(used, f);
}

// An entry of a list, worked out once: the pixels of a block `width` wide whose first is `pixel`, and the list's rows up to its end.
struct __align__(8) Entry {
    unsigned where;                  // pixel (a map has at most 2^20), width << 21
    int end;
    static __device__ __forceinline__ Entry of(const Geometry& g, const Block& b, int end) {
        return {(unsigned)(b.y0 * g.W + b.x0) | (unsigned)b.w << 21, end};
    }
};

// One unit of work: 64 rows (part `part`) of block r, of one image and head.
struct Unit {
    int row0, r;                     // the first row within the block
    size_t list, image;              // (image, head) number, image number
    int h;
    Block own;
    float inv;                       // 1 / width
    int rows;                        // rows of this part, or none
    __device__ __forceinline__ void find(const Geometry& g, unsigned u) {
        unsigned rest = u;
        unsigned next = g.by_heads.divide(rest);
        h = (int)rest;
        rest = next;
        next = g.by_tiles.divide(rest);
        row0 = (int)rest * kRows;
        rest = next;
        next = g.by_blocks.divide(rest);
        r = (int)rest;
        image = next;
        list = (size_t)next * (unsigned)g.heads + (unsigned)h;
        own = block_of(g, r);
        inv = __fdividef(1.0f, (float)own.w);
        rows = min(own.size() - row0, kRows);
    }
    // the first element of the image's head; elements from pixel to pixel: heads d
    __device__ __forceinline__ size_t plane(const Geometry& g, int d) const { return (image * (unsigned)(g.H * g.W) * (unsigned)g.heads + (unsigned)h) * (unsigned)d; }
    __device__ __forceinline__ const int* entries(const Geometry& g, const int* idx) const { return idx + (list * (unsigned)g.blocks + (unsigned)r) * (unsigned)g.top; }
    __device__ __forceinline__ unsigned pixel(const Geometry& g, int row) const {
        const int at = row0 + row, y = (int)(((float)at + 0.5f) * inv);
        return (unsigned)((own.y0 + y) * g.W + own.x0 + (at - y * own.w));
    }
};

// The pixels of a list, row by row; rows are asked for in rising order and lie within the list.
struct Cursor {
    const Entry* next;
    int start, end;
    int pixel0, skip;                // the block's first pixel, and what a row of the map has beside the block's
    float inv;                       // 1 / width
    __device__ __forceinline__ void reset(const Entry* table) { next = table; start = end = 0; }
    __device__ __forceinline__ unsigned pixel(const Geometry& g, int j) {
        if (j >= end) {
            Entry at;
            do {
                at = *next++;
                start = end;
                end = at.end;
            } while (j >= end);
            const int width = (int)(at.where >> 21);
            pixel0 = (int)(at.where & 0x1FFFFFu);
            skip = g.W - width;
            inv = __fdividef(1.0f, (float)width);
        }
        const int r = j - start, y = (int)(((float)r + 0.5f) * inv);      // exact: see pixel_of
        return (unsigned)(pixel0 + y * skip + r);
    }
};

// The ring of S stages between the warp that copies and those that compute.  Two barriers a stage: full, empty.  The copies of three steps
// (S = 4) may be on their way; a step is handed over when the next but one has been sent for, so that the computing warps find
// the next step there when they are done with one.
template <int S> struct Ring {
    static constexpr int kLate = S - 2;                          // steps between sending for one and handing it over
    int sent = 0, handed = 0, slot = 0, late_slot = 0;
    static __device__ __forceinline__ int full(int slot) { return 1 + slot; }
    static __device__ __forceinline__ int empty(int slot) { return 1 + S + slot; }
    static __device__ __forceinline__ int after(int slot) { return slot == S - 1 ? 0 : slot + 1; }
    // the copying warp: before the copies of a step ...
    __device__ __forceinline__ void claim() { if (sent >= S) bar_sync<kBlock>(empty(slot)); }
    // ... behind them ...
    __device__ __forceinline__ void commit() {
        copies_commit();
        slot = after(slot);
        if (++sent - handed > kLate) {
            copies_wait<kLate>();
            hand_over();
        }
    }
    __device__ __forceinline__ void hand_over() {
        bar_arrive<kBlock>(full(late_slot));
        late_slot = after(late_slot);
        ++handed;
    }
    // ... before a pause ...
    __device__ __forceinline__ void drain() {
        copies_wait<0>();
        while (handed < sent) hand_over();
    }
    // ... and at the end: the barriers are left as they were found.
    __device__ __forceinline__ void finish() {
        drain();
        slot = sent >= S ? slot : 0;
        for (int i = min(sent, S); i > 0; --i) {
            bar_sync<kBlock>(empty(slot));
            slot = after(slot);
        }
    }
};

// Copies of the copying warp: N rows of one map or of two, a row by as many neighbouring lanes as it has pieces.  Lane l has looked up rows l,
// l + 32, ...
template <typename T, int D, int N> struct Sender {
    using L = Layout<T, D>;
    static constexpr int kRowsAtOnce = 32 / L::kPieces, kPasses = N / kRowsAtOnce, kLookups = N / 32;
    static_assert(N % 32 == 0 && kRowsAtOnce >= 1, "rows by lanes");
    // pixels[i]: of row lane + 32 i, anything where there is none; rows from `count` on are zeros
    static __device__ __forceinline__ void send(uint32_t tile_a, uint32_t tile_b, const void* plane_a, const void* plane_b, unsigned pixel_bytes,
                                                const unsigned (&pixels)[kLookups], int count, int lane) {
        if (count >= N) rows<true>(tile_a, tile_b, plane_a, plane_b, pixel_bytes, pixels, count, lane);
        else rows<false>(tile_a, tile_b, plane_a, plane_b, pixel_bytes, pixels, count, lane);
    }
    template <bool Full>
    static __device__ __forceinline__ void rows(uint32_t tile_a, uint32_t tile_b, const void* plane_a, const void* plane_b, unsigned pixel_bytes,
                                                const unsigned (&pixels)[kLookups], int count, int lane) {
        const int row0 = lane / L::kPieces, piece = lane % L::kPieces;
        const unsigned char* const a = static_cast<const unsigned char*>(plane_a) + piece * 16;
        const unsigned char* const b = static_cast<const unsigned char*>(plane_b) + piece * 16;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int row = i * kRowsAtOnce + row0;
            unsigned pixel = __shfl_sync(0xffffffffu, pixels[i * kRowsAtOnce / 32], row & 31);
            const uint32_t at = L::at(row, piece);
            const bool there = Full || row < count;
            if constexpr (!Full) pixel = there ? pixel : 0u;
            const size_t off = (size_t)pixel * pixel_bytes;
            copy16(tile_a + at, a + off, there);
            if (plane_b) copy16(tile_b + at, b + off, there);
        }
    }
};

// What the kernels that keep queries share (the one that keeps keys takes its stages and operands, and sends for them in its own way): a CTA takes its even share of the units, neighbours, one after the other, and the copies run ahead of the
// arithmetic across the units' ends: a list is short (four tiles, often), and the way from its numbers to the first scores takes three
// trips to memory.  There are as many CTAs as the SMs hold.  (Several times as many, of up to eight units, took 3 % longer for
// the forward of 64 x 56 x 56, 2 heads, bf16, and for 32 x 28 x 42, 3 heads of 64, bf16, forward and backward.)
// A unit begins with the step (or steps) that bring the rows that stay.
//   own0, own1: the rows that stay (queries; gradients of the output, or null);  k, v: the tiles.
template <typename T, int D, int N_, int S_, int Own> struct QueryPipe {
    using L = Layout<T, D>;
    static constexpr int N = N_, S = S_;
    static constexpr int kTotals = 8;                                                // more than units that may be under way: S + 1
    static constexpr uint32_t kTile = N * L::kRowBytes, kStage = 2 * kTile, kOwn = kRows * L::kRowBytes;
    static constexpr int kOwnSteps = Own * kRows <= 2 * N ? 1 : Own;                 // one for all, or one each
    static_assert(kRows <= 2 * N, "rows that stay fit a stage");
    static constexpr uint32_t kPlane = 2 * N * 2 * D, kOwnPlane = kRows * 2 * D;      // a plane holds keys and, behind them, values
    static constexpr uint32_t kBehind = L::kSplit ? kPlane / 2 : kTile;              // from the keys to the values
    static constexpr uint32_t kPartsAt = S * kStage, kOwnPartsAt = kPartsAt + (L::kSplit ? 3 * kPlane : 0);
    static constexpr uint32_t kTableAt = kOwnPartsAt + (L::kSplit ? Own * 3 * kOwnPlane : 0);
    static constexpr uint32_t kTotalsAt = kTableAt + kMaxTop * sizeof(Entry);
    static constexpr size_t kSmem = kTotalsAt + kTotals * sizeof(int);

    unsigned char* smem;
    uint32_t base;
    unsigned first;
    int items;
    int slot;                                                                        // the computing warps' stage

    __device__ __forceinline__ QueryPipe(unsigned char* memory, unsigned units) : smem(memory) {
        base = smem_u32(memory);
        const unsigned each = units / gridDim.x, more = units - each * gridDim.x;     // `more` CTAs take one more
        first = blockIdx.x * each + min(blockIdx.x, more);
        items = (int)each + (blockIdx.x < more);
        slot = 0;
    }
    // Rows of a unit's list, known when its first step has arrived.
    __device__ __forceinline__ int& rows_of(int i) const { return reinterpret_cast<int*>(smem + kTotalsAt)[i & (kTotals - 1)]; }

    // All that the copying warp does.
    __device__ __forceinline__ void copy_all(const Geometry& g, const T* own0, const T* own1, const T* k, const T* v, const int* idx) {
        const int lane = threadIdx.x % 32;
        Entry* table = reinterpret_cast<Entry*>(smem + kTableAt);
        const unsigned pixel_bytes = (unsigned)(g.heads * D * (int)sizeof(T));
        Ring<S> ring;
        Unit unit;
        unit.find(g, first);
        int ids[kMaxTop / 32];
        auto read = [&]() {
#pragma unroll
            for (int i = 0; i < kMaxTop / 32; ++i) ids[i] = i * 32 + lane < g.top ? unit.entries(g, idx)[i * 32 + lane] : -1;
        };
        read();
#pragma unroll 1
        for (int item = 0; item < items; ++item) {
            // the rows that stay
            const size_t plane = unit.plane(g, D);
            {
                unsigned pixels[kRows / 32];
#pragma unroll
                for (int i = 0; i < kRows / 32; ++i) pixels[i] = unit.pixel(g, lane + 32 * i);
#pragma unroll
                for (int o = 0; o < kOwnSteps; ++o) {
                    ring.claim();
                    if (o == 0) {
                        // the list: entries that name no block are left out
                        int n = 0, total = 0;
#pragma unroll
                        for (int i = 0; i < kMaxTop / 32; ++i) {
                            if (i * 32 >= g.top) break;
                            const bool there = unit.rows > 0 && (unsigned)ids[i] < (unsigned)g.blocks;
                            Block block = {};
                            if (there) block = block_of(g, ids[i]);
                            int end = block.size();
#pragma unroll
                            for (int d = 1; d < 32; d *= 2) {
                                const int x = __shfl_up_sync(0xffffffffu, end, d);
                                if (lane >= d) end += x;
                            }
                            const unsigned ones = __ballot_sync(0xffffffffu, there);
                            if (there) table[n + __popc(ones & ((1u << lane) - 1u))] = Entry::of(g, block, total + end);
                            n += __popc(ones);
                            total += __shfl_sync(0xffffffffu, end, 31);
                        }
                        if (lane == 0) rows_of(item) = total;
                        __syncwarp();
                    }
                    const uint32_t stage = base + (uint32_t)ring.slot * kStage;
                    if constexpr (Own > 1 && kOwnSteps == 1)
                        Sender<T, D, kRows>::send(stage, stage + kOwn, own0 + plane, own1 + plane, pixel_bytes, pixels, unit.rows, lane);
                    else
                        Sender<T, D, kRows>::send(stage, 0, (o ? own1 : own0) + plane, nullptr, pixel_bytes, pixels, unit.rows, lane);
                    ring.commit();
                }
            }
            const int total = uniform(rows_of(item));
            if (item + 1 < items) {
                unit.find(g, first + item + 1);
                read();                                          // on its way while this unit's tiles are sent for
            }
            Cursor cursor;
            cursor.reset(table);
#pragma unroll 1
            for (int done = 0; done < total; done += N) {
                unsigned pixels[N / 32];
#pragma unroll
                for (int i = 0; i < N / 32; ++i) pixels[i] = done + 32 * i + lane < total ? cursor.pixel(g, done + 32 * i + lane) : 0u;
                ring.claim();
                const uint32_t stage = base + (uint32_t)ring.slot * kStage;
                Sender<T, D, N>::send(stage, stage + kTile, k + plane, v + plane, pixel_bytes, pixels, total - done, lane);
                ring.commit();
            }
            __syncwarp();                                        // the table is free again
        }
        ring.finish();
    }

    // The computing warps: what the next step brings has arrived ...
    __device__ __forceinline__ uint32_t next() {
        bar_sync<kBlock>(Ring<S>::full(slot));
        return base + (uint32_t)slot * kStage;
    }
    // ... and is not needed any more.
    __device__ __forceinline__ void release() {
        bar_arrive<kBlock>(Ring<S>::empty(slot));
        slot = Ring<S>::after(slot);
    }
    // Takes the rows that stay from a unit's first steps.
    __device__ __forceinline__ void take(uint32_t at, int step, int row0, int lane, Rows<D, L::kPlanes>& rows0, Rows<D, L::kPlanes>* rows1) {
        if constexpr (L::kSplit) compute_sync();                 // nobody reads the planes of the unit before any more
#pragma unroll
        for (int o = 0; o < Own; ++o) {
            if (kOwnSteps > 1 && o != step) continue;
            uint32_t from = kOwnSteps > 1 ? at : at + o * kOwn;
            if constexpr (L::kSplit) {
                cut_rows<D, kRows>(from, base + kOwnPartsAt + o * 3 * kOwnPlane);        // read behind a later barrier
                from = base + kOwnPartsAt + o * 3 * kOwnPlane;
            }
            (o ? *rows1 : rows0).load(from, kOwnPlane, row0, lane);
        }
    }
    // The tile as the tensor core reads it: as it is, or its planes.  Returns where the keys are.
    __device__ __forceinline__ uint32_t tile(uint32_t at) {
        if constexpr (!L::kSplit) return at;
        compute_sync();                                          // nobody reads the planes of the tile before any more
        cut_rows<D, 2 * N>(at, base + kPartsAt);
        compute_sync();
        return base + kPartsAt;
    }
};

// How many CTAs of a kernel the current device holds at once, with `Smem` bytes of shared memory each; set up on a device's first call.
template <auto Kernel, size_t Smem> cudaError_t resident(int sms, int* ctas) {
    static std::atomic<int> known[64];                     // of an SM
    int dev = 0, n = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64) n = known[dev].load(std::memory_order_acquire);
    if (n == 0) {
        e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Smem);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, Kernel, kBlock, Smem);
        if (e != cudaSuccess) return e;
        if (n < 1) n = 1;
        if (dev < 64) known[dev].store(n, std::memory_order_release);
    }
    *ctas = n * sms;
    return cudaSuccess;
}

// Two neighbouring values of a row.
__device__ __forceinline__ void store2(float* at, float x, float y) { *reinterpret_cast<float2*>(at) = make_float2(x, y); }
__device__ __forceinline__ void store2(__nv_bfloat16* at, float x, float y) { *reinterpret_cast<uint32_t*>(at) = pack_bf16(x, y); }

}  // namespace sparse
}  // namespace slide_attn
