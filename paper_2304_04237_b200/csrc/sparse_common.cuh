// Block-sparse attention: what its forward and its backward kernels share.
//
// The map of an image is cut into blocks of bh x bw pixels (smaller at its right and lower edges); a list of blocks says which pixels a
// block of queries attends to.  A CTA keeps 64 rows (queries of one block, or keys of one block in the gradient of keys and values) and
// takes the pixels of the listed blocks one after the other, packed into tiles without gaps whatever the blocks' sizes: each row of a
// tile is looked up by itself and copied in pieces of 16 bytes.
//
// bf16: mma.sync m16n8k16 on the tiles as they are.  fp32: every tile is cut into three bf16 planes in shared memory, once for the four
// warps (split.cuh: exact), and a product is six bf16 products, down to 2^-24 of it.
#pragma once
#include "common.cuh"
#include "ptx.cuh"
#include "split.cuh"

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

// (d0, d1) = (a0, a1) * (b0, b1) + (c0, c1)
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b0, float b1, float c0, float c1) {
    asm("{\n\t.reg .b64 ra, rb, rc;\n\t"
        "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmov.b64 rc, {%6, %7};\n\t"
        "fma.rn.f32x2 rc, ra, rb, rc;\n\t"
        "mov.b64 {%0, %1}, rc;\n\t}"
        : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 16 (4) bytes to shared memory, zeros where there is nothing to copy.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
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
    __device__ __forceinline__ void get(int ks, int, uint32_t (&r)[1][4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[0][i] = a[ks][i];
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

// large (+)= a . b and small (+)= the five products of parts below, for two neighbouring n-tiles.  Operands that are not finite have parts
// that are not numbers: where `large` is not finite it is the result (`settle`).
__device__ __forceinline__ void products(float (&large0)[4], float (&large1)[4], float (&small0)[4], float (&small1)[4], const uint32_t (&a)[3][4],
                                         const uint32_t (&b)[3][4]) {
    constexpr int kA[5] = {2, 0, 1, 1, 0}, kB[5] = {0, 2, 1, 0, 1};
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        mma_bf16(small0, a[kA[i]], b[kB[i]][0], b[kB[i]][1]);
        mma_bf16(small1, a[kA[i]], b[kB[i]][2], b[kB[i]][3]);
    }
    mma_bf16(large0, a[0], b[0][0], b[0][1]);
    mma_bf16(large1, a[0], b[0][2], b[0][3]);
}
__device__ __forceinline__ float settle(float large, float small) {
    return (__float_as_uint(large) & 0x7F800000u) == 0x7F800000u ? large : large + small;
}

// s[n-tile] = rows . tile^T (16 x D times D x 8 NT); `stride`: from a plane of the tile to the next.  `used` rows of the tile hold something; runs of 16 behind them are skipped (zeros).
template <int D, int Planes, int NT>
__device__ __forceinline__ void scores(const Rows<D, Planes>& rows, uint32_t tile, uint32_t stride, int lane, int used, float (&s)[NT][4]) {
    const int row = (lane & 7) + ((lane >> 4) << 3), piece = (lane >> 3) & 1;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] = 0.0f;
    if constexpr (Planes == 1) {
#pragma unroll
        for (int n = 0; n < NT; n += 2) {
            if (n * 8 < used) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t b[4];
                    ldmatrix4(tile + plane_at<D>(n * 8 + row, 2 * ks + piece), b);
                    mma_bf16(s[n], rows.a[ks], b[0], b[1]);
                    mma_bf16(s[n + 1], rows.a[ks], b[2], b[3]);
                }
            }
        }
    } else {
        float small[NT][4] = {};
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            uint32_t a[3][4];
            rows.get(ks, lane, a);
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                if (n * 8 < used) {
                    uint32_t b[3][4];
#pragma unroll
                    for (int p = 0; p < 3; ++p) ldmatrix4(tile + p * stride + plane_at<D>(n * 8 + row, 2 * ks + piece), b[p]);
                    products(s[n], s[n + 1], small[n], small[n + 1], a, b);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = settle(s[n][e], small[n][e]);
    }
}

// o[n-tile] += weights . tile (16 x 8 NT times 8 NT x D), the weights as `scores` leaves them.  fp32: the tensor core truncates as it adds, so a
// tile's sums start at zero and are added in fp32.
template <int D, int Planes, int NT>
__device__ __forceinline__ void gather(const float (&w)[NT][4], uint32_t tile, uint32_t stride, int lane, int used, float (&o)[D / 8][4]) {
    if constexpr (Planes == 1) {
#pragma unroll
        for (int ks = 0; ks < NT / 2; ++ks) {
            if (ks * 16 < used) {
                const uint32_t a[4] = {pack_bf16(w[2 * ks][0], w[2 * ks][1]), pack_bf16(w[2 * ks][2], w[2 * ks][3]),
                                       pack_bf16(w[2 * ks + 1][0], w[2 * ks + 1][1]), pack_bf16(w[2 * ks + 1][2], w[2 * ks + 1][3])};
#pragma unroll
                for (int n = 0; n < D / 8; n += 2) {
                    uint32_t b[4];
                    ldmatrix4_trans(tile + plane_at<D>(ks * 16 + (lane & 15), n + (lane >> 4)), b);
                    mma_bf16(o[n], a, b[0], b[1]);
                    mma_bf16(o[n + 1], a, b[2], b[3]);
                }
            }
        }
    } else {
        float large[D / 8][4] = {}, small[D / 8][4] = {};
#pragma unroll
        for (int ks = 0; ks < NT / 2; ++ks) {
            if (ks * 16 < used) {
                uint32_t a[3][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 v = make_float2(w[2 * ks + (i >> 1)][2 * (i & 1)], w[2 * ks + (i >> 1)][2 * (i & 1) + 1]);
                    a[0][i] = split::pack_upper(v.x, v.y);
                    v = split::rest2(v);
                    a[1][i] = split::pack_upper(v.x, v.y);
                    v = split::rest2(v);
                    a[2][i] = split::pack_upper(v.x, v.y);
                }
#pragma unroll
                for (int n = 0; n < D / 8; n += 2) {
                    uint32_t b[3][4];
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        ldmatrix4_trans(tile + p * stride + plane_at<D>(ks * 16 + (lane & 15), n + (lane >> 4)), b[p]);
                    products(large[n], large[n + 1], small[n], small[n + 1], a, b);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] += settle(large[n][e], small[n][e]);
    }
}

// The row of a list that a thread copies next; rows are asked for in rising order and lie within the list.  Entries that name no block
// hold no rows.
struct Cursor {
    int at, start, end;
    Block block;
    __device__ __forceinline__ void reset() { at = -1; start = end = 0; }
    __device__ __forceinline__ int pixel(const Geometry& g, const int* list, int j) {
        while (j >= end) {
            const int id = list[++at];
            if ((unsigned)id < (unsigned)g.blocks) {
                block = block_of(g, id);
                start = end;
                end += block.size();
            }
        }
        return pixel_of(g, block, j - start);
    }
};

// Copies row threadIdx.x / (kThreads / N) of a tile (and of the tile behind it) from that pixel of a head's plane, or zeros.
template <typename T, int D, int N>
__device__ __forceinline__ void copy_rows(uint32_t tile_a, uint32_t tile_b, const T* a, const T* b, size_t offset, bool there) {
    using L = Layout<T, D>;
    constexpr int kPer = kThreads / N, kEach = L::kPieces / kPer;
    static_assert(kEach >= 1 && kEach * kPer == L::kPieces, "whole pieces for each thread");
    const int row = threadIdx.x / kPer, part = threadIdx.x % kPer;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int piece = part + i * kPer;
        copy16(tile_a + L::at(row, piece), reinterpret_cast<const unsigned char*>(a + offset) + piece * 16, there);
        if (b) copy16(tile_b + L::at(row, piece), reinterpret_cast<const unsigned char*>(b + offset) + piece * 16, there);
    }
}

// One unit of work of the kernels that keep queries: 64 rows (part `part`) of block r, of one image and head.
struct Unit {
    int h, part, r;
    long long b;
    Block own;
    int rows;                        // rows of this part, or none
    __device__ __forceinline__ void find(const Geometry& g, unsigned u) {
        h = u % g.heads; u /= g.heads;
        part = u % g.tiles; u /= g.tiles;
        r = u % g.blocks;
        b = u / g.blocks;
        own = block_of(g, r);
        rows = min(own.size() - part * kRows, kRows);
    }
    __device__ __forceinline__ size_t plane(const Geometry& g, int d) const { return ((size_t)b * g.H * g.W * g.heads + h) * d; }
    __device__ __forceinline__ const int* list(const Geometry& g, const int* idx) const { return idx + ((b * g.heads + h) * (size_t)g.blocks + r) * g.top; }
    __device__ __forceinline__ int pixel(const Geometry& g, int row) const { return pixel_of(g, own, part * kRows + row); }
};

// What the kernels that keep queries share: a CTA takes `chain` neighbouring units one after the other, and the copies run S - 1 tiles ahead
// of the arithmetic, across the units' ends: a list is short (four tiles, often), and the way from its numbers to the first scores takes three
// trips to memory.  Lists come S - 1 units ahead.
//   own0, own1: the rows that stay (queries; gradients of the output, or null);  k, v: the tiles.
template <typename T, int D, int N, int S, int Own> struct QueryPipe {
    using L = Layout<T, D>;
    static constexpr int kLists = 8;                                                 // 2 S - 1 at least
    static constexpr uint32_t kTile = N * L::kRowBytes, kStage = 2 * kTile, kOwn = kRows * L::kRowBytes;
    static constexpr uint32_t kPlane = 2 * N * 2 * D, kOwnPlane = kRows * 2 * D;      // a plane holds keys and, behind them, values
    static constexpr uint32_t kBehind = L::kSplit ? kPlane / 2 : kTile;              // from the keys to the values
    static constexpr uint32_t kOwnAt = S * kStage, kPartsAt = kOwnAt + S * Own * kOwn;
    static constexpr uint32_t kOwnPartsAt = kPartsAt + (L::kSplit ? 3 * kPlane : 0), kListsAt = kOwnPartsAt + (L::kSplit ? Own * 3 * kOwnPlane : 0);
    static constexpr size_t kSmem = kListsAt + kLists * (kMaxTop + 1) * sizeof(int);

    const Geometry& g;
    const T *own0, *own1, *k, *v;
    const int* idx;
    unsigned first;
    int items;
    uint32_t base;
    int* lists;
    int* rows_of;                    // rows of an item's list
    // the copies' place
    int item, step, steps, listed;
    Unit unit;
    Cursor cursor;
    size_t plane;

    __device__ __forceinline__ QueryPipe(const Geometry& geometry, unsigned char* smem, const T* o0, const T* o1, const T* keys, const T* values,
                                         const int* index, unsigned units, int chain)
        : g(geometry), own0(o0), own1(o1), k(keys), v(values), idx(index) {
        base = smem_u32(smem);
        lists = reinterpret_cast<int*>(smem + kListsAt);
        rows_of = lists + kLists * kMaxTop;
        first = blockIdx.x * (unsigned)chain;
        items = (int)min((unsigned)chain, units - first);
        item = step = 0;
    }
    __device__ __forceinline__ void start() {
        for (int i = 0; i < min(S - 1, items); ++i) {
            Unit u;
            u.find(g, first + i);
            if ((int)threadIdx.x < g.top) lists[i * kMaxTop + threadIdx.x] = u.list(g, idx)[threadIdx.x];
        }
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < S - 1; ++i) copy(i);
    }
    // The copies of the tile that comes `number` tiles after the CTA's first.
    __device__ __forceinline__ void copy(int number) {
        if (item < items) {
            const int* list = lists + (item % kLists) * kMaxTop;
            if (step == 0) {
                unit.find(g, first + item);
                plane = unit.plane(g, D);
                const int lane = threadIdx.x % 32;
                listed = 0;
                if (unit.rows > 0)
                    for (int i = 0; i < g.top; i += 32) {
                        const int id = i + lane < g.top ? list[i + lane] : -1;
                        listed += (int)__reduce_add_sync(0xffffffffu, (unsigned)id < (unsigned)g.blocks ? (unsigned)block_of(g, id).size() : 0u);
                    }
                steps = max(1, (listed + N - 1) / N);
                if (threadIdx.x == 0) rows_of[item % kLists] = listed;
                cursor.reset();
                const int row = threadIdx.x / (kThreads / kRows);
                const bool there = row < unit.rows;
                const uint32_t at = base + kOwnAt + (uint32_t)(item % S) * (Own * kOwn);
                copy_rows<T, D, kRows>(at, at + kOwn, own0 + plane, Own > 1 ? own1 + plane : static_cast<const T*>(nullptr),
                                       there ? (size_t)unit.pixel(g, row) * g.heads * D : 0, there);
                if (item + S - 1 < items && (int)threadIdx.x < g.top) {
                    Unit u;
                    u.find(g, first + item + S - 1);
                    copy4(smem_u32(lists + ((item + S - 1) % kLists) * kMaxTop + threadIdx.x), u.list(g, idx) + threadIdx.x);
                }
            }
            const int j = step * N + (int)threadIdx.x / (kThreads / N);
            const bool there = j < listed;
            const uint32_t at = base + (uint32_t)(number % S) * kStage;
            copy_rows<T, D, N>(at, at + kTile, k + plane, v + plane, there ? (size_t)cursor.pixel(g, list, j) * g.heads * D : 0, there);
            if (++step == steps) { step = 0; ++item; }
        }
        copies_commit();
    }
    // Tile `number` has arrived and every thread is done with the one before; the next copies are sent for.  fp32: the tile's planes, and
    // (`fresh`) those of the unit's own rows, are made.  Returns where the keys are.
    __device__ __forceinline__ uint32_t next(int number, bool fresh, int compute_item) {
        copies_wait<S - 2>();
        __syncthreads();
        copy(number + S - 1);
        const uint32_t raw = base + (uint32_t)(number % S) * kStage;
        if constexpr (!L::kSplit) return raw;
        cut_rows<D, 2 * N>(raw, base + kPartsAt);
        if (fresh) {
            const uint32_t at = base + kOwnAt + (uint32_t)(compute_item % S) * (Own * kOwn);
#pragma unroll
            for (int o = 0; o < Own; ++o) cut_rows<D, kRows>(at + o * kOwn, base + kOwnPartsAt + o * 3 * kOwnPlane);
        }
        __syncthreads();
        return base + kPartsAt;
    }
    __device__ __forceinline__ uint32_t own_at(int compute_item, int which) const {
        if constexpr (L::kSplit) return base + kOwnPartsAt + which * 3 * kOwnPlane;
        else return base + kOwnAt + (uint32_t)(compute_item % S) * (Own * kOwn) + which * kOwn;
    }
};

// Units a CTA takes one after the other: enough for some ten tiles, while the CTAs still fill the SMs a few times over.
inline int chain_of(const Geometry& g, unsigned units, int sms, int tile) {
    const int steps = (g.top * g.bh * g.bw + tile - 1) / tile;
    int chain = 1;
    while (chain < 8 && chain * steps < 10 && units / (2 * chain) >= 8u * (unsigned)sms) chain *= 2;
    return chain;
}

// Two neighbouring values of a row.
__device__ __forceinline__ void store2(float* at, float x, float y) { *reinterpret_cast<float2*>(at) = make_float2(x, y); }
__device__ __forceinline__ void store2(__nv_bfloat16* at, float x, float y) { *reinterpret_cast<uint32_t*>(at) = pack_bf16(x, y); }

}  // namespace sparse
}  // namespace slide_attn
