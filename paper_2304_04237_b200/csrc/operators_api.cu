// C ABI of the operators around and beside the local attention: group norm, dropout, block-sparse attention.  They take sizes instead of a
// context and workspaces instead of owning any; here their arguments are checked, the arithmetic lives in the kernel files.
#include <math.h>

#include <atomic>

#include "operators.cuh"

using namespace slide_attn;

namespace {

bool misaligned(const void* p, unsigned to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

template <typename... P> bool any_null(P... p) { return (... || (p == nullptr)); }
template <typename... P> bool any_misaligned(P... p) { return (... || misaligned(p)); }

// Memory that a call reads or writes.
struct Span {
    uintptr_t at;
    size_t bytes;
    Span(const void* p, size_t n) : at(reinterpret_cast<uintptr_t>(p)), bytes(p ? n : 0) {}
};
// Whether an output shares memory with one of the others.
bool meet(const Span& a, const Span& b) { return a.bytes && b.bytes && a.at < b.at + b.bytes && b.at < a.at + a.bytes; }
template <typename... S> bool meets(const Span& out, const S&... s) { return (... || meet(out, s)); }

size_t size_of(slide_attn_dtype t) { return t == SLIDE_ATTN_BF16 ? 2 : 4; }

// The current device is one that the kernels run on; its SMs.
slide_attn_status current_device(int* num_sms) {
    static std::atomic<int> known[64];                 // host threads may call at once
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return SLIDE_ATTN_ERR_CUDA; }
    if (dev < 64) n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        int major = 0;
        if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
            cudaGetLastError();
            return SLIDE_ATTN_ERR_CUDA;
        }
        if (major != 10) return SLIDE_ATTN_ERR_ARCH;
        if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    }
    *num_sms = n;
    return SLIDE_ATTN_OK;
}

slide_attn_status launched(cudaError_t e) {
    if (e == cudaSuccess) return SLIDE_ATTN_OK;
    cudaGetLastError();
    return SLIDE_ATTN_ERR_CUDA;
}

bool known_dtype(slide_attn_dtype t) { return t == SLIDE_ATTN_F32 || t == SLIDE_ATTN_BF16; }

slide_attn_status norm_shape(int B, int H, int W, int C, int groups, slide_attn_dtype dtype, bool backward, size_t* workspace) {
    if (B < 1 || H < 1 || W < 1 || C < 1 || groups < 1 || !known_dtype(dtype)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (C % groups != 0 || C % 8 != 0) return SLIDE_ATTN_ERR_UNSUPPORTED;
    const long long P = (long long)H * W;
    if (P > (1LL << 30) || B > (1LL << 40) / P / C) return SLIDE_ATTN_ERR_UNSUPPORTED;
    return group_norm_workspace(B, P, C, groups, dtype, backward ? 2 : 1, workspace) ? SLIDE_ATTN_OK : SLIDE_ATTN_ERR_UNSUPPORTED;
}

bool known_activation(slide_attn_activation a) { return a == SLIDE_ATTN_ACT_NONE || a == SLIDE_ATTN_ACT_SILU || a == SLIDE_ATTN_ACT_GELU; }

slide_attn_status sparse_shape(int B, int H, int W, int heads, int head_dim, int block_h, int block_w, sparse::Geometry* g) {
    if (B < 1 || H < 1 || W < 1 || heads < 1 || head_dim < 1 || block_h < 1 || block_w < 1) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (head_dim != 16 && head_dim != 32 && head_dim != 64) return SLIDE_ATTN_ERR_UNSUPPORTED;
    if (heads >= (1 << 29) / head_dim) return SLIDE_ATTN_ERR_UNSUPPORTED;       // the kernels count a pixel's bytes in 31 bits
    if (block_h > sparse::kMaxEdge || block_w > sparse::kMaxEdge) return SLIDE_ATTN_ERR_UNSUPPORTED;
    const long long across = ((long long)W + block_w - 1) / block_w, down = ((long long)H + block_h - 1) / block_h;
    if (across > sparse::kMaxBlocks || down > sparse::kMaxBlocks || across * down > sparse::kMaxBlocks) return SLIDE_ATTN_ERR_UNSUPPORTED;
    g->H = H; g->W = W; g->heads = heads; g->bh = block_h; g->bw = block_w;
    g->across = (int)across; g->blocks = (int)(across * down); g->top = 0;
    g->tiles = (block_h * block_w + sparse::kRows - 1) / sparse::kRows;
    // the CTAs of one image and head (also a bound for those that pool and rank), times those of the batch, in a grid's first dimension
    if ((long long)B * heads > (1LL << 30) / ((long long)g->blocks * g->tiles)) return SLIDE_ATTN_ERR_UNSUPPORTED;
    return SLIDE_ATTN_OK;
}

// The threads that pool are counted in 31 bits.
bool poolable(const sparse::Geometry& g, long long B, int head_dim) { return B * g.heads * g.blocks < (1LL << 31) / (head_dim / 4); }

size_t map_bytes(const sparse::Geometry& g, int B, int head_dim, slide_attn_dtype t) { return (size_t)B * g.H * g.W * g.heads * head_dim * size_of(t); }
size_t lse_bytes(const sparse::Geometry& g, int B) { return (size_t)B * g.H * g.W * g.heads * sizeof(float); }
// Two floats a query, a counter, and the lists turned round.
size_t backward_bytes(const sparse::Geometry& g, int B) {
    return 2 * lse_bytes(g, B) + sizeof(int) * (1 + (size_t)B * g.heads * (g.blocks + 1 + (size_t)g.blocks * g.top));
}
size_t list_bytes(const sparse::Geometry& g, int B) { return (size_t)B * g.heads * g.blocks * g.top * sizeof(int); }
size_t pooled_bytes(const sparse::Geometry& g, int B, int head_dim) { return 2 * (size_t)B * g.heads * g.blocks * head_dim * sizeof(double); }

slide_attn_status with_top(sparse::Geometry* g, int top) {
    if (top < 1) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (top > sparse::kMaxTop) return SLIDE_ATTN_ERR_UNSUPPORTED;
    g->top = top;
    return SLIDE_ATTN_OK;
}

}  // namespace

extern "C" {

slide_attn_status slide_attn_group_norm_workspace(int B, int H, int W, int C, int groups, slide_attn_dtype dtype, int backward, size_t* bytes)
{
    if (!bytes) return SLIDE_ATTN_ERR_INVALID_ARG;
    size_t need = 0;
    const slide_attn_status st = norm_shape(B, H, W, C, groups, dtype, backward != 0, &need);
    if (st == SLIDE_ATTN_OK) *bytes = need;
    return st;
}

slide_attn_status slide_attn_group_norm_forward(const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, int B, int H,
                                                int W, int C, int groups, float eps, slide_attn_activation act, slide_attn_dtype dtype,
                                                void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (any_null(x, static_cast<const void*>(y), static_cast<const void*>(mean), static_cast<const void*>(rstd))) return SLIDE_ATTN_ERR_INVALID_ARG;
    size_t need = 0;
    slide_attn_status st = norm_shape(B, H, W, C, groups, dtype, false, &need);
    if (st != SLIDE_ATTN_OK) return st;
    if (!known_activation(act) || !(eps >= 0.0f) || isinf(eps) || workspace_bytes < need || (need && !workspace)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (any_misaligned(x, gamma, beta, y, mean, rstd, workspace)) return SLIDE_ATTN_ERR_ALIGNMENT;
    const size_t map = (size_t)B * H * W * C * size_of(dtype), weights = (size_t)C * sizeof(float), moments = (size_t)B * groups * sizeof(float);
    const Span sx(x, map), sg(gamma, weights), sb(beta, weights), sy(y, map), sm(mean, moments), sr(rstd, moments), sw(workspace, need);
    if (meets(sy, sx, sg, sb, sm, sr, sw) || meets(sm, sx, sg, sb, sr, sw) || meets(sr, sx, sg, sb, sw) || meets(sw, sx, sg, sb))
        return SLIDE_ATTN_ERR_INVALID_ARG;
    int sms = 0;
    st = current_device(&sms);
    if (st != SLIDE_ATTN_OK) return st;
    return launched(launch_group_norm_forward(x, gamma, beta, B, (long long)H * W, C, groups, eps, act, dtype, y, mean, rstd, workspace,
                                              static_cast<cudaStream_t>(cuda_stream)));
}

slide_attn_status slide_attn_group_norm_backward(const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd,
                                                 const void* dy, void* dx, float* dgamma, float* dbeta, int B, int H, int W, int C, int groups,
                                                 slide_attn_activation act, slide_attn_dtype dtype, void* workspace, size_t workspace_bytes,
                                                 void* cuda_stream)
{
    if (any_null(x, static_cast<const void*>(mean), static_cast<const void*>(rstd), dy, static_cast<const void*>(dx), static_cast<const void*>(workspace)))
        return SLIDE_ATTN_ERR_INVALID_ARG;
    if ((dgamma == nullptr) != (dbeta == nullptr)) return SLIDE_ATTN_ERR_INVALID_ARG;
    size_t need = 0;
    slide_attn_status st = norm_shape(B, H, W, C, groups, dtype, true, &need);
    if (st != SLIDE_ATTN_OK) return st;
    if (!known_activation(act) || workspace_bytes < need) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (any_misaligned(x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, workspace)) return SLIDE_ATTN_ERR_ALIGNMENT;
    const size_t map = (size_t)B * H * W * C * size_of(dtype), weights = (size_t)C * sizeof(float), moments = (size_t)B * groups * sizeof(float);
    const Span sx(x, map), sg(gamma, weights), sb(beta, weights), sm(mean, moments), sr(rstd, moments), sy(dy, map), so(dx, map), sdg(dgamma, weights),
        sdb(dbeta, weights), sw(workspace, need);
    for (const Span& o : {so, sdg, sdb, sw})
        if (meets(o, sx, sg, sb, sm, sr, sy)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (meets(so, sdg, sdb, sw) || meets(sdg, sdb, sw) || meets(sdb, sw)) return SLIDE_ATTN_ERR_INVALID_ARG;
    int sms = 0;
    st = current_device(&sms);
    if (st != SLIDE_ATTN_OK) return st;
    return launched(launch_group_norm_backward(x, gamma, beta, mean, rstd, dy, B, (long long)H * W, C, groups, act, dtype, dx, dgamma, dbeta,
                                               workspace, static_cast<cudaStream_t>(cuda_stream)));
}

namespace {

slide_attn_status dropout(const void* x, const void* residual, void* y, long long images, long long per_image, float p, slide_attn_drop_unit unit,
                          const void* rng, slide_attn_dtype dtype, void* cuda_stream) {
    if (any_null(x, static_cast<const void*>(y), rng)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (images < 1 || per_image < 1 || !known_dtype(dtype) || (unit != SLIDE_ATTN_DROP_ELEMENTS && unit != SLIDE_ATTN_DROP_IMAGES))
        return SLIDE_ATTN_ERR_INVALID_ARG;
    if (!(p >= 0.0f && p <= 1.0f)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (per_image > (1LL << 40) / images || !dropout_supports(images, per_image, unit == SLIDE_ATTN_DROP_IMAGES)) return SLIDE_ATTN_ERR_UNSUPPORTED;
    if (any_misaligned(x, residual, y) || misaligned(rng, 8)) return SLIDE_ATTN_ERR_ALIGNMENT;
    const size_t map = (size_t)images * per_image * size_of(dtype);
    const Span sy(y, map);
    if ((y != x && meets(sy, Span(x, map))) || (y != residual && meets(sy, Span(residual, map))) || meets(sy, Span(rng, 16)))
        return SLIDE_ATTN_ERR_INVALID_ARG;
    int sms = 0;
    const slide_attn_status st = current_device(&sms);
    if (st != SLIDE_ATTN_OK) return st;
    return launched(launch_dropout(x, residual, y, images, per_image, p, unit == SLIDE_ATTN_DROP_IMAGES,
                                   static_cast<const unsigned long long*>(rng), dtype, sms, static_cast<cudaStream_t>(cuda_stream)));
}

}  // namespace

slide_attn_status slide_attn_dropout_forward(const void* x, const void* residual, void* y, long long images, long long per_image, float p,
                                             slide_attn_drop_unit unit, const void* rng, slide_attn_dtype dtype, void* cuda_stream)
{
    return dropout(x, residual, y, images, per_image, p, unit, rng, dtype, cuda_stream);
}

slide_attn_status slide_attn_dropout_backward(const void* dy, void* dx, long long images, long long per_image, float p, slide_attn_drop_unit unit,
                                              const void* rng, slide_attn_dtype dtype, void* cuda_stream)
{
    return dropout(dy, nullptr, dx, images, per_image, p, unit, rng, dtype, cuda_stream);
}

slide_attn_status slide_attn_select_workspace(int B, int H, int W, int heads, int head_dim, int block_h, int block_w, size_t* bytes)
{
    if (!bytes) return SLIDE_ATTN_ERR_INVALID_ARG;
    sparse::Geometry g;
    const slide_attn_status st = sparse_shape(B, H, W, heads, head_dim, block_h, block_w, &g);
    if (st == SLIDE_ATTN_OK && !poolable(g, B, head_dim)) return SLIDE_ATTN_ERR_UNSUPPORTED;
    if (st == SLIDE_ATTN_OK) *bytes = pooled_bytes(g, B, head_dim);
    return st;
}

slide_attn_status slide_attn_select_blocks(const void* q, const void* k, int* idx, int B, int H, int W, int heads, int head_dim, int block_h,
                                           int block_w, int top, slide_attn_dtype dtype, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (any_null(q, k, static_cast<const void*>(idx), static_cast<const void*>(workspace)) || !known_dtype(dtype)) return SLIDE_ATTN_ERR_INVALID_ARG;
    sparse::Geometry g;
    slide_attn_status st = sparse_shape(B, H, W, heads, head_dim, block_h, block_w, &g);
    if (st == SLIDE_ATTN_OK) st = with_top(&g, top);
    if (st != SLIDE_ATTN_OK) return st;
    if (!poolable(g, B, head_dim)) return SLIDE_ATTN_ERR_UNSUPPORTED;
    if (top > g.blocks || workspace_bytes < pooled_bytes(g, B, head_dim)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (any_misaligned(q, k, idx, workspace)) return SLIDE_ATTN_ERR_ALIGNMENT;
    const size_t map = map_bytes(g, B, head_dim, dtype);
    const Span sq(q, map), sk(k, map), si(idx, list_bytes(g, B)), sw(workspace, pooled_bytes(g, B, head_dim));
    if (meets(si, sq, sk, sw) || meets(sw, sq, sk)) return SLIDE_ATTN_ERR_INVALID_ARG;
    int sms = 0;
    st = current_device(&sms);
    if (st != SLIDE_ATTN_OK) return st;
    return launched(launch_select(g, B, head_dim, dtype, q, k, static_cast<double*>(workspace), idx, sms, static_cast<cudaStream_t>(cuda_stream)));
}

slide_attn_status slide_attn_sparse_forward(const void* q, const void* k, const void* v, const int* idx, void* out, float* lse, int B, int H, int W,
                                            int heads, int head_dim, int block_h, int block_w, int top, slide_attn_dtype dtype, void* cuda_stream)
{
    if (any_null(q, k, v, static_cast<const void*>(idx), static_cast<const void*>(out), static_cast<const void*>(lse)) || !known_dtype(dtype))
        return SLIDE_ATTN_ERR_INVALID_ARG;
    sparse::Geometry g;
    slide_attn_status st = sparse_shape(B, H, W, heads, head_dim, block_h, block_w, &g);
    if (st == SLIDE_ATTN_OK) st = with_top(&g, top);
    if (st != SLIDE_ATTN_OK) return st;
    if (any_misaligned(q, k, v, idx, out, lse)) return SLIDE_ATTN_ERR_ALIGNMENT;
    const size_t map = map_bytes(g, B, head_dim, dtype);
    const Span sq(q, map), sk(k, map), sv(v, map), si(idx, list_bytes(g, B)), so(out, map), sl(lse, lse_bytes(g, B));
    if (meets(so, sq, sk, sv, si, sl) || meets(sl, sq, sk, sv, si)) return SLIDE_ATTN_ERR_INVALID_ARG;
    int sms = 0;
    st = current_device(&sms);
    if (st != SLIDE_ATTN_OK) return st;
    return launched(launch_sparse_forward(g, B, head_dim, dtype, q, k, v, idx, out, lse, sms, static_cast<cudaStream_t>(cuda_stream)));
}

slide_attn_status slide_attn_sparse_workspace(int B, int H, int W, int heads, int head_dim, int block_h, int block_w, int top, size_t* bytes)
{
    if (!bytes) return SLIDE_ATTN_ERR_INVALID_ARG;
    sparse::Geometry g;
    slide_attn_status st = sparse_shape(B, H, W, heads, head_dim, block_h, block_w, &g);
    if (st == SLIDE_ATTN_OK) st = with_top(&g, top);
    if (st == SLIDE_ATTN_OK) *bytes = backward_bytes(g, B);
    return st;
}

slide_attn_status slide_attn_sparse_backward(const void* q, const void* k, const void* v, const int* idx, const void* out, const float* lse,
                                             const void* dout, void* dq, void* dk, void* dv, int B, int H, int W, int heads, int head_dim, int block_h,
                                             int block_w, int top, slide_attn_dtype dtype, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (any_null(q, k, v, static_cast<const void*>(idx), out, static_cast<const void*>(lse), dout, static_cast<const void*>(dq),
                 static_cast<const void*>(dk), static_cast<const void*>(dv), static_cast<const void*>(workspace)) ||
        !known_dtype(dtype))
        return SLIDE_ATTN_ERR_INVALID_ARG;
    sparse::Geometry g;
    slide_attn_status st = sparse_shape(B, H, W, heads, head_dim, block_h, block_w, &g);
    if (st == SLIDE_ATTN_OK) st = with_top(&g, top);
    if (st != SLIDE_ATTN_OK) return st;
    if (workspace_bytes < backward_bytes(g, B)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (any_misaligned(q, k, v, idx, out, lse, dout, dq, dk, dv) || misaligned(workspace)) return SLIDE_ATTN_ERR_ALIGNMENT;
    const size_t map = map_bytes(g, B, head_dim, dtype);
    const Span sq(q, map), sk(k, map), sv(v, map), si(idx, list_bytes(g, B)), so(out, map), sl(lse, lse_bytes(g, B)), sd(dout, map), sdq(dq, map),
        sdk(dk, map), sdv(dv, map), sw(workspace, backward_bytes(g, B));
    for (const Span& o : {sdq, sdk, sdv, sw})
        if (meets(o, sq, sk, sv, si, so, sl, sd)) return SLIDE_ATTN_ERR_INVALID_ARG;
    if (meets(sdq, sdk, sdv, sw) || meets(sdk, sdv, sw) || meets(sdv, sw)) return SLIDE_ATTN_ERR_INVALID_ARG;
    int sms = 0;
    st = current_device(&sms);
    if (st != SLIDE_ATTN_OK) return st;
    const sparse::BackwardMaps m = {q, k, v, idx, out, lse, dout, dq, dk, dv};
    return launched(launch_sparse_backward(g, B, head_dim, dtype, m, workspace, sms, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
