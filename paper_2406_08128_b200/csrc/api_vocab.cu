// C ABI entry points of the token embedding and the vocabulary's cross entropy: argument validation and dispatch.  No kernel
// code here.
#include <atomic>

#include "common.cuh"

using namespace chela;

namespace {

constexpr int kMaxTokens = 0x7fffffff - 4095;
constexpr long long kMaxStride = 1LL << 36;   // a row's distance in elements: within a tensor map's strides
constexpr int kMaxRows = 1 << 30, kMaxCols = 1 << 20;

constexpr float kMaxScale = 1e30f;            // its product with log2 e stays finite

bool dtype_ok(chela_dtype_t t) { return t == CHELA_F32 || t == CHELA_BF16; }
bool stride_ok(long long stride, long long n) { return stride >= n && stride % 8 == 0 && stride <= kMaxStride; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }   // arrays of one value a token
bool ids_ok(const void *ids, int wide) { return ids && (wide == 0 || wide == 1) && (reinterpret_cast<uintptr_t>(ids) & (wide ? 7u : 3u)) == 0; }

// sizes that both operators take
chela_status_t check_sizes(int T, int V, int D)
{
    if (T < 1 || V < 1 || D < 1) return CHELA_ERR_INVALID_ARG;
    return T <= kMaxTokens && V <= kMaxRows && D <= kMaxCols && D % 8 == 0 ? CHELA_OK : CHELA_ERR_UNSUPPORTED;
}

// the tiles of the logits, 256 tokens by 64 words, are counted in 32 bits
bool loss_sizes_ok(int T, int V) { return (T / 256 + 1LL) * (V / 64 + 1LL) <= 0x7fffffff; }

template <size_t A, size_t B>
bool distinct(const void *const (&outs)[A], const void *const (&operands)[B])
{
    for (const void *o : outs)
        for (const void *i : operands)
            if (o && o == i) return false;
    return true;
}

chela_status_t check_loss(const chela_vocabloss_args_t *a)
{
    if (!a || !a->h || !a->w || !ids_ok(a->targets, a->wide_ids) || !dtype_ok(a->in_dtype) || !aligned16(a->h) || !aligned16(a->w)) return CHELA_ERR_INVALID_ARG;
    const chela_status_t st = check_sizes(a->T, a->V, a->D);
    if (st != CHELA_OK) return st;
    if (!loss_sizes_ok(a->T, a->V)) return CHELA_ERR_UNSUPPORTED;
    return stride_ok(a->h_stride, a->D) && stride_ok(a->w_stride, a->D) && a->scale > 0.f && a->scale <= kMaxScale ? CHELA_OK : CHELA_ERR_INVALID_ARG;
}

bool query_ok(int T, int V, int D) { return check_sizes(T, V, D) == CHELA_OK; }
bool loss_query_ok(int T, int V, int D) { return query_ok(T, V, D) && loss_sizes_ok(T, V); }

}  // namespace

namespace chela {

int current_sm_count()
{
    static std::atomic<int> counts[64];   // of a device, once asked for: it does not change
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 148;
    int n = dev < 64 ? counts[dev].load(std::memory_order_relaxed) : 0;
    if (n > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
    if (dev < 64) counts[dev].store(n, std::memory_order_relaxed);
    return n;
}

}  // namespace chela

extern "C" {

chela_status_t chela_embed_fwd(const void *ids, int wide_ids, const void *w, long long w_stride, void *out, int T, int V, int D, float scale, chela_dtype_t w_dtype,
                               chela_dtype_t out_dtype, cudaStream_t stream)
{
    if (!ids_ok(ids, wide_ids) || !w || !out || !aligned16(w) || !aligned16(out) || !dtype_ok(w_dtype) || !dtype_ok(out_dtype) || out == w || out == ids) return CHELA_ERR_INVALID_ARG;
    const chela_status_t st = check_sizes(T, V, D);
    if (st != CHELA_OK) return st;
    if (!stride_ok(w_stride, D)) return CHELA_ERR_INVALID_ARG;
    return launch_embed_fwd(ids, wide_ids != 0, w, w_stride, out, T, V, D, scale, w_dtype, out_dtype, stream);
}

size_t chela_embed_bwd_workspace_bytes(int T, int V, int D) { return query_ok(T, V, D) ? embed_bwd_workspace_bytes(T, V, D) : 0; }

chela_status_t chela_embed_bwd(const void *ids, int wide_ids, const void *d_out, long long d_out_stride, const void *d_w_in, void *d_w, int T, int V, int D, float scale,
                               chela_dtype_t d_out_dtype, chela_dtype_t grad_dtype, void *workspace, size_t workspace_bytes, cudaStream_t stream)
{
    if (!ids_ok(ids, wide_ids) || !d_out || !d_w || !aligned16(d_out) || !aligned16(d_w) || !aligned16(d_w_in) || !aligned16(workspace) || !dtype_ok(d_out_dtype) || !dtype_ok(grad_dtype))
        return CHELA_ERR_INVALID_ARG;
    const chela_status_t st = check_sizes(T, V, D);
    if (st != CHELA_OK) return st;
    if (!stride_ok(d_out_stride, D) || !distinct({d_w, workspace}, {ids, d_out}) || !distinct({workspace}, {d_w, d_w_in})) return CHELA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < embed_bwd_workspace_bytes(T, V, D)) return CHELA_ERR_WORKSPACE;
    return launch_embed_bwd(ids, wide_ids != 0, d_out, d_out_stride, d_w_in, d_w, T, V, D, scale, d_out_dtype, grad_dtype, workspace, stream);
}

size_t chela_vocabloss_workspace_bytes(int T, int V, int D, chela_dtype_t in_dtype)
{
    return loss_query_ok(T, V, D) && dtype_ok(in_dtype) ? vocabloss_workspace_bytes(T, V, D, in_dtype) : 0;
}

chela_status_t chela_vocabloss_fwd(const chela_vocabloss_args_t *args, float *loss, float *lse, void *workspace, size_t workspace_bytes, cudaStream_t stream)
{
    const chela_status_t st = check_loss(args);
    if (st != CHELA_OK) return st;
    if (!loss || !lse || loss == lse || !aligned4(loss) || !aligned4(lse) || !aligned16(workspace) || !distinct({loss, lse, workspace}, {args->h, args->w, args->targets}) ||
        !distinct({loss, lse}, {workspace}))
        return CHELA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < vocabloss_workspace_bytes(args->T, args->V, args->D, args->in_dtype)) return CHELA_ERR_WORKSPACE;
    return launch_vocabloss_fwd(*args, loss, lse, workspace, stream);
}

size_t chela_vocabloss_bwd_workspace_bytes(int T, int V, int D, chela_dtype_t in_dtype, chela_dtype_t grad_dtype)
{
    return loss_query_ok(T, V, D) && dtype_ok(in_dtype) && dtype_ok(grad_dtype) ? vocabloss_bwd_workspace_bytes(T, V, D, in_dtype, grad_dtype) : 0;
}

chela_status_t chela_vocabloss_bwd(const chela_vocabloss_args_t *args, const float *lse, const float *d_loss, const float *d_lse, void *d_h, const void *d_w_in, void *d_w,
                                   chela_dtype_t grad_dtype, void *workspace, size_t workspace_bytes, cudaStream_t stream)
{
    const chela_status_t st = check_loss(args);
    if (st != CHELA_OK) return st;
    if (!lse || (!d_loss && !d_lse) || !d_h || !d_w || !dtype_ok(grad_dtype) || !aligned4(lse) || !aligned4(d_loss) || !aligned4(d_lse) || !aligned16(d_h) ||
        !aligned16(d_w) || !aligned16(d_w_in) || !aligned16(workspace))
        return CHELA_ERR_INVALID_ARG;
    if (d_h == d_w || !distinct({d_h, d_w, workspace}, {args->h, args->w, args->targets, lse, d_loss, d_lse}) || !distinct({d_h, workspace}, {d_w_in}) ||
        !distinct({workspace}, {d_h, d_w}))
        return CHELA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < vocabloss_bwd_workspace_bytes(args->T, args->V, args->D, args->in_dtype, grad_dtype)) return CHELA_ERR_WORKSPACE;
    return launch_vocabloss_bwd(*args, lse, d_loss, d_lse, d_h, d_w_in, d_w, grad_dtype, workspace, stream);
}

}  // extern "C"
