// C ABI entry points of the operators over packed sequences: argument validation and dispatch.  No kernel code here.
#include "common.cuh"

using namespace chela;

namespace {

constexpr int kNormMaxD = 8192;
constexpr int kMaxTokens = 0x7fffffff - 4095;   // token positions and the slices past the last one stay within int
constexpr int kMaxSeqs = 1 << 30;               // and so do the numbers of work items (tokens / 8 + sequences)

bool dtype_ok(chela_dtype_t t) { return t == CHELA_F32 || t == CHELA_BF16; }
// act or softplus: 0 or 1, and the flag
bool switch_ok(int v) { return (v & ~CHELA_ZERO_REST) == 0 || (v & ~CHELA_ZERO_REST) == 1; }
// token stride of an operand whose row has n elements
bool stride_ok(long long stride, long long n) { return stride >= n && stride % 8 == 0; }

chela_status_t check_seqs(const int *seq_offsets, int S, int T)
{
    if (S < 1 || T < 1) return CHELA_ERR_INVALID_ARG;
    if (!seq_offsets && T % S != 0) return CHELA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(seq_offsets) & 3u) return CHELA_ERR_INVALID_ARG;
    return T <= kMaxTokens && S <= kMaxSeqs ? CHELA_OK : CHELA_ERR_UNSUPPORTED;
}

// no output may be an operand's buffer: rows of other strides or types would overlap (a null pointer aliases nothing)
template <size_t A, size_t B>
bool distinct(const void *const (&outs)[A], const void *const (&operands)[B])
{
    for (const void *o : outs)
        for (const void *i : operands)
            if (o && o == i) return false;
    return true;
}

// nor may two outputs share one
template <size_t A>
bool all_different(const void *const (&outs)[A])
{
    for (size_t i = 0; i < A; ++i)
        for (size_t j = 0; j < i; ++j)
            if (outs[i] && outs[i] == outs[j]) return false;
    return true;
}

chela_status_t check_conv(const void *x, long long x_stride, const float *w, const float *bias, const void *state_in,
                          const void *state_out, const int *seq_offsets, int S, int T, int D, int width, int act, chela_dtype_t io_dtype)
{
    if (!x || !w || D < 1 || width < 1 || !dtype_ok(io_dtype) || !switch_ok(act)) return CHELA_ERR_INVALID_ARG;
    const chela_status_t st = check_seqs(seq_offsets, S, T);
    if (st != CHELA_OK) return st;
    if (!aligned16(x) || !aligned16(w) || !aligned16(bias) || !aligned16(state_in) || !aligned16(state_out)) return CHELA_ERR_INVALID_ARG;
    if (width > 16 || D % 8 != 0) return CHELA_ERR_UNSUPPORTED;
    return stride_ok(x_stride, D) ? CHELA_OK : CHELA_ERR_INVALID_ARG;
}

// y and state_out lie in no operand's buffer, but for state_out in state_in's
bool conv_outputs_ok(const void *x, const void *w, const void *bias, const void *y, const void *state_in, const void *state_out,
                     const void *seq_offsets, int width)
{
    if (width == 1) state_in = state_out = nullptr;   // ignored
    return distinct({y, state_out}, {x, w, bias, seq_offsets}) && distinct({y}, {state_in}) && all_different({y, state_out});
}

chela_status_t check_scan(const chela_selscan_args_t *a)
{
    if (!a || !a->x || !a->dt || !a->b || !a->c || !a->a || a->D < 1 || a->N < 1 || a->G < 1 || !dtype_ok(a->in_dtype) ||
        !switch_ok(a->softplus))
        return CHELA_ERR_INVALID_ARG;
    const chela_status_t st = check_seqs(a->seq_offsets, a->S, a->T);
    if (st != CHELA_OK) return st;
    const void *ptrs[] = {a->x, a->dt, a->b, a->c, a->z, a->a, a->d_skip, a->dt_bias, a->state_in};
    for (const void *p : ptrs)
        if (!aligned16(p)) return CHELA_ERR_INVALID_ARG;
    if ((a->N != 8 && a->N != 16 && a->N != 32 && a->N != 64) || a->D % 8 != 0) return CHELA_ERR_UNSUPPORTED;
    if (a->G > 1 && a->D % ((long long)a->G * 32) != 0) return CHELA_ERR_UNSUPPORTED;
    const long long gn = (long long)a->G * a->N;
    if (!stride_ok(a->x_stride, a->D) || !stride_ok(a->dt_stride, a->D) || !stride_ok(a->b_stride, gn) || !stride_ok(a->c_stride, gn) ||
        (a->z && !stride_ok(a->z_stride, a->D)))
        return CHELA_ERR_INVALID_ARG;
    return CHELA_OK;
}

// no output lies in the buffer of an operand other than the state, or in another output's
template <size_t A>
bool scan_outputs_ok(const chela_selscan_args_t &a, const void *const (&outs)[A])
{
    return distinct(outs, {a.x, a.dt, a.b, a.c, a.z, a.a, a.d_skip, a.dt_bias, a.seq_offsets}) && all_different(outs);
}

bool norm_kind_ok(chela_norm_t n) { return n == CHELA_NORM_NONE || n == CHELA_NORM_RMS || n == CHELA_NORM_LAYER; }

chela_status_t check_norm(const chela_blocknorm_args_t *a)
{
    if (!a || a->T < 1 || a->D < 1 || !dtype_ok(a->in_dtype) || !dtype_ok(a->res_dtype) || !norm_kind_ok(a->norm_post) ||
        !norm_kind_ok(a->norm_pre) || !(a->eps >= 0.f) || a->gate_act < 0 || a->gate_act > 2 || (a->gate_after != 0 && a->gate_after != 1))
        return CHELA_ERR_INVALID_ARG;
    if ((!a->res && !a->y) || (a->gate && !a->y)) return CHELA_ERR_INVALID_ARG;
    const void *ptrs[] = {a->res, a->y, a->gate, a->w_post, a->b_post, a->scale, a->w_pre, a->b_pre};
    for (const void *p : ptrs)
        if (!aligned16(p)) return CHELA_ERR_INVALID_ARG;
    if (a->D % 8 != 0 || a->D > kNormMaxD || a->T > kMaxTokens) return CHELA_ERR_UNSUPPORTED;
    if ((a->res && !stride_ok(a->res_stride, a->D)) || (a->y && !stride_ok(a->y_stride, a->D)) ||
        (a->gate && !stride_ok(a->gate_stride, a->D)))
        return CHELA_ERR_INVALID_ARG;
    return CHELA_OK;
}

}  // namespace

extern "C" {

chela_status_t chela_shortconv_carry_fwd(const void *x, long long x_stride, const float *w, const float *bias, void *y,
                                         const void *state_in, void *state_out, const int *seq_offsets, int S, int T, int D,
                                         int width, int act, chela_dtype_t io_dtype, cudaStream_t stream)
{
    const chela_status_t st = check_conv(x, x_stride, w, bias, state_in, state_out, seq_offsets, S, T, D, width, act, io_dtype);
    if (st != CHELA_OK) return st;
    if (!y || y == x || !aligned16(y) || !conv_outputs_ok(x, w, bias, y, state_in, state_out, seq_offsets, width)) return CHELA_ERR_INVALID_ARG;
    return launch_shortconv_carry(x, x_stride, w, bias, y, state_in, state_out, seq_offsets, S, T, D, width, act, io_dtype, stream);
}

chela_status_t chela_shortconv_step(const void *x, long long x_stride, const float *w, const float *bias, void *y,
                                    const void *state_in, void *state_out, int S, int D, int width, int act, chela_dtype_t io_dtype,
                                    cudaStream_t stream)
{
    const chela_status_t st = check_conv(x, x_stride, w, bias, state_in, state_out, nullptr, S, S, D, width, act, io_dtype);
    if (st != CHELA_OK) return st;
    if (!y || y == x || !aligned16(y) || (width > 1 && (!state_in || !state_out)) ||
        !conv_outputs_ok(x, w, bias, y, state_in, state_out, nullptr, width))
        return CHELA_ERR_INVALID_ARG;
    return launch_shortconv_step(x, x_stride, w, bias, y, state_in, state_out, S, D, width, act, io_dtype, stream);
}

size_t chela_shortconv_bwd_workspace_bytes(int T, int D, int width)
{
    if (T < 1 || D < 1 || D % 8 != 0 || width < 1 || width > 16) return 0;
    return shortconv_bwd_workspace_bytes(T, D, width);
}

chela_status_t chela_shortconv_bwd(const void *x, long long x_stride, const float *w, const float *bias, const void *d_y,
                                   long long d_y_stride, const void *state_in, const void *d_state_out, void *d_x, float *d_w,
                                   float *d_bias, void *d_state_in, const int *seq_offsets, int S, int T, int D, int width, int act,
                                   chela_dtype_t io_dtype, chela_dtype_t grad_dtype, void *workspace, size_t workspace_bytes,
                                   cudaStream_t stream)
{
    const chela_status_t st = check_conv(x, x_stride, w, bias, state_in, d_state_out, seq_offsets, S, T, D, width, act, io_dtype);
    if (st != CHELA_OK) return st;
    if (!d_y || !d_x || d_x == x || d_x == d_y || !dtype_ok(grad_dtype) || !stride_ok(d_y_stride, D) || !aligned16(d_y) || !aligned16(d_x) ||
        !aligned16(d_w) || !aligned16(d_bias) || !aligned16(d_state_in) || !aligned16(workspace))
        return CHELA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < shortconv_bwd_workspace_bytes(T, D, width)) return CHELA_ERR_WORKSPACE;
    if (width == 1) state_in = d_state_out = d_state_in = nullptr;   // ignored
    if (!distinct({d_x, d_w, d_bias, d_state_in}, {x, w, bias, d_y, state_in, d_state_out, seq_offsets}) ||
        !all_different({d_x, d_w, d_bias, d_state_in}))
        return CHELA_ERR_INVALID_ARG;
    return launch_shortconv_bwd(x, x_stride, w, bias, d_y, d_y_stride, state_in, d_state_out, d_x, d_w, d_bias, d_state_in, seq_offsets, S,
                                T, D, width, act, io_dtype, grad_dtype, workspace, stream);
}

size_t chela_selscan_checkpoint_bytes(int T, int S, int D, int N)
{
    if (T < 1 || S < 1 || D < 1 || (N != 8 && N != 16 && N != 32 && N != 64)) return 0;
    return selscan_checkpoint_bytes(T, S, D, N);
}

size_t chela_selscan_workspace_bytes(int T, int S, int D, int N)
{
    if (T < 1 || S < 1 || D < 1 || D % 8 != 0 || (N != 8 && N != 16 && N != 32 && N != 64)) return 0;
    return selscan_workspace_bytes(T, S, D, N);
}

chela_status_t chela_selscan_fwd(const chela_selscan_args_t *args, void *y, float *state_out, void *checkpoints,
                                 chela_dtype_t out_dtype, void *workspace, size_t workspace_bytes, cudaStream_t stream)
{
    const chela_status_t st = check_scan(args);
    if (st != CHELA_OK) return st;
    if (!dtype_ok(out_dtype) || (!y && !state_out && !checkpoints) || !aligned16(y) || !aligned16(state_out) || !aligned16(checkpoints) ||
        !aligned16(workspace))
        return CHELA_ERR_INVALID_ARG;
    if (!distinct({y}, {args->x, args->dt, args->b, args->c, args->z})) return CHELA_ERR_INVALID_ARG;
    const size_t need = selscan_workspace_bytes(args->T, args->S, args->D, args->N);
    if (need && (!workspace || workspace_bytes < need)) return CHELA_ERR_WORKSPACE;
    if (!distinct({y, checkpoints}, {args->state_in}) || !scan_outputs_ok(*args, {y, state_out, checkpoints})) return CHELA_ERR_INVALID_ARG;
    return launch_selscan_fwd(*args, y, state_out, checkpoints, out_dtype, workspace, stream);
}

chela_status_t chela_selscan_step(const chela_selscan_args_t *args, void *y, float *state_out, chela_dtype_t out_dtype,
                                  cudaStream_t stream)
{
    const chela_status_t st = check_scan(args);
    if (st != CHELA_OK) return st;
    if (args->T != args->S || args->seq_offsets || !args->state_in || !y || !state_out || !dtype_ok(out_dtype) || !aligned16(y) ||
        !aligned16(state_out) || !distinct({y}, {args->state_in}) || !scan_outputs_ok(*args, {y, state_out}))
        return CHELA_ERR_INVALID_ARG;
    return launch_selscan_step(*args, y, state_out, out_dtype, stream);
}

size_t chela_selscan_bwd_workspace_bytes(int T, int S, int D, int N, int have_checkpoints)
{
    if (T < 1 || S < 1 || D < 1 || D % 8 != 0 || (N != 8 && N != 16 && N != 32 && N != 64)) return 0;
    return selscan_bwd_workspace_bytes(T, S, D, N, have_checkpoints != 0);
}

chela_status_t chela_selscan_bwd(const chela_selscan_args_t *args, const void *d_y, long long d_y_stride, const float *d_state_out,
                                 const void *checkpoints, void *d_x, void *d_dt, float *d_a, void *d_b, void *d_c, float *d_skip_grad,
                                 void *d_z, float *d_dt_bias, float *d_state_in, chela_dtype_t grad_dtype, void *workspace,
                                 size_t workspace_bytes, cudaStream_t stream)
{
    const chela_status_t st = check_scan(args);
    if (st != CHELA_OK) return st;
    if (!d_y || !d_x || !d_dt || !d_a || !d_b || !d_c || (d_z != nullptr) != (args->z != nullptr) || !dtype_ok(grad_dtype) ||
        !stride_ok(d_y_stride, args->D))
        return CHELA_ERR_INVALID_ARG;
    const void *ptrs[] = {d_y, d_state_out, checkpoints, d_x, d_dt, d_a, d_b, d_c, d_skip_grad, d_z, d_dt_bias, d_state_in, workspace};
    for (const void *p : ptrs)
        if (!aligned16(p)) return CHELA_ERR_INVALID_ARG;
    if (!distinct({d_x, d_dt, d_z, d_b, d_c}, {args->x, args->dt, args->z, args->b, args->c, d_y})) return CHELA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < selscan_bwd_workspace_bytes(args->T, args->S, args->D, args->N, checkpoints != nullptr))
        return CHELA_ERR_WORKSPACE;
    if (!scan_outputs_ok(*args, {d_x, d_dt, d_a, d_b, d_c, d_skip_grad, d_z, d_dt_bias, d_state_in}) ||
        !distinct({d_x, d_dt, d_a, d_b, d_c, d_skip_grad, d_z, d_dt_bias, d_state_in}, {args->state_in, d_y, d_state_out, checkpoints}))
        return CHELA_ERR_INVALID_ARG;
    return launch_selscan_bwd(*args, d_y, d_y_stride, d_state_out, checkpoints, d_x, d_dt, d_a, d_b, d_c, d_skip_grad, d_z, d_dt_bias,
                              d_state_in, grad_dtype, workspace, stream);
}

chela_status_t chela_blocknorm_fwd(const chela_blocknorm_args_t *args, void *res_out, void *o, chela_dtype_t out_dtype,
                                   cudaStream_t stream)
{
    const chela_status_t st = check_norm(args);
    if (st != CHELA_OK) return st;
    if (!dtype_ok(out_dtype) || (!res_out && !o) || (res_out && !args->y) || !aligned16(res_out) || !aligned16(o)) return CHELA_ERR_INVALID_ARG;
    if (res_out && (res_out == args->y || res_out == args->gate || res_out == o)) return CHELA_ERR_INVALID_ARG;
    if (res_out && res_out == args->res && args->res_stride != args->D) return CHELA_ERR_INVALID_ARG;   // rows would overlap
    if (o && (o == args->res || o == args->y || o == args->gate)) return CHELA_ERR_INVALID_ARG;
    if (!distinct({res_out, o}, {args->w_post, args->b_post, args->scale, args->w_pre, args->b_pre})) return CHELA_ERR_INVALID_ARG;
    return launch_blocknorm_fwd(*args, res_out, o, out_dtype, stream);
}

size_t chela_blocknorm_bwd_workspace_bytes(int T, int D)
{
    if (T < 1 || D < 1 || D % 8 != 0 || D > kNormMaxD) return 0;
    return blocknorm_bwd_workspace_bytes(T, D);
}

chela_status_t chela_blocknorm_bwd(const chela_blocknorm_args_t *args, const void *d_o, const void *d_res_out, void *d_res, void *d_y,
                                   void *d_gate, float *d_w_post, float *d_b_post, float *d_scale, float *d_w_pre, float *d_b_pre,
                                   chela_dtype_t grad_dtype, void *workspace, size_t workspace_bytes, cudaStream_t stream)
{
    const chela_status_t st = check_norm(args);
    if (st != CHELA_OK) return st;
    if ((!d_o && !d_res_out) || !d_res || (d_y != nullptr) != (args->y != nullptr) || (d_gate != nullptr) != (args->gate != nullptr) ||
        !dtype_ok(grad_dtype) || (d_o && !args->res))
        return CHELA_ERR_INVALID_ARG;
    const void *ptrs[] = {d_o, d_res_out, d_res, d_y, d_gate, d_w_post, d_b_post, d_scale, d_w_pre, d_b_pre, workspace};
    for (const void *p : ptrs)
        if (!aligned16(p)) return CHELA_ERR_INVALID_ARG;
    if (!distinct({d_y, d_gate}, {args->res, args->y, args->gate, d_o, d_res_out}) || !distinct({d_res}, {args->res, args->y, args->gate, d_o}))
        return CHELA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < blocknorm_bwd_workspace_bytes(args->T, args->D)) return CHELA_ERR_WORKSPACE;
    if (!distinct({d_res, d_y, d_gate, d_w_post, d_b_post, d_scale, d_w_pre, d_b_pre},
                  {args->w_post, args->b_post, args->scale, args->w_pre, args->b_pre}) ||
        !distinct({d_w_post, d_b_post, d_scale, d_w_pre, d_b_pre}, {args->res, args->y, args->gate, d_o, d_res_out}) ||
        !all_different({d_res, d_y, d_gate, d_w_post, d_b_post, d_scale, d_w_pre, d_b_pre}))
        return CHELA_ERR_INVALID_ARG;
    return launch_blocknorm_bwd(*args, d_o, d_res_out, d_res, d_y, d_gate, d_w_post, d_b_post, d_scale, d_w_pre, d_b_pre, grad_dtype,
                                workspace, stream);
}

}  // extern "C"
