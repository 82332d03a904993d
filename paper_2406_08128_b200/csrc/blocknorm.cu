// The junction of two blocks: gate, norm and scale of one block's output, residual addition, norm before the next block,
// in one pass over each row, and its backward pass.  Per row
//   v = y act(g) | y,  n = Norm(v) w_post + b_post,  m = n | n act(g),  r' = res + scale m,  o = Norm(r') w_pre + b_pre.
//
// Bound by HBM: every operand is read once and every result written once; rows stay in registers between the two norms.
// A lane holds 8 consecutive channels a vector (16 bytes of bf16), WPR warps share a row; sums over a row are fp32
// shuffles and, for WPR > 1, one exchange through shared memory.  Layer statistics are two-pass (mean first) on the
// registers, so a large mean costs no digits.
#include "packed.cuh"

namespace chela {
namespace {

struct NormParams {
    const void *res, *y, *gate;
    long long rs, ys, gs;
    const float *w_post, *b_post, *scale, *w_pre, *b_pre;
    int T, D, gate_act, gate_after, norm_post, norm_pre;
    float eps;
    void *res_out, *o;
};

struct Vec8 {
    float v[8];
};
template <typename T>
__device__ __forceinline__ Vec8 load8(const T *p)
{
    const float4 a = load4(p), b = load4(p + 4);
    return Vec8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
template <>
__device__ __forceinline__ Vec8 load8<__nv_bfloat16>(const __nv_bfloat16 *p)
{
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    Vec8 r;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.v[2 * i] = __uint_as_float(w[i] << 16);
        r.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    return r;
}
__device__ __forceinline__ void store8(float *p, const Vec8 &v)
{
    store4(p, make_float4(v.v[0], v.v[1], v.v[2], v.v[3]));
    store4(p + 4, make_float4(v.v[4], v.v[5], v.v[6], v.v[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const Vec8 &v)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.v[2 * i], v.v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ Vec8 fill8(float a) { return Vec8{{a, a, a, a, a, a, a, a}}; }
__device__ __forceinline__ Vec8 opt8(const float *p, int c, float other) { return p ? load8(p + c) : fill8(other); }

__device__ __forceinline__ float act_f(float u, int act) { return act == 0 ? u : (act == 1 ? u * sigmoid_acc(u) : sigmoid_acc(u)); }
__device__ __forceinline__ float d_act_f(float u, int act)
{
    if (act == 0) return 1.f;
    const float s = sigmoid_acc(u);
    return act == 1 ? s * fmaf(u, 1.f - s, 1.f) : s * (1.f - s);
}

// Sum of K values over the lanes of a row (WPR warps); every lane gets the result.  `buf` holds 2 x WPR x K floats per
// row group, the halves used in turn so that one barrier per sum is enough.
template <int WPR, int K>
struct RowSum {
    float *buf;
    int parity, group, wr, lane;
    __device__ __forceinline__ void operator()(float (&v)[K])
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        if (WPR > 1) {
            float *b = buf + (group * 2 + parity) * WPR * K;
            parity ^= 1;
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) b[wr * K + k] = v[k];
            }
            asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(WPR * 32) : "memory");
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < WPR; ++w) t += b[w * K + k];
                v[k] = t;
            }
        }
    }
};

// ------------------------------------------------------------------------------------------------ forward

template <typename TI, typename TR, typename TO, int WPR, int VPT>
__global__ void __launch_bounds__(WPR > 8 ? 32 * WPR : 256) blocknorm_fwd_kernel(const NormParams p)
{
    constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
    __shared__ float buf[GROUPS * 2 * WPR];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp / WPR, wr = warp % WPR;
    RowSum<WPR, 1> sum = {buf, 0, group, wr, lane};
    const float inv_d = 1.f / p.D;

    for (long long row = (long long)blockIdx.x * GROUPS + group; row < p.T; row += (long long)gridDim.x * GROUPS) {
        Vec8 r[VPT];
        auto col = [&](int k) { return 8 * ((k * WPR + wr) * 32 + lane); };
        auto normalise = [&](Vec8 (&x)[VPT], int kind) {
            if (kind == CHELA_NORM_NONE) return;
            float s[1];
            if (kind == CHELA_NORM_LAYER) {
                s[0] = 0.f;
#pragma unroll
                for (int k = 0; k < VPT; ++k)
                    if (col(k) < p.D)
#pragma unroll
                        for (int e = 0; e < 8; ++e) s[0] += x[k].v[e];
                sum(s);
                const float mean = s[0] * inv_d;
#pragma unroll
                for (int k = 0; k < VPT; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[k].v[e] -= mean;
            }
            s[0] = 0.f;
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (col(k) < p.D)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[0] = fmaf(x[k].v[e], x[k].v[e], s[0]);
            sum(s);
            const float inv = 1.0f / sqrtf(fmaf(s[0], inv_d, p.eps));
#pragma unroll
            for (int k = 0; k < VPT; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k].v[e] *= inv;
        };

#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            r[k] = fill8(0.f);
            if (p.res && col(k) < p.D) r[k] = load8(static_cast<const TR *>(p.res) + (size_t)row * p.rs + col(k));
        }
        if (p.y) {
            Vec8 v[VPT], g[VPT];
#pragma unroll
            for (int k = 0; k < VPT; ++k) {
                v[k] = fill8(0.f);
                g[k] = fill8(1.f);
                if (col(k) < p.D) {
                    v[k] = load8(static_cast<const TI *>(p.y) + (size_t)row * p.ys + col(k));
                    if (p.gate) {
                        g[k] = load8(static_cast<const TI *>(p.gate) + (size_t)row * p.gs + col(k));
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            g[k].v[e] = act_f(g[k].v[e], p.gate_act);
                            if (!p.gate_after) v[k].v[e] *= g[k].v[e];
                        }
                    }
                }
            }
            normalise(v, p.norm_post);
#pragma unroll
            for (int k = 0; k < VPT; ++k) {
                if (col(k) < p.D) {
                    const Vec8 w = opt8(p.w_post, col(k), 1.f), b = opt8(p.b_post, col(k), 0.f), s = opt8(p.scale, col(k), 1.f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float m = fmaf(v[k].v[e], w.v[e], b.v[e]);
                        if (p.gate && p.gate_after) m *= g[k].v[e];
                        r[k].v[e] = fmaf(s.v[e], m, r[k].v[e]);
                    }
                    if (p.res_out) store8(static_cast<TR *>(p.res_out) + (size_t)row * p.D + col(k), r[k]);
                }
            }
        }
        if (p.o) {
            normalise(r, p.norm_pre);
#pragma unroll
            for (int k = 0; k < VPT; ++k) {
                if (col(k) < p.D) {
                    const Vec8 w = opt8(p.w_pre, col(k), 1.f), b = opt8(p.b_pre, col(k), 0.f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[k].v[e] = fmaf(r[k].v[e], w.v[e], b.v[e]);
                    store8(static_cast<TO *>(p.o) + (size_t)row * p.D + col(k), r[k]);
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ backward

struct NormBwdParams {
    NormParams f;   // res = r'
    const void *d_o, *d_ro;
    void *d_res, *d_y, *d_gate;
    float *part;    // [row groups of the grid][5][D]: w_post, b_post, scale, w_pre, b_pre
};

// One vector of 8 channels a lane, so that the five parameter gradients of its channels (40 registers) stay in registers
// over all rows the group walks; D <= 256 WPR.
template <typename TI, typename TR, typename TG, int WPR>
__global__ void __launch_bounds__(WPR > 8 ? 32 * WPR : 256, 1) blocknorm_bwd_kernel(const NormBwdParams q)
{
    constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
    const NormParams &p = q.f;
    __shared__ float buf[GROUPS * 2 * WPR * 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp / WPR, wr = warp % WPR;
    RowSum<WPR, 2> sum = {buf, 0, group, wr, lane};
    const float inv_d = 1.f / p.D;
    const int c = 8 * (wr * 32 + lane);
    const bool live = c < p.D;
    Vec8 acc[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) acc[k] = fill8(0.f);
    const bool post = p.y != nullptr, pre = q.d_o != nullptr;

    for (long long row = (long long)blockIdx.x * GROUPS + group; row < p.T; row += (long long)gridDim.x * GROUPS) {
        Vec8 hat = fill8(0.f), v = fill8(0.f), y = fill8(0.f), gr = fill8(0.f), ga = fill8(1.f), d_o = fill8(0.f), d_r = fill8(0.f);
        if (live) {
            if (q.d_ro) d_r = load8(static_cast<const TR *>(q.d_ro) + (size_t)row * p.D + c);
            if (pre) {
                d_o = load8(static_cast<const TI *>(q.d_o) + (size_t)row * p.D + c);
                hat = load8(static_cast<const TR *>(p.res) + (size_t)row * p.rs + c);
            }
            if (post) {
                y = load8(static_cast<const TI *>(p.y) + (size_t)row * p.ys + c);
                if (p.gate) {
                    gr = load8(static_cast<const TI *>(p.gate) + (size_t)row * p.gs + c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) ga.v[e] = act_f(gr.v[e], p.gate_act);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v.v[e] = p.gate_after ? y.v[e] : y.v[e] * ga.v[e];
            }
        }
        // statistics of both norms together: [0] = r', [1] = v
        float s[2];
        const bool l0 = pre && p.norm_pre == CHELA_NORM_LAYER, l1 = post && p.norm_post == CHELA_NORM_LAYER;
        if (l0 || l1) {
            s[0] = s[1] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[0] += hat.v[e];
                s[1] += v.v[e];
            }
            sum(s);
            const float m0 = l0 && live ? s[0] * inv_d : 0.f, m1 = l1 && live ? s[1] * inv_d : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                hat.v[e] -= m0;
                v.v[e] -= m1;
            }
        }
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[0] = fmaf(hat.v[e], hat.v[e], s[0]);
            s[1] = fmaf(v.v[e], v.v[e], s[1]);
        }
        sum(s);
        const float i0 = p.norm_pre == CHELA_NORM_NONE ? 1.f : 1.0f / sqrtf(fmaf(s[0], inv_d, p.eps));
        const float i1 = p.norm_post == CHELA_NORM_NONE ? 1.f : 1.0f / sqrtf(fmaf(s[1], inv_d, p.eps));
        // norm before the next block: d hat, then d r'
        if (pre) {
            Vec8 dh = fill8(0.f);
            s[0] = s[1] = 0.f;
            const Vec8 w = live ? opt8(p.w_pre, c, 1.f) : fill8(0.f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                hat.v[e] *= i0;
                acc[3].v[e] = fmaf(d_o.v[e], hat.v[e], acc[3].v[e]);
                acc[4].v[e] += d_o.v[e];
                dh.v[e] = d_o.v[e] * w.v[e];
                s[0] = fmaf(dh.v[e], hat.v[e], s[0]);
                s[1] += dh.v[e];
            }
            if (p.norm_pre != CHELA_NORM_NONE) {
                sum(s);
                const float k0 = s[0] * inv_d, k1 = l0 ? s[1] * inv_d : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) d_r.v[e] = fmaf(i0, fmaf(-hat.v[e], k0, dh.v[e]) - k1, d_r.v[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) d_r.v[e] += dh.v[e];
            }
        }
        if (live) store8(static_cast<TR *>(q.d_res) + (size_t)row * p.D + c, d_r);
        if (post) {
            Vec8 dn = fill8(0.f), dm = fill8(0.f), n = fill8(0.f);
            s[0] = s[1] = 0.f;
            if (live) {
                const Vec8 w = opt8(p.w_post, c, 1.f), b = opt8(p.b_post, c, 0.f), sc = opt8(p.scale, c, 1.f);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v.v[e] *= i1;
                    n.v[e] = fmaf(v.v[e], w.v[e], b.v[e]);
                    dm.v[e] = d_r.v[e] * sc.v[e];
                    const float after = p.gate_after ? ga.v[e] : 1.f;
                    acc[2].v[e] = fmaf(d_r.v[e], n.v[e] * after, acc[2].v[e]);
                    const float d_n = dm.v[e] * after;
                    acc[0].v[e] = fmaf(d_n, v.v[e], acc[0].v[e]);
                    acc[1].v[e] += d_n;
                    dn.v[e] = d_n * w.v[e];
                    s[0] = fmaf(dn.v[e], v.v[e], s[0]);
                    s[1] += dn.v[e];
                }
            }
            if (p.norm_post != CHELA_NORM_NONE) {
                sum(s);
                const float k0 = s[0] * inv_d, k1 = l1 ? s[1] * inv_d : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) dn.v[e] = i1 * (fmaf(-v.v[e], k0, dn.v[e]) - k1);
            }
            if (live) {
                Vec8 out;
#pragma unroll
                for (int e = 0; e < 8; ++e) out.v[e] = p.gate_after ? dn.v[e] : dn.v[e] * ga.v[e];
                store8(static_cast<TG *>(q.d_y) + (size_t)row * p.D + c, out);
                if (p.gate) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        out.v[e] = (p.gate_after ? dm.v[e] * n.v[e] : dn.v[e] * y.v[e]) * d_act_f(gr.v[e], p.gate_act);
                    store8(static_cast<TG *>(q.d_gate) + (size_t)row * p.D + c, out);
                }
            }
        }
    }
    if (live) {
        float *o = q.part + ((size_t)blockIdx.x * GROUPS + group) * 5 * p.D + c;
#pragma unroll
        for (int k = 0; k < 5; ++k) store8(o + (size_t)k * p.D, acc[k]);
    }
}

struct NormSums {
    float *out[5];
};
// sums over the row groups in two fixed steps: 8 warps take every eighth partial, then meet in shared memory
__global__ void __launch_bounds__(256) blocknorm_sum_kernel(const float *part, NormSums sums, int nparts, int D)
{
    __shared__ float red[8][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, k = blockIdx.y;
    if (!sums.out[k]) return;
    float o = 0.f;
    if (c < D)
        for (int i = warp; i < nparts; i += 8) o += part[((size_t)i * 5 + k) * D + c];
    red[warp][lane] = o;
    __syncthreads();
    if (warp == 0 && c < D) {
        o = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) o += red[w][lane];
        sums.out[k][c] = o;
    }
}

template <typename TI, typename TR, typename TO>
chela_status_t fwd_d(const NormParams &p, cudaStream_t stream)
{
#define CHELA_NORM_FWD(WPR, VPT)                                                                                   \
    do {                                                                                                           \
        constexpr int groups = WPR > 8 ? 1 : 8 / WPR;                                                              \
        const long long need = ((long long)p.T + groups - 1) / groups;                                             \
        const unsigned grid = (unsigned)(need < 148 * 64 ? need : 148 * 64);                                       \
        blocknorm_fwd_kernel<TI, TR, TO, WPR, VPT><<<grid, WPR > 8 ? 32 * WPR : 256, 0, stream>>>(p);              \
    } while (0)
    if (p.D <= 256) CHELA_NORM_FWD(1, 1);
    else if (p.D <= 512) CHELA_NORM_FWD(1, 2);
    else if (p.D <= 1024) CHELA_NORM_FWD(2, 2);
    else if (p.D <= 2048) CHELA_NORM_FWD(4, 2);
    else if (p.D <= 4096) CHELA_NORM_FWD(8, 2);
    else CHELA_NORM_FWD(16, 2);
#undef CHELA_NORM_FWD
    return last_launch_status();
}

int bwd_wpr(int D)
{
    int w = 1;
    while (w * 256 < D) w <<= 1;
    return w;
}
int bwd_groups(int wpr) { return wpr > 8 ? 1 : 8 / wpr; }
int bwd_grid(int T, int D)
{
    const int g = bwd_groups(bwd_wpr(D)), need = (int)(((long long)T + g - 1) / g);
    return need < 148 * 4 ? need : 148 * 4;
}

template <typename TI, typename TR, typename TG>
chela_status_t bwd_d(const NormBwdParams &q, const NormSums &sums, cudaStream_t stream)
{
    const NormParams &p = q.f;
    const int wpr = bwd_wpr(p.D), grid = bwd_grid(p.T, p.D);
    switch (wpr) {
    case 1: blocknorm_bwd_kernel<TI, TR, TG, 1><<<grid, 256, 0, stream>>>(q); break;
    case 2: blocknorm_bwd_kernel<TI, TR, TG, 2><<<grid, 256, 0, stream>>>(q); break;
    case 4: blocknorm_bwd_kernel<TI, TR, TG, 4><<<grid, 256, 0, stream>>>(q); break;
    case 8: blocknorm_bwd_kernel<TI, TR, TG, 8><<<grid, 256, 0, stream>>>(q); break;
    case 16: blocknorm_bwd_kernel<TI, TR, TG, 16><<<grid, 512, 0, stream>>>(q); break;
    default: blocknorm_bwd_kernel<TI, TR, TG, 32><<<grid, 1024, 0, stream>>>(q); break;
    }
    chela_status_t st = last_launch_status();
    bool any = false;
    for (int k = 0; k < 5; ++k) any = any || sums.out[k];
    if (st == CHELA_OK && any) {
        blocknorm_sum_kernel<<<dim3((p.D + 31) / 32, 5), 256, 0, stream>>>(q.part, sums, grid * bwd_groups(wpr), p.D);
        st = last_launch_status();
    }
    return st;
}

NormParams norm_params(const chela_blocknorm_args_t &a)
{
    NormParams p = {};
    p.res = a.res; p.y = a.y; p.gate = a.gate;
    p.rs = a.res_stride; p.ys = a.y_stride; p.gs = a.gate_stride;
    p.w_post = a.w_post; p.b_post = a.b_post; p.scale = a.scale; p.w_pre = a.w_pre; p.b_pre = a.b_pre;
    p.T = a.T; p.D = a.D; p.gate_act = a.gate_act; p.gate_after = a.gate_after;
    p.norm_post = a.norm_post; p.norm_pre = a.norm_pre;
    p.eps = a.eps;
    return p;
}

}  // namespace

chela_status_t launch_blocknorm_fwd(const chela_blocknorm_args_t &a, void *res_out, void *o, chela_dtype_t out_dtype, cudaStream_t stream)
{
    using bf = __nv_bfloat16;
    NormParams p = norm_params(a);
    p.res_out = res_out;
    p.o = o;
    const bool i32 = a.in_dtype == CHELA_F32, r32 = a.res_dtype == CHELA_F32, o32 = out_dtype == CHELA_F32;
    if (i32) {
        if (r32) return o32 ? fwd_d<float, float, float>(p, stream) : fwd_d<float, float, bf>(p, stream);
        return o32 ? fwd_d<float, bf, float>(p, stream) : fwd_d<float, bf, bf>(p, stream);
    }
    if (r32) return o32 ? fwd_d<bf, float, float>(p, stream) : fwd_d<bf, float, bf>(p, stream);
    return o32 ? fwd_d<bf, bf, float>(p, stream) : fwd_d<bf, bf, bf>(p, stream);
}

size_t blocknorm_bwd_workspace_bytes(int T, int D)
{
    return align_up((size_t)bwd_grid(T, D) * bwd_groups(bwd_wpr(D)) * 5 * D * sizeof(float), 256);
}

chela_status_t launch_blocknorm_bwd(const chela_blocknorm_args_t &a, const void *d_o, const void *d_res_out, void *d_res, void *d_y,
                                    void *d_gate, float *d_w_post, float *d_b_post, float *d_scale, float *d_w_pre, float *d_b_pre,
                                    chela_dtype_t grad_dtype, void *workspace, cudaStream_t stream)
{
    using bf = __nv_bfloat16;
    NormBwdParams q = {};
    q.f = norm_params(a);
    q.d_o = d_o; q.d_ro = d_res_out;
    q.d_res = d_res; q.d_y = d_y; q.d_gate = d_gate;
    q.part = static_cast<float *>(workspace);
    const NormSums sums = {{d_w_post, d_b_post, d_scale, d_w_pre, d_b_pre}};
    const bool i32 = a.in_dtype == CHELA_F32, r32 = a.res_dtype == CHELA_F32, g32 = grad_dtype == CHELA_F32;
    if (i32) {
        if (r32) return g32 ? bwd_d<float, float, float>(q, sums, stream) : bwd_d<float, float, bf>(q, sums, stream);
        return g32 ? bwd_d<float, bf, float>(q, sums, stream) : bwd_d<float, bf, bf>(q, sums, stream);
    }
    if (r32) return g32 ? bwd_d<bf, float, float>(q, sums, stream) : bwd_d<bf, float, bf>(q, sums, stream);
    return g32 ? bwd_d<bf, bf, float>(q, sums, stream) : bwd_d<bf, bf, bf>(q, sums, stream);
}

}  // namespace chela
