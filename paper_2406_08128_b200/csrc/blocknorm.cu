// The junction of two blocks: gate, norm and scale of one block's output, residual addition, norm before the next block,
// in one pass over each row, and its backward pass.  Per row
//   v = y act(g) | y,  n = Norm(v) w_post + b_post,  m = n | n act(g),  r' = res + scale m,  o = Norm(r') w_pre + b_pre.
//
// Bound by HBM: every operand is read once and every result written once; rows stay in registers between the two norms.
// A lane holds 8 consecutive channels (16 bytes of bf16), WPR warps share a row; sums over a row are fp32 shuffles and, for
// WPR > 1, one exchange through shared memory.  The next row's operands are loaded while a row is worked on.  Layer
// statistics are two-pass (mean first) on the registers, so a large mean costs no digits.
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
    bool wide;   // all fp32 tensors lie on 32-byte boundaries: 8 values are one access
};

struct Vec8 {
    float v[8];
};
// 8 elements as they lie in memory
template <typename T>
struct Raw8 {
    Raw4<T> lo, hi;
    __device__ __forceinline__ void load(const T *p, bool wide)
    {
        if constexpr (sizeof(T) == 2) {
            const uint4 u = *reinterpret_cast<const uint4 *>(p);
            lo.v = make_uint2(u.x, u.y);
            hi.v = make_uint2(u.z, u.w);
        } else if (wide) {   // a whole sector at once
            asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(lo.v.x), "=f"(lo.v.y), "=f"(lo.v.z), "=f"(lo.v.w), "=f"(hi.v.x), "=f"(hi.v.y), "=f"(hi.v.z), "=f"(hi.v.w)
                         : "l"(p) : "memory");
        } else {
            lo.load(p);
            hi.load(p + 4);
        }
    }
    __device__ __forceinline__ void zero()
    {
        lo.zero();
        hi.zero();
    }
    // from 16-byte vectors `step` vectors apart
    __device__ __forceinline__ void from(const uint4 *p, int step)
    {
        const uint4 u = p[0];
        if constexpr (sizeof(T) == 2) {
            lo.v = make_uint2(u.x, u.y);
            hi.v = make_uint2(u.z, u.w);
        } else {
            const uint4 w = p[step];
            lo.v = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
            hi.v = make_float4(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w));
        }
    }
    __device__ __forceinline__ Vec8 get() const
    {
        const float4 a = lo.get(), b = hi.get();
        return Vec8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
    }
};
__device__ __forceinline__ Vec8 load8(const float *p)
{
    const float4 a = load4(p), b = load4(p + 4);
    return Vec8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ void store8(float *p, const Vec8 &v)
{
    store4(p, make_float4(v.v[0], v.v[1], v.v[2], v.v[3]));
    store4(p + 4, make_float4(v.v[4], v.v[5], v.v[6], v.v[7]));
}
// 8 values to a tensor.  In two stores of 16 bytes each a warp would touch every sector twice, which costs L2 twice the
// requests: forward of 16384 x 2048 in fp32 121 us, in one store (and load) 105.  The backward kernel is not bound by
// them and is 2 % slower with them.
__device__ __forceinline__ void put8(float *p, const Vec8 &v, bool wide)
{
    if (wide)
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v.v[0]), "f"(v.v[1]), "f"(v.v[2]), "f"(v.v[3]),
                     "f"(v.v[4]), "f"(v.v[5]), "f"(v.v[6]), "f"(v.v[7]) : "memory");
    else
        store8(p, v);
}
__device__ __forceinline__ void put8(__nv_bfloat16 *p, const Vec8 &v, bool)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.v[2 * i], v.v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
// elementwise, in pairs: half the instructions
__device__ __forceinline__ Vec8 mul8(const Vec8 &a, const Vec8 &b)
{
    Vec8 o;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float2 t = mul2v(make_float2(a.v[e], a.v[e + 1]), make_float2(b.v[e], b.v[e + 1]));
        o.v[e] = t.x;
        o.v[e + 1] = t.y;
    }
    return o;
}
__device__ __forceinline__ Vec8 add8(const Vec8 &a, const Vec8 &b)
{
    Vec8 o;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float2 t = add2v(make_float2(a.v[e], a.v[e + 1]), make_float2(b.v[e], b.v[e + 1]));
        o.v[e] = t.x;
        o.v[e + 1] = t.y;
    }
    return o;
}
__device__ __forceinline__ Vec8 fma8(const Vec8 &a, const Vec8 &b, const Vec8 &c)
{
    Vec8 o;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float2 t = fma2v(make_float2(a.v[e], a.v[e + 1]), make_float2(b.v[e], b.v[e + 1]), make_float2(c.v[e], c.v[e + 1]));
        o.v[e] = t.x;
        o.v[e + 1] = t.y;
    }
    return o;
}
__device__ __forceinline__ float dot8(const Vec8 &a, const Vec8 &b)
{
    float2 t = mul2v(make_float2(a.v[0], a.v[1]), make_float2(b.v[0], b.v[1]));
#pragma unroll
    for (int e = 2; e < 8; e += 2) t = fma2v(make_float2(a.v[e], a.v[e + 1]), make_float2(b.v[e], b.v[e + 1]), t);
    return t.x + t.y;
}
__device__ __forceinline__ float sum8(const Vec8 &a)
{
    float2 t = make_float2(a.v[0], a.v[1]);
#pragma unroll
    for (int e = 2; e < 8; e += 2) t = add2v(t, make_float2(a.v[e], a.v[e + 1]));
    return t.x + t.y;
}
__device__ __forceinline__ Vec8 fill8(float a) { return Vec8{{a, a, a, a, a, a, a, a}}; }
__device__ __forceinline__ void stage_weight(float *to, const float *from, float other, const float *scale, int D, int width)
{
    // of each warp's 256 channels the even groups of four first, so that 32 lanes read 8 channels each without bank conflicts
    for (int c = threadIdx.x; c < width; c += blockDim.x) to[(c & ~255) + (c & 4) * 32 + (c >> 3 & 31) * 4 + (c & 3)] = (from && c < D ? from[c] : other) * (scale && c < D ? scale[c] : 1.f);
}

__device__ __forceinline__ Vec8 staged8(const float *p)   // of a lane's own vectors
{
    const float4 a = load4(p), b = load4(p + 128);
    return Vec8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

// act(u) in place; act is the same for all threads, so the branch is taken once and not per element
__device__ __forceinline__ void activate8(Vec8 &u, int act)
{
    if (act == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) u.v[e] *= sigmoid_acc(u.v[e]);
    } else if (act == 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e) u.v[e] = sigmoid_acc(u.v[e]);
    }
}

// Sums over the lanes of a row (WPR warps); every lane gets the result.  `buf` holds 2 x WPR pairs per row group, the
// halves used in turn so that one barrier per sum is enough.  A pair of sums takes 5 exchanges, not 10: the first one gives
// one value to each half of the warp.
template <int WPR>
struct RowSum {
    float2 *buf;
    int parity, group, wr, lane;
    __device__ __forceinline__ float2 meet(float2 mine, bool writer, bool second)   // second: this lane writes .y
    {
        float2 *b = buf + (group * 2 + parity) * WPR;
        parity ^= 1;
        if (writer) reinterpret_cast<float *>(b + wr)[second] = second ? mine.y : mine.x;
        asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(WPR * 32) : "memory");
        float2 t = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WPR; w += 2) {
            const float4 v = *reinterpret_cast<const float4 *>(b + w);
            t.x += v.x + v.z;
            t.y += v.y + v.w;
        }
        return t;
    }
    __device__ __forceinline__ float one(float v)
    {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return WPR == 1 ? v : meet(make_float2(v, 0.f), lane == 0, false).x;
    }
    __device__ __forceinline__ float2 two(float a, float b)
    {
        const bool up = lane & 16;
        float v = (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (WPR == 1) {
            const float w = __shfl_xor_sync(0xffffffffu, v, 16);
            return make_float2(up ? w : v, up ? v : w);
        }
        return meet(make_float2(v, v), (lane & 15) == 0, up);
    }
};

// ------------------------------------------------------------------------------------------------ forward

// kBias: without the two bias vectors a lane needs 80 registers and three CTAs are resident, with them two (32768 x 1024
// with biases and layer norms 85 us, without either 78).
template <typename TI, typename TR, typename TO, int WPR, bool kBias>
__global__ void __launch_bounds__(WPR > 8 ? 32 * WPR : 256, WPR > 8 ? 1 : (kBias ? 2 : 3)) blocknorm_fwd_kernel(const NormParams p)
{
    constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
    __shared__ __align__(16) float2 buf[GROUPS * 2 * WPR];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp / WPR, wr = warp % WPR;
    RowSum<WPR> sum = {buf, 0, group, wr, lane};
    const float inv_d = 1.f / p.D;
    const int c = 8 * (wr * 32 + lane);
    const bool live = c < p.D, post = p.y != nullptr, pre = p.o != nullptr, gated = p.gate != nullptr;
    // this lane's weights, in registers for all its rows: from shared memory they kept the load pipe 80 % busy.  scale is
    // folded into the post norm's weight and bias; channels past D get zeros there and stay zero in r'.
    Vec8 w_post = fill8(0.f), b_post, w_pre = fill8(0.f), b_pre;
    if (live && post) {
        const Vec8 sc = p.scale ? load8(p.scale + c) : fill8(1.f);
        w_post = p.w_post ? load8(p.w_post + c) : fill8(1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) w_post.v[e] *= sc.v[e];
        if (kBias) {
            b_post = p.b_post ? load8(p.b_post + c) : fill8(0.f);
#pragma unroll
            for (int e = 0; e < 8; ++e) b_post.v[e] *= sc.v[e];
        }
    } else if (kBias) {
        b_post = fill8(0.f);
    }
    if (live && pre) w_pre = p.w_pre ? load8(p.w_pre + c) : fill8(1.f);
    if (kBias) b_pre = live && pre && p.b_pre ? load8(p.b_pre + c) : fill8(0.f);

    auto normalise = [&](Vec8 &x, int kind) {
        if (kind == CHELA_NORM_NONE) return;
        if (kind == CHELA_NORM_LAYER) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += x.v[e];
            s = sum.one(s);
            const float mean = live ? s * inv_d : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[e] -= mean;
        }
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x.v[e], x.v[e], s);
        const float inv = 1.0f / sqrtf(fmaf(sum.one(s), inv_d, p.eps));
#pragma unroll
        for (int e = 0; e < 8; ++e) x.v[e] *= inv;
    };

    const long long stride = (long long)gridDim.x * GROUPS;
    long long row = (long long)blockIdx.x * GROUPS + group;
    Raw8<TR> rr;
    Raw8<TI> ry, rg;
    auto fetch = [&](long long at) {
        const bool ok = live && at < p.T;
        if (ok && p.res) rr.load(static_cast<const TR *>(p.res) + (size_t)at * p.rs + c, p.wide); else rr.zero();
        if (ok && post) ry.load(static_cast<const TI *>(p.y) + (size_t)at * p.ys + c, p.wide); else ry.zero();
        if (ok && gated) rg.load(static_cast<const TI *>(p.gate) + (size_t)at * p.gs + c, p.wide); else rg.zero();
    };
    fetch(row);
    for (; row < p.T; row += stride) {
        Vec8 r = rr.get(), v = ry.get(), g = rg.get();
        fetch(row + stride);
        if (post) {
            if (gated) {
                activate8(g, p.gate_act);
                if (!p.gate_after) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v.v[e] *= g.v[e];
                }
            }
            normalise(v, p.norm_post);
#pragma unroll
            for (int e = 0; e < 8; ++e) v.v[e] = kBias ? fmaf(v.v[e], w_post.v[e], b_post.v[e]) : v.v[e] * w_post.v[e];
            if (gated && p.gate_after) {
#pragma unroll
                for (int e = 0; e < 8; ++e) r.v[e] = fmaf(v.v[e], g.v[e], r.v[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) r.v[e] += v.v[e];
            }
            if (live && p.res_out) put8(static_cast<TR *>(p.res_out) + (size_t)row * p.D + c, r, p.wide);
        }
        if (pre) {
            normalise(r, p.norm_pre);
#pragma unroll
            for (int e = 0; e < 8; ++e) r.v[e] = kBias ? fmaf(r.v[e], w_pre.v[e], b_pre.v[e]) : r.v[e] * w_pre.v[e];
            if (live) put8(static_cast<TO *>(p.o) + (size_t)row * p.D + c, r, p.wide);
        }
    }
}

// ------------------------------------------------------------------------------------------------ backward

struct NormBwdParams {
    NormParams f;   // res = r'
    const void *d_o, *d_ro;
    void *d_res, *d_y, *d_gate;
    float *part;    // [CTAs][4][D]: sums over the rows of d n hat / scale and d n / scale, of d o hat' and d o
};

// One vector of 8 channels a lane, so that the sums that the parameters' gradients are made of (32 registers) stay in
// registers over all rows the group walks; D <= 256 WPR.  With P = sum d n hat / scale and Q = sum d n / scale, where d n /
// scale is d r' (times the gate behind the norm): d_w_post = scale P, d_b_post = scale Q, d_scale = w_post P + b_post Q.
// 16 warps an SM of 128 registers and three or four dependent sums over the row: the chain of these, not HBM, bounds it
// (32749 x 1024, layer norms, gate, bf16 beside an fp32 residual: 159 us for 113 us of traffic; one operation a channel
// and five sums instead of pairs and four: 197).  Two rows a warp at a time need 168 registers, 12 warps: 158 us where one
// takes 165 at 1024 channels, but 215 at 512 and 379 against 271 in fp32, whose operands then fill shared memory.  Channels past D have zero operands, and zero weights where that is not
// enough, so they add nothing to the sums.
template <typename TI, typename TR, typename TG, int WPR>
__global__ void __launch_bounds__(WPR > 8 ? 32 * WPR : 256, WPR > 8 ? 1 : 2) blocknorm_bwd_kernel(const NormBwdParams q)
{
    constexpr int GROUPS = WPR > 8 ? 1 : 8 / WPR;
    const NormParams &p = q.f;
    constexpr int WIDTH = WPR * 256;
    __shared__ __align__(16) float2 buf[GROUPS * 2 * WPR];
    extern __shared__ __align__(16) float s_w[];   // w_post scale, b_post scale, w_pre [WIDTH]; in the end the groups' sums
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp / WPR, wr = warp % WPR;
    RowSum<WPR> sum = {buf, 0, group, wr, lane};
    const float inv_d = 1.f / p.D;
    const int c = 8 * (wr * 32 + lane);
    const bool live = c < p.D;
    Vec8 acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = fill8(0.f);
    const bool post = p.y != nullptr, pre = q.d_o != nullptr, gated = p.gate != nullptr;
    stage_weight(s_w, p.w_post, 1.f, p.scale, p.D, WIDTH);
    stage_weight(s_w + WIDTH, p.b_post, 0.f, p.scale, p.D, WIDTH);
    stage_weight(s_w + 2 * WIDTH, p.w_pre, 1.f, nullptr, p.D, WIDTH);
    __syncthreads();

    // Operands of a row.  Up to 2048 channels they are copied to shared memory one row ahead, every lane what it will read
    // itself, so nothing but its own copies has to be waited for and registers are not held meanwhile; wider rows are read
    // where they are wanted.
    constexpr bool AHEAD = WPR <= 8;
    constexpr int NR = sizeof(TR) / 2, NI = sizeof(TI) / 2, SLOTS = 2 * NR + 3 * NI;   // 16-byte vectors of r', d r', d o, y, gate
    uint4 *s_row = reinterpret_cast<uint4 *>(s_w + (GROUPS > 4 ? GROUPS - 1 : 3) * WIDTH) + warp * (2 * SLOTS * 32) + lane;
    const float *s_lane = s_w + wr * 256 + 4 * lane;
    const long long stride = (long long)gridDim.x * GROUPS;
    long long row = (long long)blockIdx.x * GROUPS + group;
    auto fetch = [&](long long at, int stage) {
        const bool ok = live && at < p.T;
        uint4 *to = s_row + stage * SLOTS * 32;
        auto vectors = [&](int slot, const char *from, int n, bool used) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i < n) copy16(to + (slot + i) * 32, from + 16 * i, ok && used);
        };
        const size_t t = ok ? (size_t)at : 0, k = ok ? c : 0;
        const bool grad = q.d_ro != nullptr;
        vectors(0, reinterpret_cast<const char *>(static_cast<const TR *>(pre ? p.res : q.d_res) + t * (pre ? p.rs : p.D) + k), NR, pre);
        vectors(NR, reinterpret_cast<const char *>(static_cast<const TR *>(grad ? q.d_ro : q.d_res) + t * p.D + k), NR, grad);
        vectors(2 * NR, static_cast<const char *>(pre ? q.d_o : q.d_res) + (t * p.D + k) * sizeof(TI), NI, pre);
        vectors(2 * NR + NI, static_cast<const char *>(post ? p.y : q.d_res) + (post ? (t * p.ys + k) * sizeof(TI) : 0), NI, post);
        vectors(2 * NR + 2 * NI, static_cast<const char *>(gated ? p.gate : q.d_res) + (gated ? (t * p.gs + k) * sizeof(TI) : 0), NI, gated);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int stage = 0;
    if (AHEAD) fetch(row, 0);
    for (; row < p.T; row += stride) {
        if (AHEAD) {
            fetch(row + stride, stage ^ 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        }
        const uint4 *now = s_row + stage * SLOTS * 32;
        stage ^= 1;
        auto res_like = [&](int slot, const void *from, long long step, bool used) -> Vec8 {
            Raw8<TR> r;
            if (AHEAD) r.from(now + slot * 32, 32);
            else if (live && used) r.load(static_cast<const TR *>(from) + (size_t)row * step + c, p.wide);
            else r.zero();
            return r.get();
        };
        auto in_like = [&](int slot, const void *from, long long step, bool used) -> Vec8 {
            Raw8<TI> r;
            if (AHEAD) r.from(now + slot * 32, 32);
            else if (live && used) r.load(static_cast<const TI *>(from) + (size_t)row * step + c, p.wide);
            else r.zero();
            return r.get();
        };
        auto read_y = [&]() { return in_like(2 * NR + NI, p.y, p.ys, post); };
        auto read_gate = [&]() { return in_like(2 * NR + 2 * NI, p.gate, p.gs, gated); };
        Vec8 hat = res_like(0, p.res, p.rs, pre), v = read_y(), ga;
        if (gated) {
            ga = read_gate();
            activate8(ga, p.gate_act);
            if (!p.gate_after) v = mul8(v, ga);
        }
        // statistics of both norms together: r' and v
        float2 s;
        const bool l0 = pre && p.norm_pre == CHELA_NORM_LAYER, l1 = post && p.norm_post == CHELA_NORM_LAYER;
        if (l0 || l1) {
            s = sum.two(sum8(hat), sum8(v));
            hat = add8(hat, fill8(l0 && live ? -s.x * inv_d : 0.f));
            v = add8(v, fill8(l1 && live ? -s.y * inv_d : 0.f));
        }
        s = sum.two(dot8(hat, hat), dot8(v, v));
        const float i0 = p.norm_pre == CHELA_NORM_NONE ? 1.f : 1.0f / sqrtf(fmaf(s.x, inv_d, p.eps));
        const float i1 = p.norm_post == CHELA_NORM_NONE ? 1.f : 1.0f / sqrtf(fmaf(s.y, inv_d, p.eps));
        // norm before the next block: d hat, then d r'
        Vec8 d_r = res_like(NR, q.d_ro, p.D, q.d_ro != nullptr);
        if (pre) {
            Vec8 d_o = in_like(2 * NR, q.d_o, p.D, pre);
            hat = mul8(hat, fill8(i0));
            acc[2] = fma8(d_o, hat, acc[2]);
            acc[3] = add8(acc[3], d_o);
            d_o = mul8(d_o, staged8(s_lane + 2 * WIDTH));
            if (p.norm_pre != CHELA_NORM_NONE) {
                s = sum.two(dot8(d_o, hat), sum8(d_o));
                const float k0 = -s.x * inv_d * i0, k1 = l0 && live ? -s.y * inv_d * i0 : 0.f;   // channels past D stay zero
                d_r = fma8(fill8(i0), d_o, d_r);
                d_r = fma8(hat, fill8(k0), d_r);
                if (l0) d_r = add8(d_r, fill8(k1));
            } else {
                d_r = add8(d_r, d_o);
            }
        }
        if (live) put8(static_cast<TR *>(q.d_res) + (size_t)row * p.D + c, d_r, false);
        if (post) {
            // d_r becomes d n / scale, then d hat, then d v
            const Vec8 w = staged8(s_lane);
            v = mul8(v, fill8(i1));
            Vec8 dg;   // gradient of act(gate)
            if (gated && p.gate_after) {
                dg = mul8(d_r, fma8(v, w, staged8(s_lane + WIDTH)));
                d_r = mul8(d_r, ga);
            }
            acc[0] = fma8(d_r, v, acc[0]);
            acc[1] = add8(acc[1], d_r);
            d_r = mul8(d_r, w);
            if (p.norm_post != CHELA_NORM_NONE) {
                s = sum.two(dot8(d_r, v), sum8(d_r));
                d_r = mul8(d_r, fill8(i1));
                d_r = fma8(v, fill8(-s.x * inv_d * i1), d_r);
                if (l1) d_r = add8(d_r, fill8(-s.y * inv_d * i1));
            }
            if (gated) {
                const Vec8 gr = read_gate();
                if (!p.gate_after) {
                    dg = mul8(d_r, read_y());
                    d_r = mul8(d_r, ga);
                }
                if (p.gate_act == 1) {   // slope sg (1 + u (1 - sg)) = sg + act (1 - sg)
                    Vec8 sg;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sg.v[e] = sigmoid_acc(gr.v[e]);
                    dg = mul8(dg, fma8(ga, fma8(sg, fill8(-1.f), fill8(1.f)), sg));
                } else if (p.gate_act == 2) {
                    dg = mul8(dg, fma8(mul8(ga, fill8(-1.f)), ga, ga));
                }
                if (live) put8(static_cast<TG *>(q.d_gate) + (size_t)row * p.D + c, dg, false);
            }
            if (live) put8(static_cast<TG *>(q.d_y) + (size_t)row * p.D + c, d_r, false);
        }
    }
    // sums of the CTA's row groups, one partial row per CTA
    if (GROUPS > 1) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            __syncthreads();
            if (group > 0) store8(s_w + (group - 1) * WIDTH + c, acc[k]);
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int w = 0; w < GROUPS - 1; ++w) {
                    const Vec8 v = load8(s_w + w * WIDTH + c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[k].v[e] += v.v[e];
                }
            }
        }
    }
    if (live && group == 0) {
        float *o = q.part + (size_t)blockIdx.x * 4 * p.D + c;
#pragma unroll
        for (int k = 0; k < 4; ++k) store8(o + (size_t)k * p.D, acc[k]);
    }
}

struct NormSums {
    float *d_w_post, *d_b_post, *d_scale, *d_w_pre, *d_b_pre;
    const float *w_post, *b_post, *scale;
};
// sums over the CTAs in two fixed steps: 32 warps take every 32nd partial, then meet in shared memory.  blockIdx.y: P and Q
// of the post norm, or the two of the pre norm
__global__ void __launch_bounds__(1024) blocknorm_sum_kernel(const float *part, NormSums sums, int nparts, int D)
{
    __shared__ float2 red[32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, k = 2 * blockIdx.y;
    if (k == 0 ? !sums.d_w_post && !sums.d_b_post && !sums.d_scale : !sums.d_w_pre && !sums.d_b_pre) return;
    float2 o = make_float2(0.f, 0.f);
    if (c < D) {
#pragma unroll 4
        for (int i = warp; i < nparts; i += 32) {
            const float *at = part + ((size_t)i * 4 + k) * D + c;
            o.x += at[0];
            o.y += at[D];
        }
    }
    red[warp][lane] = o;
    __syncthreads();
    if (warp != 0 || c >= D) return;
    o = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 32; ++w) o = add2v(o, red[w][lane]);
    if (k == 0) {
        const float sc = sums.scale ? sums.scale[c] : 1.f;
        if (sums.d_w_post) sums.d_w_post[c] = sc * o.x;
        if (sums.d_b_post) sums.d_b_post[c] = sc * o.y;
        if (sums.d_scale) sums.d_scale[c] = fmaf(sums.w_post ? sums.w_post[c] : 1.f, o.x, sums.b_post ? sums.b_post[c] * o.y : 0.f);
    } else {
        if (sums.d_w_pre) sums.d_w_pre[c] = o.x;
        if (sums.d_b_pre) sums.d_b_pre[c] = o.y;
    }
}

int row_warps(int D)
{
    int w = 1;
    while (w * 256 < D) w <<= 1;
    return w;
}
int row_groups(int wpr) { return wpr > 8 ? 1 : 8 / wpr; }
// CTAs that walk the rows: as many as are resident, no more than there are row groups
int row_grid(int T, int D, int per_sm)
{
    const int g = row_groups(row_warps(D)), need = (int)(((long long)T + g - 1) / g);
    return need < 148 * per_sm ? need : 148 * per_sm;
}
constexpr int kBwdPerSm = 2;

template <typename K, typename P>
chela_status_t norm_launch(K kern, const P &p, int grid, int threads, size_t smem, cudaStream_t stream)
{
    if (smem > 47 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return cuda_status(e);
    }
    kern<<<grid, threads, smem, stream>>>(p);
    return last_launch_status();
}

template <typename TI, typename TR, typename TO, bool kBias>
chela_status_t fwd_bias(const NormParams &p, cudaStream_t stream)
{
    const int wpr = row_warps(p.D), grid = row_grid(p.T, p.D, kBias ? 2 : 3);
    switch (wpr) {
    case 1: return norm_launch(blocknorm_fwd_kernel<TI, TR, TO, 1, kBias>, p, grid, 256, 0, stream);
    case 2: return norm_launch(blocknorm_fwd_kernel<TI, TR, TO, 2, kBias>, p, grid, 256, 0, stream);
    case 4: return norm_launch(blocknorm_fwd_kernel<TI, TR, TO, 4, kBias>, p, grid, 256, 0, stream);
    case 8: return norm_launch(blocknorm_fwd_kernel<TI, TR, TO, 8, kBias>, p, grid, 256, 0, stream);
    case 16: return norm_launch(blocknorm_fwd_kernel<TI, TR, TO, 16, kBias>, p, grid, 512, 0, stream);
    default: return norm_launch(blocknorm_fwd_kernel<TI, TR, TO, 32, kBias>, p, grid, 1024, 0, stream);
    }
}

template <typename TI, typename TR, typename TO>
chela_status_t fwd_d(const NormParams &p, cudaStream_t stream)
{
    return p.b_post || p.b_pre ? fwd_bias<TI, TR, TO, true>(p, stream) : fwd_bias<TI, TR, TO, false>(p, stream);
}

template <typename TI, typename TR, typename TG>
chela_status_t bwd_d(const NormBwdParams &q, const NormSums &sums, cudaStream_t stream)
{
    const NormParams &p = q.f;
    const int wpr = row_warps(p.D), grid = row_grid(p.T, p.D, kBwdPerSm);
    // weights (in the end the row groups' sums); two rows of operands a warp where they are fetched ahead
    const int rows = row_groups(wpr) > 4 ? row_groups(wpr) - 1 : 3;
    const size_t ahead = wpr <= 8 ? (size_t)8 * 2 * (sizeof(TR) + 3 * sizeof(TI) / 2) * 32 * 16 : 0;
    const size_t smem = (size_t)rows * wpr * 256 * 4 + ahead;
    chela_status_t st;
    switch (wpr) {
    case 1: st = norm_launch(blocknorm_bwd_kernel<TI, TR, TG, 1>, q, grid, 256, smem, stream); break;
    case 2: st = norm_launch(blocknorm_bwd_kernel<TI, TR, TG, 2>, q, grid, 256, smem, stream); break;
    case 4: st = norm_launch(blocknorm_bwd_kernel<TI, TR, TG, 4>, q, grid, 256, smem, stream); break;
    case 8: st = norm_launch(blocknorm_bwd_kernel<TI, TR, TG, 8>, q, grid, 256, smem, stream); break;
    case 16: st = norm_launch(blocknorm_bwd_kernel<TI, TR, TG, 16>, q, grid, 512, smem, stream); break;
    default: st = norm_launch(blocknorm_bwd_kernel<TI, TR, TG, 32>, q, grid, 1024, smem, stream); break;
    }
    if (st == CHELA_OK && (sums.d_w_post || sums.d_b_post || sums.d_scale || sums.d_w_pre || sums.d_b_pre)) {
        blocknorm_sum_kernel<<<dim3((p.D + 31) / 32, 2), 1024, 0, stream>>>(q.part, sums, grid, p.D);
        st = last_launch_status();
    }
    return st;
}

bool on_sector(const void *p, bool is_f32) { return !is_f32 || reinterpret_cast<uintptr_t>(p) % 32 == 0; }
NormParams norm_params(const chela_blocknorm_args_t &a)
{
    NormParams p = {};
    const bool i32 = a.in_dtype == CHELA_F32;
    p.wide = on_sector(a.res, a.res_dtype == CHELA_F32) && on_sector(a.y, i32) && on_sector(a.gate, i32);
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
    p.wide = p.wide && on_sector(res_out, a.res_dtype == CHELA_F32) && on_sector(o, out_dtype == CHELA_F32);
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
    return align_up((size_t)row_grid(T, D, kBwdPerSm) * 4 * D * sizeof(float), 256);
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
    q.f.wide = q.f.wide && on_sector(d_o, a.in_dtype == CHELA_F32) && on_sector(d_res_out, a.res_dtype == CHELA_F32);   // for its loads
    q.part = static_cast<float *>(workspace);
    const NormSums sums = {d_w_post, d_b_post, d_scale, d_w_pre, d_b_pre, a.w_post, a.b_post, a.scale};
    const bool i32 = a.in_dtype == CHELA_F32, r32 = a.res_dtype == CHELA_F32, g32 = grad_dtype == CHELA_F32;
    if (i32) {
        if (r32) return g32 ? bwd_d<float, float, float>(q, sums, stream) : bwd_d<float, float, bf>(q, sums, stream);
        return g32 ? bwd_d<float, bf, float>(q, sums, stream) : bwd_d<float, bf, bf>(q, sums, stream);
    }
    if (r32) return g32 ? bwd_d<bf, float, float>(q, sums, stream) : bwd_d<bf, float, bf>(q, sums, stream);
    return g32 ? bwd_d<bf, bf, float>(q, sums, stream) : bwd_d<bf, bf, bf>(q, sums, stream);
}

}  // namespace chela
