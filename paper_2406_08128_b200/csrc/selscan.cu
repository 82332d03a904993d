// Selective state space scan over packed sequences:
//   h_t[n] = exp(dt_t a[c,n]) h_{t-1}[n] + dt_t b_t[n] x_t,   y_t = (<c_t, h_t> + d_skip x_t) silu(z_t)   per channel c.
//
// What bounds it: N exponentials a token and channel against 8 bytes of bf16 operands.  An SM evaluates 16 exponentials
// a cycle, so N = 16 costs 1.2 cycles a token and channel (with softplus and the gate) where its share of the measured
// HBM rate needs 0.36: the forward pass is bound by the exponentials, not by memory.
//
// Layout of the work: a thread holds 4 states of one channel; N / 4 neighbouring lanes make up a channel, the other lane
// bits are channels, and the warps of a CTA are time slices of kTok tokens of the same channels.  A slice is scanned from
// a zero state while its decays are multiplied up; slices then meet in shared memory, and each adds what the state
// before it contributes, c_t[n] (prod decay)[n] h_in[n], from registers.  So every exponential is evaluated once whatever the
// number of time slices, and a long sequence with few channels still fills the SM.
#include "packed.cuh"

namespace chela {
namespace {

constexpr int kCkptTok = 32;   // tokens between checkpoints; also the tile of the backward kernel

struct ScanParams {
    const void *x, *dt, *b, *c, *z;
    long long xs, dts, bs, cs, zs;
    const float *a, *dsk, *bias;
    const float *state_in;
    const int *off;
    int S, T, D, G, softplus;
    void *y;
    float *state_out, *ckpt;
    // a sequence split into segments of seg tokens (0: not split): seg_state [segments][D][N]; seg_sum [segments][D] is
    // given in the pass that finds the segments' ends from zero states
    int seg;
    float *seg_state, *seg_sum;
};

__device__ __forceinline__ float4 zero4() { return make_float4(0.f, 0.f, 0.f, 0.f); }
__device__ __forceinline__ float4 opt4(const float *p, int i, float v)
{
    return p ? *reinterpret_cast<const float4 *>(p + i) : make_float4(v, v, v, v);
}
// a log2(e), minus infinity replaced by the lowest finite value: exp(dt a) is 0 for dt > 0 all the same, and the tokens
// past a sequence's end (dt = 0) keep the state instead of producing 0 * infinity
__device__ __forceinline__ float decay_rate(float a)
{
    const float v = a * kLog2e;
    return v < -3.0e38f ? -3.0e38f : v;
}
__device__ __forceinline__ float gate_f(float z) { return z * sigmoid_acc(z); }

// ------------------------------------------------------------------------------------------------ forward

__device__ __forceinline__ void named_sync(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void named_arrive(int id) { asm volatile("bar.arrive %0, 64;" ::"r"(id) : "memory"); }
// 16 bytes from global to shared memory, zeros where ok is false (the address is then not read)
__device__ __forceinline__ void copy16(void *dst, const void *src, bool ok)
{
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(ok ? 16 : 0) : "memory");
}

// NS = 8 states and CH channels a lane; R = N / 8 lanes share CH channels.
template <typename TI, int N, int CH, int TOK>
struct FwdShape {
    static constexpr int NS = 8, NP = 4, R = N / NS, CPW = 32 / R * CH, E16 = 16 / (int)sizeof(TI);
    static constexpr int PT = TOK * CH / R;                              // tokens a lane prepares, of one channel
    static constexpr int XC = CPW / E16, BC = N / E16;                   // 16-byte pieces of a token's x, b
    static constexpr int CHUNKS = TOK * (3 * XC + 2 * BC), CPL = (CHUNKS + 31) / 32;   // of a slice, a lane
    static constexpr int RAW_E = CHUNKS * E16;                           // elements of a raw slice
    static constexpr int HAND_B = 32 * CH * NS * 4;
    static constexpr int BC_F = 2 * TOK * N;                             // b, c of a slice in fp32
    static constexpr int WARP_B = 2 * RAW_E * (int)sizeof(TI) + BC_F * 4 + HAND_B;
};

// One CTA: WT warps that take turns with the slices of TOK tokens of one chain: CPW channels of a sequence, or of a
// segment of one.  A warp fetches its slice (asynchronously, one slice ahead), evaluates its decays, waits for the state
// from the warp before it, runs the recurrence, hands the state on and forms the outputs; only the recurrence is serial.
// A lane prepares (time step, gate, output) PT tokens of one channel, "its" channel, and runs 8 states of all CH
// channels of its R lanes: slot 0 is its own channel, slot 1 its neighbour's, so that one exchange with lane ^ 1 turns
// partial outputs around, and one 16-byte read of b or c (2 cycles an SM for 16 broadcast bytes) serves CH channels.
// Two pools of work run beside each other here and are about equally long, which is why taking away any one part changes
// the time by a few per cent only: exponentials (8 cycles a warp instruction) with the shared memory traffic behind the
// same queue, and the multiply-adds.  Two-wide multiply-adds of three different register pairs take 4.2 cycles of a
// scheduler, two single ones 2.6 but twice the issue slots; as a whole the two-wide form is 10 % faster.
template <typename TI, typename TO, int N, int CH, int TOK, int WT, int OCC>
__global__ void __launch_bounds__(32 * WT, OCC) selscan_fwd_kernel(const ScanParams p)
{
    using Sh = FwdShape<TI, N, CH, TOK>;
    constexpr int NS = Sh::NS, R = Sh::R, NP = Sh::NP, CPW = Sh::CPW, E16 = Sh::E16, XC = Sh::XC, BC = Sh::BC, CPL = Sh::CPL, PT = Sh::PT;
    static_assert(XC >= 1 && BC >= 1 && kCkptTok % TOK == 0 && PT >= 1 && WT > 1 && WT <= 15 && R >= CH, "shapes");
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ longlong2 s_src[5];                                       // address of token 0, bytes between a warp's slices
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned char *s_mine = smem + warp * Sh::WARP_B;
    TI *s_raw = reinterpret_cast<TI *>(s_mine);                          // two slices: x, dt, z [TOK][CPW], b, c [TOK][N]
    float *s_f = reinterpret_cast<float *>(s_mine + 2 * Sh::RAW_E * sizeof(TI));   // b, c [TOK][N] in fp32
    float4 *s_hand = reinterpret_cast<float4 *>(s_mine + Sh::WARP_B - Sh::HAND_B);   // [CH NS / 4][32] the state handed on

    const int nblk = (p.D + CPW - 1) / CPW;
    const long long blk = blockIdx.x / nblk;
    const int c0 = (blockIdx.x % nblk) * CPW;
    int s, b = 0;
    SeqRange sr;
    if (p.seg) {
        s = packed_block_seq(p.off, p.S, p.T, p.seg, blk);
        sr = seq_range(p.off, s, p.S, p.T);
        b = (int)(blk - (sr.start / p.seg + s));
        if (b < 0 || (b > 0 && b * p.seg >= sr.len)) return;
    } else {
        s = (int)blk;
        sr = seq_range(p.off, s, p.S, p.T);
    }
    const int begin = b * p.seg, end = p.seg ? min(begin + p.seg, sr.len) : sr.len;   // tokens of the sequence
    const bool final = end == sr.len;
    const int q = lane % R, grp = lane / R;
    const int chl = grp * CH + q % CH, ch = c0 + chl, tok0 = (q / CH) * PT;   // this lane's channel, its first token of a slice
    const int n0 = NS * q;
    const bool live = ch < p.D;
    const int g = p.G == 1 ? 0 : c0 / (p.D / p.G);

    if (threadIdx.x < 5) {
        const int w = threadIdx.x;
        const void *base = w == 0 ? p.x : w == 1 ? p.dt : w == 2 ? p.z : w == 3 ? p.b : p.c;
        const long long stride = w == 0 ? p.xs : w == 1 ? p.dts : w == 2 ? p.zs : w == 3 ? p.bs : p.cs;
        const long long at = ((long long)sr.start + begin) * stride + (w < 3 ? c0 : g * N);
        s_src[w] = base ? make_longlong2((long long)base + at * (long long)sizeof(TI), stride * (long long)sizeof(TI)) : make_longlong2(0, 0);
    }

    // decay rates in shared memory, [CH NS / 4][32]: they are wanted before the state is, so that one takes the other's
    // registers
    __shared__ float4 s_a[CH * NP / 2][32];
    float2 h[CH][NP];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int cj = ch ^ j;   // pairs of channels start at even ones, so the neighbour is ch ^ 1
        const bool ok = cj < p.D;
        const size_t at = (size_t)cj * N + n0;
        const float *init = p.seg_sum ? nullptr : (b > 0 ? p.seg_state + (size_t)blk * p.D * N : (p.state_in ? p.state_in + (size_t)s * p.D * N : nullptr));
#pragma unroll
        for (int k = 0; k < NP; k += 2) {
            float4 av = zero4(), hv = zero4();
            if (ok) {
                av = *reinterpret_cast<const float4 *>(p.a + at + 2 * k);
                av = make_float4(decay_rate(av.x), decay_rate(av.y), decay_rate(av.z), decay_rate(av.w));
                if (init) hv = *reinterpret_cast<const float4 *>(init + at + 2 * k);
            }
            h[j][k] = make_float2(hv.x, hv.y);
            h[j][k + 1] = make_float2(hv.z, hv.w);
            if (warp == 0) s_a[j * NP / 2 + k / 2][lane] = av;
        }
    }
    auto keep = [&](float *to, const float2 (&v)[CH][NP]) {   // states of this lane to a [D][N] array
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if ((ch ^ j) < p.D) {
                float4 *o = reinterpret_cast<float4 *>(to + (size_t)(ch ^ j) * N + n0);
                o[0] = make_float4(v[j][0].x, v[j][0].y, v[j][1].x, v[j][1].y);
                o[1] = make_float4(v[j][2].x, v[j][2].y, v[j][3].x, v[j][3].y);
            }
        }
    };
    const float bias = live && p.bias ? p.bias[ch] : 0.f, skip = live && p.dsk ? p.dsk[ch] : 0.f;
    __syncthreads();

    // this lane's 16-byte pieces of a slice
    const char *src[CPL];
    int tok[CPL];
    long long step[CPL];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
        int id = lane + 32 * i;
        const bool in_x = id < 3 * TOK * XC;
        int which = in_x ? id / (TOK * XC) : 3 + (id - 3 * TOK * XC) / (TOK * BC);
        id = in_x ? id % (TOK * XC) : (id - 3 * TOK * XC) % (TOK * BC);
        const int per = in_x ? XC : BC;
        tok[i] = id / per;
        const bool used = lane + 32 * i < Sh::CHUNKS;
        if (!used) which = 0;
        const longlong2 from = s_src[which];
        const bool ok = used && from.x && (!in_x || c0 + (id % per) * E16 < p.D);
        src[i] = reinterpret_cast<const char *>(ok ? from.x + (long long)(warp * TOK + tok[i]) * from.y + (id % per) * 16 : (long long)p.x);
        step[i] = ok ? from.y * (WT * TOK) : 0;
        if (!ok) tok[i] = 0x40000000;   // never inside; the address stays where it is
    }
    auto fetch = [&](int t0, int to) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            if (lane + 32 * i < Sh::CHUNKS) copy16(s_raw + to * Sh::RAW_E + (lane + 32 * i) * E16, src[i], tok[i] < end - t0);
            src[i] += step[i];
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    if (begin >= end && warp == 0 && p.state_out && !p.seg_sum) keep(p.state_out + (size_t)s * p.D * N, h);
    TO *py = static_cast<TO *>(p.y) + (p.y ? ((size_t)sr.start + begin + warp * TOK + tok0) * p.D + ch : 0);
    float all_dt = 0.f;
    int stage = 0;
    fetch(begin + warp * TOK, 0);
    for (int t0 = begin + warp * TOK; t0 < end; t0 += WT * TOK) {
        fetch(t0 + WT * TOK, stage ^ 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        const TI *raw = s_raw + stage * Sh::RAW_E;
#pragma unroll
        for (int i = 0; i < (Sh::BC_F / 4 + 31) / 32; ++i)
            if (lane + 32 * i < Sh::BC_F / 4) reinterpret_cast<float4 *>(s_f)[lane + 32 * i] = load4(raw + 3 * TOK * CPW + 4 * (lane + 32 * i));
        const float *s_b = s_f + n0, *s_c = s_b + TOK * N;
        auto row_of = [&](const float *m, float2 (&o)[NP]) {
            const float4 u = reinterpret_cast<const float4 *>(m)[0], v = reinterpret_cast<const float4 *>(m)[1];
            o[0] = make_float2(u.x, u.y);
            o[1] = make_float2(u.z, u.w);
            o[2] = make_float2(v.x, v.y);
            o[3] = make_float2(v.z, v.w);
        };
        float dt[PT], dx[PT];
#pragma unroll
        for (int i = 0; i < PT; ++i) dt[i] = load1(raw + (TOK + tok0 + i) * CPW + chl) + bias;
        if (p.softplus) {
#pragma unroll
            for (int i = 0; i < PT; i += 2) {
                const float2 v = softplus_acc(make_float2(dt[i], dt[i + 1 < PT ? i + 1 : i]));
                dt[i] = v.x;
                if (i + 1 < PT) dt[i + 1] = v.y;
            }
        }
        if (t0 + TOK > end) {   // past the end: decay 1, no input
#pragma unroll
            for (int i = 0; i < PT; ++i)
                if (t0 + tok0 + i >= end) dt[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < PT; ++i) dx[i] = dt[i] * load1(raw + (tok0 + i) * CPW + chl);
        if (p.seg_sum) {
#pragma unroll
            for (int i = 0; i < PT; ++i) all_dt += dt[i];
        }
        __syncwarp();
        // value of the token i, slot j, from the lane that prepared it
        auto of = [&](const float (&v)[PT], int i, int j) -> float {
            if (R == 1) return v[i % PT];
            if (R == 2) return j == 0 ? v[i % PT] : __shfl_xor_sync(0xffffffffu, v[i % PT], 1);
            return __shfl_sync(0xffffffffu, v[i % PT], (lane & ~(R - 1)) + ((q % CH) ^ j) + CH * (i / PT));
        };
        float2 e[TOK][CH][NP];
        auto rates = [&](int j, float2 (&o)[NP]) {
            const float4 u = s_a[j * NP / 2][lane], v = s_a[j * NP / 2 + 1][lane];
            o[0] = make_float2(u.x, u.y);
            o[1] = make_float2(u.z, u.w);
            o[2] = make_float2(v.x, v.y);
            o[3] = make_float2(v.z, v.w);
        };
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float2 a[NP];
            rates(j, a);
#pragma unroll
            for (int i = 0; i < TOK; ++i) {
                const float d = of(dt, i, j);
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const float2 v = mul2v(a[k], splat2(d));
                    e[i][j][k] = make_float2(ex2(v.x), ex2(v.y));
                }
            }
        }
        float dxs[TOK][CH];
#pragma unroll
        for (int i = 0; i < TOK; ++i)
#pragma unroll
            for (int j = 0; j < CH; ++j) dxs[i][j] = of(dx, i, j);
        const bool last = t0 + TOK >= end;
        if (t0 > begin) {
            const int from = (warp + WT - 1) % WT;
            named_sync(1 + from);
            const float4 *m = reinterpret_cast<const float4 *>(smem + from * Sh::WARP_B + Sh::WARP_B - Sh::HAND_B);
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int k = 0; k < NP; k += 2) {
                    const float4 v = m[(j * NP / 2 + k / 2) * 32 + lane];
                    h[j][k] = make_float2(v.x, v.y);
                    h[j][k + 1] = make_float2(v.z, v.w);
                }
        }
        auto hand_on = [&](const float2 (&v)[CH][NP]) {
            if (!last) {
#pragma unroll
                for (int j = 0; j < CH; ++j)
#pragma unroll
                    for (int k = 0; k < NP; k += 2)
                        s_hand[(j * NP / 2 + k / 2) * 32 + lane] = make_float4(v[j][k].x, v[j][k].y, v[j][k + 1].x, v[j][k + 1].y);
                named_arrive(1 + warp);
            } else if (p.seg_sum) {
                keep(p.seg_state + (size_t)blk * p.D * N, v);
            } else if (final && p.state_out) {
                keep(p.state_out + (size_t)s * p.D * N, v);
            }
        };
        if (p.ckpt && t0 % kCkptTok == 0) keep(p.ckpt + ((size_t)(sr.start / kCkptTok) + s + t0 / kCkptTok) * p.D * N, h);
#pragma unroll
        for (int i = 0; i < TOK; ++i) {
            float2 bv[NP];
            row_of(s_b + i * N, bv);
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    h[j][k] = fma2v(e[i][j][k], h[j][k], mul2v(splat2(dxs[i][j]), bv[k]));
                    e[i][j][k] = h[j][k];
                }
        }
        hand_on(h);
        if (p.y) {
            float y[TOK];   // of this lane's channel, after its neighbour's share has come in
#pragma unroll
            for (int i = 0; i < TOK; ++i) {
                float2 cv[NP];
                row_of(s_c + i * N, cv);
                float part[CH];
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    float2 u = mul2v(cv[0], e[i][j][0]);
#pragma unroll
                    for (int k = 1; k < NP; ++k) u = fma2v(cv[k], e[i][j][k], u);
                    part[j] = u.x + u.y;
                }
                y[i] = CH == 1 ? part[0] : part[0] + __shfl_xor_sync(0xffffffffu, part[CH - 1], 1);
            }
            // R > CH: the other lanes of this channel hold other states; halve the tokens at each exchange
            if (R > CH) {
                int n = TOK;
#pragma unroll
                for (int o = R / 2; o >= CH; o >>= 1) {
                    n >>= 1;
                    const bool up = lane & o;
#pragma unroll
                    for (int i = 0; i < TOK / 2; ++i) {
                        if (i < n) {
                            const float send = up ? y[i] : y[i + n], mine = up ? y[i + n] : y[i];
                            y[i] = mine + __shfl_xor_sync(0xffffffffu, send, o);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                float v = fmaf(skip, load1(raw + (tok0 + i) * CPW + chl), y[i]);
                if (p.z) v *= gate_f(load1(raw + (2 * TOK + tok0 + i) * CPW + chl));
                if (live && t0 + tok0 + i < end) store1(py + (size_t)i * p.D, v);
            }
            py += (size_t)(WT * TOK) * p.D;
        }
        stage ^= 1;
        __syncwarp();
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (p.seg_sum) {   // the segment's whole time, for its decay
        __syncthreads();
        float *s_dt = reinterpret_cast<float *>(smem);
        s_dt[warp * 32 + lane] = all_dt;
        __syncthreads();
        if (warp == 0 && live && q < CH) {
            float t = 0.f;
            for (int w = 0; w < WT; ++w)
#pragma unroll
                for (int o = 0; o < R; o += CH) t += s_dt[w * 32 + lane + o];
            p.seg_sum[(size_t)blk * p.D + ch] = t;
        }
    }
}

// Segments of a sequence in turn: the state each ends with becomes the state it starts with.
template <int N>
__global__ void __launch_bounds__(128) selscan_segments_kernel(const ScanParams p)
{
    const size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x;   // (s, channel, state)
    const size_t per = (size_t)p.D * N;
    if (i >= per * p.S) return;
    const int s = (int)(i / per), ch = (int)(i % per / N), n = (int)(i % N);
    const SeqRange sr = seq_range(p.off, s, p.S, p.T);
    const float a = decay_rate(p.a[(size_t)ch * N + n]);
    float h = p.state_in ? p.state_in[i] : 0.f;
    size_t k = (size_t)(sr.start / p.seg) + s;
    for (int t = 0; t < sr.len; t += p.seg, ++k) {
        float *m = p.seg_state + (k * p.D + ch) * N + n;
        const float own = *m;
        *m = h;
        h = fmaf(ex2(a * p.seg_sum[k * p.D + ch]), h, own);
    }
}

// ------------------------------------------------------------------------------------------------ single token

template <typename TI, typename TO, int N>
__global__ void __launch_bounds__(256) selscan_step_kernel(const ScanParams p)
{
    constexpr int R = N / 4;
    const size_t idx = blockIdx.x * (size_t)blockDim.x + threadIdx.x;
    const size_t row_ch = idx / R;
    const int r = (int)(idx % R);
    const bool live = row_ch < (size_t)p.S * p.D;
    const int s = live ? (int)(row_ch / p.D) : 0, ch = live ? (int)(row_ch % p.D) : 0;
    const int g = p.G == 1 ? 0 : ch / (p.D / p.G);
    const size_t st = ((size_t)s * p.D + ch) * N + 4 * r;
    const float4 h = *reinterpret_cast<const float4 *>(p.state_in + st);
    const float4 a = *reinterpret_cast<const float4 *>(p.a + (size_t)ch * N + 4 * r);
    const float4 b = load4(static_cast<const TI *>(p.b) + (size_t)s * p.bs + g * N + 4 * r);
    const float4 c = load4(static_cast<const TI *>(p.c) + (size_t)s * p.cs + g * N + 4 * r);
    const float x = load1(static_cast<const TI *>(p.x) + (size_t)s * p.xs + ch);
    float dt = load1(static_cast<const TI *>(p.dt) + (size_t)s * p.dts + ch) + (p.bias ? p.bias[ch] : 0.f);
    if (p.softplus) dt = softplus_acc(dt);
    const float dx = dt * x;
    float4 n;
    n.x = fmaf(ex2(dt * decay_rate(a.x)), h.x, dx * b.x);
    n.y = fmaf(ex2(dt * decay_rate(a.y)), h.y, dx * b.y);
    n.z = fmaf(ex2(dt * decay_rate(a.z)), h.z, dx * b.z);
    n.w = fmaf(ex2(dt * decay_rate(a.w)), h.w, dx * b.w);
    float y = fmaf(c.x, n.x, c.y * n.y) + fmaf(c.z, n.z, c.w * n.w);
#pragma unroll
    for (int o = 1; o < R; o <<= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
    if (!live) return;
    *reinterpret_cast<float4 *>(p.state_out + st) = n;
    if (r == 0) {
        y = fmaf(p.dsk ? p.dsk[ch] : 0.f, x, y);
        if (p.z) y *= gate_f(load1(static_cast<const TI *>(p.z) + (size_t)s * p.zs + ch));
        store1(static_cast<TO *>(p.y) + (size_t)s * p.D + ch, y);
    }
}

// ------------------------------------------------------------------------------------------------ backward

struct ScanBwdParams {
    ScanParams f;
    const void *dy;
    long long dys;
    const float *d_state_out;
    void *d_x, *d_dt, *d_z;
    float *d_state_in;
    float *part_bc;     // [channel blocks][T][2 N]: dB | dC of one block's channels
    float *part_a;      // [S][D][N]
    float *part_d;      // [S][2][D]: d_skip, d_dt_bias
};

// Tiles of kCkptTok tokens from the last to the first.  With e_t = a_t g_t, the gradient that reaches h_{t-1},
//   g_t = c_t dy_t + e_{t+1},   e_t = exp(dt_t a) g_t,
// which is the forward recurrence run backwards, so the slices of a tile meet in the same way in both directions.  h is
// scanned again from the tile's checkpoint; decays and states of a slice (8 tokens x 4 states each) stay in registers.
// The sums over channels that dB and dC need are folded over the warp's channel lanes by halves (each fold sends one half
// of the values away and keeps the other), then over the CTA's channel warps in shared memory, and leave as one partial
// sum per channel block for selscan_bc_kernel: no atomics, so equal calls give equal bits.
template <typename TI, typename TG, int N, int WD>
__global__ void __launch_bounds__(32 * WD * 4) selscan_bwd_kernel(const ScanBwdParams q)
{
    constexpr int WT = 4, TOK = 8, TILE = WT * TOK;
    static_assert(TILE == kCkptTok, "one tile per checkpoint");
    constexpr int R = N / 4, CPW = 32 / R, DC = CPW * WD, NT = 32 * WD * WT;
    constexpr int NV = TILE * DC / 4, VPT = (NV + NT - 1) / NT;
    constexpr int NB = TILE * N / 4, BPT = (NB + NT - 1) / NT;
    constexpr int YP = TILE * DC + 8;
    constexpr int LEFT = CPW >= 8 ? 1 : 8 / CPW;                        // dB, dC values a lane is left with
    const ScanParams &p = q.f;
    extern __shared__ __align__(16) unsigned char smem[];
    float4 *s_in = reinterpret_cast<float4 *>(smem);                   // [TILE][DC] dt, dt x, dy silu(z), -
    float *s_b = reinterpret_cast<float *>(s_in + TILE * DC);          // [TILE][N]
    float *s_c = s_b + TILE * N;
    float *s_y = s_c + TILE * N;                                       // [3][R][YP]: <c,h>, <g,b>, sum g a h_prev A
    float4 *s_p = reinterpret_cast<float4 *>(s_y + 3 * R * YP);        // [WT][WD * 32]
    float4 *s_h = s_p + WT * WD * 32;
    float4 *s_e = s_h + WT * WD * 32;
    float *s_bc = reinterpret_cast<float *>(s_e + WT * WD * 32);       // [WD][TILE][2 N]
    static_assert((R * YP) % 4 == 0, "16-byte aligned planes");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int wd = warp % WD, wt = warp / WD;
    const int nblk = (p.D + DC - 1) / DC;
    const int s = blockIdx.x / nblk, cb = blockIdx.x % nblk, c0 = cb * DC;
    const int cl_ = lane / R, chl = wd * CPW + cl_, r = lane % R, ch = c0 + chl;
    const bool live = ch < p.D;
    const SeqRange sr = seq_range(p.off, s, p.S, p.T);
    const int g_ = p.G == 1 ? 0 : c0 / (p.D / p.G);
    const int slot = wd * 32 + lane;

    const TI *px = static_cast<const TI *>(p.x), *pdt = static_cast<const TI *>(p.dt), *pz = static_cast<const TI *>(p.z);
    const TI *pdy = static_cast<const TI *>(q.dy);
    const TI *pb = static_cast<const TI *>(p.b) + g_ * N, *pc = static_cast<const TI *>(p.c) + g_ * N;

    float4 a = zero4(), ar = zero4(), ecarry = zero4();
    float2 da01 = make_float2(0.f, 0.f), da23 = da01;
    const size_t st = ((size_t)s * p.D + ch) * N + 4 * r;
    if (live) {
        ar = *reinterpret_cast<const float4 *>(p.a + (size_t)ch * N + 4 * r);
        a = make_float4(decay_rate(ar.x), decay_rate(ar.y), decay_rate(ar.z), decay_rate(ar.w));
        if (q.d_state_out) ecarry = *reinterpret_cast<const float4 *>(q.d_state_out + st);
    }
    const float2 a01 = make_float2(a.x, a.y), a23 = make_float2(a.z, a.w);
    float4 acc_d[VPT], acc_b[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) acc_d[i] = acc_b[i] = zero4();

    const int ntile = (sr.len + TILE - 1) / TILE;
    for (int tile = ntile - 1; tile >= 0; --tile) {
        const int t0 = tile * TILE;
        float4 kx[VPT], kz[VPT], kdy[VPT], kraw[VPT];
        __syncthreads();   // the previous tile's readers of shared memory are done
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = tid + i * NT, t = t0 + v / (DC / 4), cl = 4 * (v % (DC / 4));
            kx[i] = kz[i] = kdy[i] = kraw[i] = zero4();
            if (v < NV) {
                float4 d = zero4(), dg = zero4();
                if (t < sr.len && c0 + cl < p.D) {
                    const size_t row = (size_t)(sr.start + t);
                    kx[i] = load4(px + row * p.xs + c0 + cl);
                    kdy[i] = load4(pdy + row * q.dys + c0 + cl);
                    d = load4(pdt + row * p.dts + c0 + cl);
                    const float4 bias = opt4(p.bias, c0 + cl, 0.f);
                    d = make_float4(d.x + bias.x, d.y + bias.y, d.z + bias.z, d.w + bias.w);
                    kraw[i] = d;
                    if (p.softplus) d = make_float4(softplus_acc(d.x), softplus_acc(d.y), softplus_acc(d.z), softplus_acc(d.w));
                    dg = kdy[i];
                    if (pz) {
                        kz[i] = load4(pz + row * p.zs + c0 + cl);
                        dg = make_float4(dg.x * gate_f(kz[i].x), dg.y * gate_f(kz[i].y), dg.z * gate_f(kz[i].z), dg.w * gate_f(kz[i].w));
                    }
                }
                float4 *o = s_in + (v / (DC / 4)) * DC + cl;
                o[0] = make_float4(d.x, d.x * kx[i].x, dg.x, 0.f);
                o[1] = make_float4(d.y, d.y * kx[i].y, dg.y, 0.f);
                o[2] = make_float4(d.z, d.z * kx[i].z, dg.z, 0.f);
                o[3] = make_float4(d.w, d.w * kx[i].w, dg.w, 0.f);
            }
        }
#pragma unroll
        for (int i = 0; i < BPT; ++i) {
            const int v = tid + i * NT, t = t0 + v / (N / 4), n = 4 * (v % (N / 4));
            if (v < NB) {
                float4 bv = zero4(), cv = zero4();
                if (t < sr.len) {
                    const size_t row = (size_t)(sr.start + t);
                    bv = load4(pb + row * p.bs + n);
                    cv = load4(pc + row * p.cs + n);
                }
                reinterpret_cast<float4 *>(s_b)[v] = bv;
                reinterpret_cast<float4 *>(s_c)[v] = cv;
            }
        }
        float4 hin = zero4();
        if (live) hin = *reinterpret_cast<const float4 *>(p.ckpt + (((size_t)(sr.start / kCkptTok) + s + tile) * p.D + ch) * N + 4 * r);
        __syncthreads();

        // states of this slice from zero; the gradient that leaves its front, likewise
        float2 e01[TOK], e23[TOK], h01[TOK], h23[TOK];
        float2 hh01 = make_float2(0.f, 0.f), hh23 = hh01, p01 = make_float2(1.f, 1.f), p23 = p01;
#pragma unroll
        for (int i = 0; i < TOK; ++i) {
            const int t = wt * TOK + i;
            const float4 in = s_in[t * DC + chl];
            const float4 bv = *reinterpret_cast<const float4 *>(s_b + t * N + 4 * r);
            float2 x01 = mul2v(a01, splat2(in.x)), x23 = mul2v(a23, splat2(in.x));
            e01[i] = make_float2(ex2(x01.x), ex2(x01.y));
            e23[i] = make_float2(ex2(x23.x), ex2(x23.y));
            hh01 = fma2v(e01[i], hh01, mul2v(splat2(in.y), make_float2(bv.x, bv.y)));
            hh23 = fma2v(e23[i], hh23, mul2v(splat2(in.y), make_float2(bv.z, bv.w)));
            h01[i] = hh01;
            h23[i] = hh23;
            p01 = mul2v(p01, e01[i]);
            p23 = mul2v(p23, e23[i]);
        }
        float2 g01 = make_float2(0.f, 0.f), g23 = g01;
#pragma unroll
        for (int i = TOK - 1; i >= 0; --i) {
            const int t = wt * TOK + i;
            const float dg = reinterpret_cast<const float *>(s_in + t * DC + chl)[2];
            const float4 cv = *reinterpret_cast<const float4 *>(s_c + t * N + 4 * r);
            g01 = mul2v(e01[i], fma2v(make_float2(cv.x, cv.y), splat2(dg), g01));
            g23 = mul2v(e23[i], fma2v(make_float2(cv.z, cv.w), splat2(dg), g23));
        }
        s_p[wt * (WD * 32) + slot] = make_float4(p01.x, p01.y, p23.x, p23.y);
        s_h[wt * (WD * 32) + slot] = make_float4(hh01.x, hh01.y, hh23.x, hh23.y);
        s_e[wt * (WD * 32) + slot] = make_float4(g01.x, g01.y, g23.x, g23.y);
        __syncthreads();
        // state before this slice, gradient behind it
#pragma unroll
        for (int w = 0; w < WT - 1; ++w) {
            if (w < wt) {
                const float4 pw = s_p[w * (WD * 32) + slot], hw = s_h[w * (WD * 32) + slot];
                hin = make_float4(fmaf(pw.x, hin.x, hw.x), fmaf(pw.y, hin.y, hw.y), fmaf(pw.z, hin.z, hw.z), fmaf(pw.w, hin.w, hw.w));
            }
        }
        float4 ein = ecarry;
#pragma unroll
        for (int w = WT - 1; w >= 0; --w) {
            if (w == wt) ein = ecarry;
            const float4 pw = s_p[w * (WD * 32) + slot], ew = s_e[w * (WD * 32) + slot];
            ecarry = make_float4(fmaf(pw.x, ecarry.x, ew.x), fmaf(pw.y, ecarry.y, ew.y), fmaf(pw.z, ecarry.z, ew.z),
                                 fmaf(pw.w, ecarry.w, ew.w));
        }
        const float2 in01 = make_float2(hin.x, hin.y), in23 = make_float2(hin.z, hin.w);
        float2 f01 = in01, f23 = in23;
#pragma unroll
        for (int i = 0; i < TOK; ++i) {
            const int t = wt * TOK + i;
            const float4 cv = *reinterpret_cast<const float4 *>(s_c + t * N + 4 * r);
            f01 = mul2v(f01, e01[i]);
            f23 = mul2v(f23, e23[i]);
            h01[i] = add2v(h01[i], f01);
            h23[i] = add2v(h23[i], f23);
            const float2 yy = fma2v(make_float2(cv.z, cv.w), h23[i], mul2v(make_float2(cv.x, cv.y), h01[i]));
            s_y[r * YP + t * DC + chl] = yy.x + yy.y;
        }
        g01 = make_float2(ein.x, ein.y);
        g23 = make_float2(ein.z, ein.w);
#pragma unroll
        for (int i = TOK - 1; i >= 0; --i) {
            const int t = wt * TOK + i;
            const float4 in = s_in[t * DC + chl];
            const float4 bv = *reinterpret_cast<const float4 *>(s_b + t * N + 4 * r);
            const float4 cv = *reinterpret_cast<const float4 *>(s_c + t * N + 4 * r);
            g01 = fma2v(make_float2(cv.x, cv.y), splat2(in.z), g01);
            g23 = fma2v(make_float2(cv.z, cv.w), splat2(in.z), g23);
            float v[8];
            {
                const float2 d01 = mul2v(g01, splat2(in.y)), d23 = mul2v(g23, splat2(in.y));
                const float2 k01 = mul2v(h01[i], splat2(in.z)), k23 = mul2v(h23[i], splat2(in.z));
                v[0] = d01.x; v[1] = d01.y; v[2] = d23.x; v[3] = d23.y;
                v[4] = k01.x; v[5] = k01.y; v[6] = k23.x; v[7] = k23.y;
            }
            const float2 gb = fma2v(g23, make_float2(bv.z, bv.w), mul2v(g01, make_float2(bv.x, bv.y)));
            g01 = mul2v(g01, e01[i]);   // e_t
            g23 = mul2v(g23, e23[i]);
            const float2 k01 = mul2v(g01, i ? h01[i ? i - 1 : 0] : in01), k23 = mul2v(g23, i ? h23[i ? i - 1 : 0] : in23);
            const float2 sa = fma2v(k23, make_float2(ar.z, ar.w), mul2v(k01, make_float2(ar.x, ar.y)));
            da01 = fma2v(k01, splat2(in.x), da01);
            da23 = fma2v(k23, splat2(in.x), da23);
            s_y[(R + r) * YP + t * DC + chl] = gb.x + gb.y;
            s_y[(2 * R + r) * YP + t * DC + chl] = sa.x + sa.y;
            // fold the 8 sums over the warp's channels
            int first = 0, n = 8;
#pragma unroll
            for (int o = 16; o >= R; o >>= 1) {
                if (n > 1) {
                    n >>= 1;
                    const bool up = lane & o;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j < n) {
                            const float send = up ? v[j] : v[j + n], keep = up ? v[j + n] : v[j];
                            v[j] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                        }
                    }
                    if (up) first += n;
                } else {
                    v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
                }
            }
            if (CPW <= 8 || (cl_ & (CPW / 8 - 1)) == 0) {
#pragma unroll
                for (int j = 0; j < LEFT; ++j) {
                    const int k = first + j;
                    s_bc[(wd * TILE + t) * (2 * N) + (k >> 2) * N + 4 * r + (k & 3)] = v[j];
                }
            }
        }
        __syncthreads();
        for (int v = tid; v < TILE * 2 * N / 4; v += NT) {
            const int t = v / (2 * N / 4);
            if (t0 + t >= sr.len) break;
            float4 o = reinterpret_cast<const float4 *>(s_bc)[v];
#pragma unroll
            for (int w = 1; w < WD; ++w) {
                const float4 k = reinterpret_cast<const float4 *>(s_bc + w * TILE * 2 * N)[v];
                o.x += k.x; o.y += k.y; o.z += k.z; o.w += k.w;
            }
            *reinterpret_cast<float4 *>(q.part_bc + ((size_t)cb * p.T + sr.start + t0) * (2 * N) + 4 * (size_t)v) = o;
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = tid + i * NT, t = t0 + v / (DC / 4), cl = 4 * (v % (DC / 4));
            if (v < NV && t < sr.len && c0 + cl < p.D) {
                float4 sums[3];
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    sums[k] = zero4();
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        const float4 part = *reinterpret_cast<const float4 *>(s_y + (k * R + j) * YP + 4 * v);
                        sums[k].x += part.x; sums[k].y += part.y; sums[k].z += part.z; sums[k].w += part.w;
                    }
                }
                const float4 dv = opt4(p.dsk, c0 + cl, 0.f);
                const size_t o = (size_t)(sr.start + t) * p.D + c0 + cl;
                float4 ox, odt, oz;
                auto one = [&](float x, float z, float dy, float raw, float dsk, float yh, float gb, float sa, float &rx, float &rdt,
                               float &rz, float &sd, float &sbias) {
                    float dg = dy;
                    if (pz) {
                        const float sg = sigmoid_acc(z);
                        dg = dy * (z * sg);
                        rz = dy * fmaf(dsk, x, yh) * (sg * fmaf(z, 1.f - sg, 1.f));
                    }
                    const float dt = p.softplus ? softplus_acc(raw) : raw;
                    rx = fmaf(dt, gb, dsk * dg);
                    rdt = fmaf(x, gb, sa);
                    if (p.softplus) rdt *= sigmoid_acc(raw);
                    sd = fmaf(dg, x, sd);
                    sbias += rdt;
                };
                one(kx[i].x, kz[i].x, kdy[i].x, kraw[i].x, dv.x, sums[0].x, sums[1].x, sums[2].x, ox.x, odt.x, oz.x, acc_d[i].x, acc_b[i].x);
                one(kx[i].y, kz[i].y, kdy[i].y, kraw[i].y, dv.y, sums[0].y, sums[1].y, sums[2].y, ox.y, odt.y, oz.y, acc_d[i].y, acc_b[i].y);
                one(kx[i].z, kz[i].z, kdy[i].z, kraw[i].z, dv.z, sums[0].z, sums[1].z, sums[2].z, ox.z, odt.z, oz.z, acc_d[i].z, acc_b[i].z);
                one(kx[i].w, kz[i].w, kdy[i].w, kraw[i].w, dv.w, sums[0].w, sums[1].w, sums[2].w, ox.w, odt.w, oz.w, acc_d[i].w, acc_b[i].w);
                store4(static_cast<TG *>(q.d_x) + o, ox);
                store4(static_cast<TG *>(q.d_dt) + o, odt);
                if (pz) store4(static_cast<TG *>(q.d_z) + o, oz);
            }
        }
    }
    if (q.d_state_in && live && wt == 0) *reinterpret_cast<float4 *>(q.d_state_in + st) = ecarry;
    // this sequence's share of the parameters' gradients
    __syncthreads();
    s_p[wt * (WD * 32) + slot] = make_float4(da01.x, da01.y, da23.x, da23.y);
    float4 *s_acc = reinterpret_cast<float4 *>(s_y);   // [2][NT * VPT]
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = tid + i * NT;
        if (v < NV) {
            s_acc[v] = acc_d[i];
            s_acc[NV + v] = acc_b[i];
        }
    }
    __syncthreads();
    if (live && wt == 0) {
        float4 o = zero4();
#pragma unroll
        for (int w = 0; w < WT; ++w) {
            const float4 k = s_p[w * (WD * 32) + slot];
            o.x += k.x; o.y += k.y; o.z += k.z; o.w += k.w;
        }
        *reinterpret_cast<float4 *>(q.part_a + st) = o;
    }
    for (int v = tid; v < 2 * DC / 4; v += NT) {
        const int which = v / (DC / 4), cq = v % (DC / 4);
        if (c0 + 4 * cq < p.D) {
            float4 o = zero4();
            for (int t = 0; t < TILE; ++t) {
                const float4 k = s_acc[which * NV + t * (DC / 4) + cq];
                o.x += k.x; o.y += k.y; o.z += k.z; o.w += k.w;
            }
            *reinterpret_cast<float4 *>(q.part_d + ((size_t)s * 2 + which) * p.D + c0 + 4 * cq) = o;
        }
    }
}

// dB, dC: sum of the channel blocks' partial sums, rounded once
template <typename TG, int N>
__global__ void __launch_bounds__(256) selscan_bc_kernel(const float *part, void *d_b, void *d_c, const int *off, int S, int T, int G,
                                                         int blocks_per_group)
{
    const size_t per_tok = (size_t)G * (2 * N / 4);
    const int end = seq_start(off, S, S, T);
    for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < (size_t)end * per_tok; i += (size_t)gridDim.x * blockDim.x) {
        const size_t t = i / per_tok;
        const int rest = (int)(i % per_tok), g = rest / (2 * N / 4), v = rest % (2 * N / 4);
        float4 o = zero4();
        for (int k = 0; k < blocks_per_group; ++k) {
            const float4 u = *reinterpret_cast<const float4 *>(part + ((size_t)(g * blocks_per_group + k) * T + t) * (2 * N) + 4 * v);
            o.x += u.x; o.y += u.y; o.z += u.z; o.w += u.w;
        }
        const bool is_c = v >= N / 4;
        store4(static_cast<TG *>(is_c ? d_c : d_b) + (t * G + g) * N + 4 * (v - (is_c ? N / 4 : 0)), o);
    }
}

// sums over the sequences: out[i] = sum_s part[s * stride + i]
__global__ void __launch_bounds__(256) sum_rows_kernel(const float *part, float *out, int S, size_t stride, size_t n)
{
    const size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x;
    if (i >= n) return;
    float o = 0.f;
    for (int s = 0; s < S; ++s) o += part[(size_t)s * stride + i];
    out[i] = o;
}

// ------------------------------------------------------------------------------------------------ launches

// Tokens of a segment, 0 = whole sequences.  A split costs a second pass over x, dt, b (their decays evaluated twice, 1.9
// times the exponentials), so it pays only where the chains leave more than half of the SMs without work.
int fwd_segment(int T, int S, int D, int N)
{
    const int cpw = N <= 16 ? 32 : 512 / N;
    const long long cols = (D + cpw - 1) / cpw, chains = cols * S;
    if (chains * 2 > 148 || T / S < 512) return 0;
    const long long want = (2 * 148 + cols - 1) / cols;   // segments in all
    const long long seg = (T + want - 1) / want;
    return (int)((seg < 256 ? 256 : seg + 127) / 128 * 128);
}

template <typename TI, typename TO, int N, int CH, int TOK, int WT, int OCC>
chela_status_t fwd_launch(ScanParams p, cudaStream_t stream)
{
    using Sh = FwdShape<TI, N, CH, TOK>;
    constexpr size_t smem = (size_t)WT * Sh::WARP_B;
    const auto kern = selscan_fwd_kernel<TI, TO, N, CH, TOK, WT, OCC>;
    if (smem > 47 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return cuda_status(e);
    }
    const long long chains = p.seg ? (long long)packed_blocks(p.T, p.S, p.seg) : p.S;
    const long long blocks = chains * ((p.D + Sh::CPW - 1) / Sh::CPW);
    if (blocks > 0x7fffffffLL) return CHELA_ERR_UNSUPPORTED;
    if (p.seg) {
        ScanParams q = p;
        q.y = nullptr;
        q.ckpt = q.state_out = nullptr;
        kern<<<(unsigned)blocks, 32 * WT, smem, stream>>>(q);
        const long long n = ((long long)p.S * p.D * N + 127) / 128;
        if (n > 0x7fffffffLL) return CHELA_ERR_UNSUPPORTED;
        selscan_segments_kernel<N><<<(unsigned)n, 128, 0, stream>>>(p);
        p.seg_sum = nullptr;
    }
    kern<<<(unsigned)blocks, 32 * WT, smem, stream>>>(p);
    return last_launch_status();
}

template <typename TI, typename TO>
chela_status_t fwd_n(const ScanParams &p, int N, cudaStream_t stream)
{
    switch (N) {
    case 8: return fwd_launch<TI, TO, 8, 1, 8, 8, 2>(p, stream);
    case 16: return fwd_launch<TI, TO, 16, 2, 4, 8, 2>(p, stream);
    case 32: return fwd_launch<TI, TO, 32, 2, 4, 8, 2>(p, stream);
    default: return fwd_launch<TI, TO, 64, 2, 4, 8, 2>(p, stream);
    }
}

template <typename TI, typename TO>
chela_status_t step_n(const ScanParams &p, int N, cudaStream_t stream)
{
    const size_t threads = (size_t)p.S * p.D * (N / 4);
    const size_t blocks = (threads + 255) / 256;
    if (blocks > 0x7fffffffULL) return CHELA_ERR_UNSUPPORTED;
    switch (N) {
    case 8: selscan_step_kernel<TI, TO, 8><<<(unsigned)blocks, 256, 0, stream>>>(p); break;
    case 16: selscan_step_kernel<TI, TO, 16><<<(unsigned)blocks, 256, 0, stream>>>(p); break;
    case 32: selscan_step_kernel<TI, TO, 32><<<(unsigned)blocks, 256, 0, stream>>>(p); break;
    default: selscan_step_kernel<TI, TO, 64><<<(unsigned)blocks, 256, 0, stream>>>(p); break;
    }
    return last_launch_status();
}

constexpr int bwd_wd(int N) { return N == 8 ? 2 : 4; }
constexpr int bwd_channels(int N) { return 32 / (N / 4) * bwd_wd(N); }   // channels of a CTA: 32, 32, 16, 8

template <typename TI, typename TG, int N>
chela_status_t bwd_launch(const ScanBwdParams &q, void *d_b, void *d_c, float *d_a, float *d_skip, float *d_bias, cudaStream_t stream)
{
    const ScanParams &p = q.f;
    constexpr int WD = bwd_wd(N), R = N / 4, DC = bwd_channels(N), TILE = kCkptTok, WT = 4;
    constexpr size_t smem = (size_t)TILE * DC * 16 + 2 * TILE * N * 4 + 3 * R * (TILE * DC + 8) * 4 + 3 * WT * WD * 32 * 16 +
                            (size_t)WD * TILE * 2 * N * 4;
    const auto kern = selscan_bwd_kernel<TI, TG, N, WD>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return cuda_status(e);
    const int nblk = (p.D + DC - 1) / DC;
    const long long blocks = (long long)p.S * nblk;
    if (blocks > 0x7fffffffLL) return CHELA_ERR_UNSUPPORTED;
    kern<<<(unsigned)blocks, 32 * WD * WT, smem, stream>>>(q);
    chela_status_t st = last_launch_status();
    if (st != CHELA_OK) return st;
    const size_t items = (size_t)p.T * p.G * (2 * N / 4);
    const size_t grid = (items + 255) / 256;
    selscan_bc_kernel<TG, N><<<(unsigned)(grid < 148 * 32 ? grid : 148 * 32), 256, 0, stream>>>(q.part_bc, d_b, d_c, p.off, p.S, p.T, p.G, nblk / p.G);
    st = last_launch_status();
    auto rows = [&](const float *part, float *out, size_t stride, size_t n) {
        if (st != CHELA_OK || !out) return;
        sum_rows_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(part, out, p.S, stride, n);
        st = last_launch_status();
    };
    rows(q.part_a, d_a, (size_t)p.D * N, (size_t)p.D * N);
    rows(q.part_d, d_skip, (size_t)2 * p.D, p.D);
    rows(q.part_d + p.D, d_bias, (size_t)2 * p.D, p.D);
    return st;
}

template <typename TI, typename TG>
chela_status_t bwd_n(const ScanBwdParams &q, int N, void *d_b, void *d_c, float *d_a, float *d_skip, float *d_bias, cudaStream_t stream)
{
    switch (N) {
    case 8: return bwd_launch<TI, TG, 8>(q, d_b, d_c, d_a, d_skip, d_bias, stream);
    case 16: return bwd_launch<TI, TG, 16>(q, d_b, d_c, d_a, d_skip, d_bias, stream);
    case 32: return bwd_launch<TI, TG, 32>(q, d_b, d_c, d_a, d_skip, d_bias, stream);
    default: return bwd_launch<TI, TG, 64>(q, d_b, d_c, d_a, d_skip, d_bias, stream);
    }
}

ScanParams scan_params(const chela_selscan_args_t &a)
{
    ScanParams p = {};
    p.x = a.x; p.dt = a.dt; p.b = a.b; p.c = a.c; p.z = a.z;
    p.xs = a.x_stride; p.dts = a.dt_stride; p.bs = a.b_stride; p.cs = a.c_stride; p.zs = a.z_stride;
    p.a = a.a; p.dsk = a.d_skip; p.bias = a.dt_bias;
    p.state_in = a.state_in;
    p.off = a.seq_offsets;
    p.S = a.S; p.T = a.T; p.D = a.D; p.G = a.G; p.softplus = a.softplus;
    return p;
}

struct ScanBwdPlan {
    size_t off_ckpt, off_fwd, off_bc, off_a, off_d, total;
};
ScanBwdPlan bwd_plan(int T, int S, int D, int N, bool have_ckpt)
{
    ScanBwdPlan p;
    const int dc = bwd_channels(N);
    p.off_ckpt = 0;
    p.off_fwd = have_ckpt ? 0 : align_up(selscan_checkpoint_bytes(T, S, D, N), 256);
    p.off_bc = p.off_fwd + (have_ckpt ? 0 : selscan_workspace_bytes(T, S, D, N));
    p.off_a = p.off_bc + align_up((size_t)((D + dc - 1) / dc) * T * 2 * N * sizeof(float), 256);
    p.off_d = p.off_a + align_up((size_t)S * D * N * sizeof(float), 256);
    p.total = p.off_d + align_up((size_t)S * 2 * D * sizeof(float), 256);
    return p;
}

}  // namespace

size_t selscan_checkpoint_bytes(int T, int S, int D, int N)
{
    return (packed_blocks(T, S, kCkptTok)) * D * N * sizeof(float);
}

size_t selscan_workspace_bytes(int T, int S, int D, int N)
{
    const int seg = fwd_segment(T, S, D, N);
    return seg ? align_up(packed_blocks(T, S, seg) * D * (N + 1) * sizeof(float), 256) : 0;
}

chela_status_t launch_selscan_fwd(const chela_selscan_args_t &a, void *y, float *state_out, void *ckpt, chela_dtype_t out_dtype,
                                  void *workspace, cudaStream_t stream)
{
    ScanParams p = scan_params(a);
    p.y = y;
    p.state_out = state_out;
    p.ckpt = static_cast<float *>(ckpt);
    p.seg = fwd_segment(a.T, a.S, a.D, a.N);
    if (p.seg) {
        p.seg_state = static_cast<float *>(workspace);
        p.seg_sum = p.seg_state + packed_blocks(a.T, a.S, p.seg) * a.D * a.N;
    }
    if (a.in_dtype == CHELA_F32)
        return out_dtype == CHELA_F32 ? fwd_n<float, float>(p, a.N, stream) : fwd_n<float, __nv_bfloat16>(p, a.N, stream);
    return out_dtype == CHELA_F32 ? fwd_n<__nv_bfloat16, float>(p, a.N, stream) : fwd_n<__nv_bfloat16, __nv_bfloat16>(p, a.N, stream);
}

chela_status_t launch_selscan_step(const chela_selscan_args_t &a, void *y, float *state_out, chela_dtype_t out_dtype, cudaStream_t stream)
{
    ScanParams p = scan_params(a);
    p.y = y;
    p.state_out = state_out;
    if (a.in_dtype == CHELA_F32)
        return out_dtype == CHELA_F32 ? step_n<float, float>(p, a.N, stream) : step_n<float, __nv_bfloat16>(p, a.N, stream);
    return out_dtype == CHELA_F32 ? step_n<__nv_bfloat16, float>(p, a.N, stream) : step_n<__nv_bfloat16, __nv_bfloat16>(p, a.N, stream);
}

size_t selscan_bwd_workspace_bytes(int T, int S, int D, int N, bool have_ckpt) { return bwd_plan(T, S, D, N, have_ckpt).total; }

chela_status_t launch_selscan_bwd(const chela_selscan_args_t &a, const void *d_y, long long d_y_stride, const float *d_state_out,
                                  const void *ckpt, void *d_x, void *d_dt, float *d_a, void *d_b, void *d_c, float *d_skip, void *d_z,
                                  float *d_bias, float *d_state_in, chela_dtype_t grad_dtype, void *workspace, cudaStream_t stream)
{
    const ScanBwdPlan w = bwd_plan(a.T, a.S, a.D, a.N, ckpt != nullptr);
    char *ws = static_cast<char *>(workspace);
    ScanBwdParams q = {};
    q.f = scan_params(a);
    q.f.ckpt = static_cast<float *>(const_cast<void *>(ckpt));
    if (!ckpt) {
        q.f.ckpt = reinterpret_cast<float *>(ws + w.off_ckpt);
        const chela_status_t st = launch_selscan_fwd(a, nullptr, nullptr, q.f.ckpt, CHELA_F32, ws + w.off_fwd, stream);
        if (st != CHELA_OK) return st;
    }
    q.dy = d_y;
    q.dys = d_y_stride;
    q.d_state_out = d_state_out;
    q.d_x = d_x; q.d_dt = d_dt; q.d_z = d_z;
    q.d_state_in = d_state_in;
    q.part_bc = reinterpret_cast<float *>(ws + w.off_bc);
    q.part_a = reinterpret_cast<float *>(ws + w.off_a);
    q.part_d = reinterpret_cast<float *>(ws + w.off_d);
    if (a.in_dtype == CHELA_F32)
        return grad_dtype == CHELA_F32 ? bwd_n<float, float>(q, a.N, d_b, d_c, d_a, d_skip, d_bias, stream)
                                       : bwd_n<float, __nv_bfloat16>(q, a.N, d_b, d_c, d_a, d_skip, d_bias, stream);
    return grad_dtype == CHELA_F32 ? bwd_n<__nv_bfloat16, float>(q, a.N, d_b, d_c, d_a, d_skip, d_bias, stream)
                                   : bwd_n<__nv_bfloat16, __nv_bfloat16>(q, a.N, d_b, d_c, d_a, d_skip, d_bias, stream);
}

}  // namespace chela
