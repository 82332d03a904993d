// Selective state space scan over packed sequences:
//   h_t[n] = exp(dt_t a[c,n]) h_{t-1}[n] + dt_t b_t[n] x_t,   y_t = (<c_t, h_t> + d_skip x_t) silu(z_t)   per channel c.
//
// What bounds it: N exponentials a token and channel against 8 bytes of bf16 operands.  An SM evaluates 16 exponentials
// a cycle, so N = 16 costs 1.2 cycles a token and channel (with softplus and the gate) where its share of the measured
// HBM rate needs 0.36; beside them 3 N multiply-adds, and the shared memory traffic of b and c, which every channel
// reads.  8 x 8192 x 1024 in bf16: 285 us of exponentials, 83 us of HBM traffic, 550 us measured.
//
// Layout of the work: a lane holds 8 states of one or two channels; the warps of a CTA take turns with short slices of the
// same channels' tokens.  Everything but the recurrence itself (copies, exponentials, outputs) is done beside the other
// warps' turns; the state passes from warp to warp through shared memory.  Where that leaves SMs without work, sequences
// are split into segments, whose ends are found from zero states first.  The backward pass walks tiles of 8 tokens from
// checkpoints of the state, the last tile first, in the same manner.
#include "packed.cuh"

namespace chela {
namespace {

constexpr int kCkptTok = 8;   // tokens between checkpoints; also the tile of the backward kernel

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
// a log2(e), minus infinity replaced by the lowest finite value: exp(dt a) is 0 for dt > 0 all the same, and the tokens
// past a sequence's end (dt = 0) keep the state instead of producing 0 * infinity
__device__ __forceinline__ float decay_rate(float a)
{
    const float v = a * kLog2e;
    return v < -3.0e38f ? -3.0e38f : v;
}
// sum += v with the digits that the sum loses carried along (Kahan): a long sequence adds thousands of tiles to one lane
__device__ __forceinline__ void compensated(float &sum, float &lost, float v)
{
    const float y = __fsub_rn(v, lost), t = __fadd_rn(sum, y);
    lost = __fsub_rn(__fsub_rn(t, sum), y);
    sum = t;
}
__device__ __forceinline__ float gate_f(float z) { return z * sigmoid_acc(z); }

// Channels of a warp (and of a chain) in both kernels, and the checkpoints' layout, which is the warps' own: for each
// checkpoint and chain, [CH NS / 4][32 lanes] vectors of four states, so that a warp writes and reads whole lines.
__host__ __device__ constexpr int chain_ch(int N) { return N == 8 ? 1 : 2; }
__host__ __device__ constexpr int chain_channels(int N) { return 32 / (N / 8) * chain_ch(N); }   // 32, 32, 16, 8
__device__ __forceinline__ float4 *ckpt_at(float *ckpt, size_t index, int chains, int chain, int per_lane)
{
    return reinterpret_cast<float4 *>(ckpt) + (index * chains + chain) * (size_t)(per_lane * 32);
}

// ------------------------------------------------------------------------------------------------ forward

__device__ __forceinline__ void named_sync(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void named_arrive(int id) { asm volatile("bar.arrive %0, 64;" ::"r"(id) : "memory"); }
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
// Two pools of work run beside each other here, exponentials (8 cycles a warp instruction) with the shared memory traffic
// behind the same queue, and the multiply-adds; neither is full (49 and 45 %): the warps wait for their turns (about 515
// cycles for four tokens), and taking away any one part changes the time by a few per cent only.  Two-wide multiply-adds of three different register pairs take 4.2 cycles of a
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
        if (b < 0 || (b > 0 && b > (sr.len - 1) / p.seg)) return;
        if (p.seg_sum && sr.len - b * p.seg <= p.seg) return;   // what a sequence's last segment ends with starts nothing
    } else {
        __shared__ int s_len[32 * WT + 1];
        s = seq_by_length(p.off, p.S, p.T, (int)blk, s_len);
        sr = seq_range(p.off, s, p.S, p.T);
    }
    // tokens of the sequence (a segment's end past the sequence's could pass 31 bits: the lengths are compared, not the ends)
    const int begin = b * p.seg, end = p.seg ? begin + min(p.seg, sr.len - begin) : sr.len;
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
    DecayShift shift[CH];
    float2 h[CH][NP];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        float2 rates[NP];
        const int cj = ch ^ j;   // pairs of channels start at even ones, so the neighbour is ch ^ 1
        const bool ok = cj < p.D;
        const size_t at = (size_t)cj * N + n0;
        // (a segment takes its state from seg_state, the first one too: state_in may be the buffer that the last one writes)
        const float *init = p.seg_sum ? nullptr : (p.seg && sr.len > 0 ? p.seg_state + (size_t)blk * p.D * N
                                                                       : (p.state_in ? p.state_in + (size_t)s * p.D * N : nullptr));
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
            rates[k] = make_float2(av.x, av.y);
            rates[k + 1] = make_float2(av.z, av.w);
            if (warp == 0) s_a[j * NP / 2 + k / 2][lane] = av;
        }
        shift[j].set(rates);
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
            if (R == 2 && CH == 2) return j == 0 ? v[i % PT] : __shfl_xor_sync(0xffffffffu, v[i % PT], 1);
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
            float2 near;
#pragma unroll
            for (int i = 0; i < TOK; ++i) {
                const float d = of(dt, i, j);
                if (i == 0) near = shift[j].at(d);
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const float2 v = fma2v(a[k], splat2(d), near);
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
        if (p.ckpt && t0 % kCkptTok == 0) {
            // the backward kernel's chain, lane and slot of this channel
            constexpr int BCH = chain_ch(N), BCPW = chain_channels(N);
            const int chains = (p.D + BCPW - 1) / BCPW, c = ch % BCPW;
            float4 *o = ckpt_at(p.ckpt, (size_t)(sr.start / kCkptTok) + s + t0 / kCkptTok, chains, ch / BCPW, BCH * NP / 2);
            if (BCH == CH) {
                o += lane;
#pragma unroll
                for (int j = 0; j < CH; ++j)
#pragma unroll
                    for (int k = 0; k < NP; k += 2) o[(j * NP / 2 + k / 2) * 32] = make_float4(h[j][k].x, h[j][k].y, h[j][k + 1].x, h[j][k + 1].y);
            } else if (live) {   // one channel here, two a lane there: slot 0 where the channel's parity is the lane's
                o += ((c ^ q) & 1) * (NP / 2) * 32 + c / 2 * R + q;
#pragma unroll
                for (int k = 0; k < NP; k += 2) o[(k / 2) * 32] = make_float4(h[0][k].x, h[0][k].y, h[0][k + 1].x, h[0][k + 1].y);
            }
        }
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
    for (int left = sr.len; left > 0; left -= p.seg, ++k) {   // tokens from here on; counted down, so that nothing passes 31 bits
        float *m = p.seg_state + (k * p.D + ch) * N + n;
        const bool more = left > p.seg;
        const float own = more ? *m : 0.f, time = more ? p.seg_sum[k * p.D + ch] : 0.f;
        *m = h;
        h = h == 0.f ? own : fmaf(ex2(a * time), h, own);   // growth over a segment may be infinite, its product with 0 is not NaN
    }
}

// ------------------------------------------------------------------------------------------------ single token

// A lane has 8 states of one channel: two 16-byte loads of the state are in flight, which is what this kernel is about
// (the state is read and written once, 8 bytes of traffic an element against 2 for everything else).
template <typename TI, typename TO, int N>
__global__ void __launch_bounds__(256) selscan_step_kernel(const ScanParams p)
{
    constexpr int R = N / 8;
    const size_t idx = blockIdx.x * (size_t)blockDim.x + threadIdx.x;
    const size_t row_ch = idx / R, all = (size_t)p.S * p.D;
    const int r = (int)(idx % R);
    const bool live = row_ch < all;
    // 32-bit division where that is enough
    const int s = !live ? 0 : (all <= 0x7fffffffu ? (int)((unsigned)row_ch / (unsigned)p.D) : (int)(row_ch / p.D));
    const int ch = live ? (int)(row_ch - (size_t)s * p.D) : 0;
    const int g = p.G == 1 ? 0 : ch / (p.D / p.G);
    const size_t st = ((size_t)s * p.D + ch) * N + 8 * r;
    const size_t wt = (size_t)ch * N + 8 * r, bt = (size_t)s * p.bs + g * N + 8 * r, ct = (size_t)s * p.cs + g * N + 8 * r;
    float4 h[2], a[2], b[2], c[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        h[k] = *reinterpret_cast<const float4 *>(p.state_in + st + 4 * k);
        a[k] = *reinterpret_cast<const float4 *>(p.a + wt + 4 * k);
        b[k] = load4(static_cast<const TI *>(p.b) + bt + 4 * k);
        c[k] = load4(static_cast<const TI *>(p.c) + ct + 4 * k);
    }
    const float x = load1(static_cast<const TI *>(p.x) + (size_t)s * p.xs + ch);
    float dt = load1(static_cast<const TI *>(p.dt) + (size_t)s * p.dts + ch) + (p.bias ? p.bias[ch] : 0.f);
    const float z = p.z ? load1(static_cast<const TI *>(p.z) + (size_t)s * p.zs + ch) : 0.f, skip = p.dsk ? p.dsk[ch] : 0.f;
    if (p.softplus) dt = softplus_acc(dt);
    const float dx = dt * x;
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        h[k].x = fmaf(decay(decay_rate(a[k].x), dt), h[k].x, dx * b[k].x);
        h[k].y = fmaf(decay(decay_rate(a[k].y), dt), h[k].y, dx * b[k].y);
        h[k].z = fmaf(decay(decay_rate(a[k].z), dt), h[k].z, dx * b[k].z);
        h[k].w = fmaf(decay(decay_rate(a[k].w), dt), h[k].w, dx * b[k].w);
        y += fmaf(c[k].x, h[k].x, c[k].y * h[k].y) + fmaf(c[k].z, h[k].z, c[k].w * h[k].w);
    }
#pragma unroll
    for (int o = 1; o < R; o <<= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
    if (!live) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) *reinterpret_cast<float4 *>(p.state_out + st + 4 * k) = h[k];
    if (r == 0) {
        y = fmaf(skip, x, y);
        if (p.z) y *= gate_f(z);
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

template <typename TI, int N, int CH>
struct BwdShape {
    static constexpr int NS = 8, NP = 4, R = N / NS, CPW = 32 / R * CH, E16 = 16 / (int)sizeof(TI), WT = 8, TOK = kCkptTok, SUB = 2;
    static constexpr int LPC = R / CH;                                  // lanes of one channel
    static constexpr int TS = SUB < LPC ? SUB : LPC, PT = SUB / TS, DUP = LPC / TS;   // see tok0
    static constexpr int XC = CPW / E16, BC = N / E16;
    static constexpr int CHUNKS = TOK * (4 * XC + 2 * BC), CPL = (CHUNKS + 31) / 32;
    static constexpr int RAW_E = CHUNKS * E16, PREP_F = 3 * TOK * CPW, BC_F = 2 * TOK * N, STATE_F = 32 * CH * NS;
    static constexpr int RAW_B = 2 * RAW_E * (int)sizeof(TI);           // two tiles, the next one's copy under way
    static constexpr int WARP_B = RAW_B + (PREP_F + BC_F + TOK / SUB * STATE_F + STATE_F) * 4;
    static constexpr size_t SMEM = (size_t)WT * WARP_B;
};

// With e_t = exp(dt_t a) g_t, the gradient that reaches h_{t-1}:  g_t = c_t dy_t + e_{t+1}.
// One CTA is a chain: CPW channels of a sequence, whose tiles of kCkptTok tokens its WT warps take in turn from the last
// to the first.  A warp runs its tile's states forwards from the checkpoint, keeping every second one in shared memory,
// and sums at the same time what the tile adds to the gradient that leaves its front, sum_t (prod_{s<=t} exp(dt_s a)) c_t
// dy_t, and the tile's whole decay.  When the gradient behind the tile has come in from the warp with the tile behind, the
// one before it (one multiply-add per state) goes on to the next warp, and the tile is run backwards two tokens at a
// time with their decays and states computed again in registers.  So the only serial part is that one step a tile, and
// few chains still fill the SMs; the second evaluation of the exponentials costs less than keeping the decays would.
// Eight warps an SM with 252 to 255 registers and no spills: twelve warps, which have 168 registers each and spill 170 to
// 230 bytes, took 640 to 740 us where eight took 490 (4 x 4096 x 1024).  However few the chains are, a sequence is not split:
// one of 32768 x 512 takes 3750 us on 16 SMs.
// Lanes as in the forward kernel: 8 states of CH channels, so that the sums over channels that dB and dC need are begun in
// the lane; they are folded over the other lanes (each exchange sends one half of the values away and keeps the other) and
// leave as one partial sum per channel block for selscan_bc_kernel: no atomics, so equal calls give equal bits.
template <typename TI, typename TG, int N, int CH>
__global__ void __launch_bounds__(32 * BwdShape<TI, N, CH>::WT, 1) selscan_bwd_kernel(const ScanBwdParams q_)
{
    using Sh = BwdShape<TI, N, CH>;
    constexpr int NS = Sh::NS, R = Sh::R, NP = Sh::NP, CPW = Sh::CPW, E16 = Sh::E16, XC = Sh::XC, BC = Sh::BC, CPL = Sh::CPL, PT = Sh::PT;
    constexpr int WT = Sh::WT, TOK = Sh::TOK, SUB = Sh::SUB, DUP = Sh::DUP, LPC = Sh::LPC;
    static_assert(XC >= 1 && BC >= 1 && R >= CH && SUB == 2 && TOK % LPC == 0 && WT <= 15, "shapes");
    const ScanParams &p = q_.f;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ longlong2 s_src[6];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned char *s_mine = smem + warp * Sh::WARP_B;
    TI *s_raw2 = reinterpret_cast<TI *>(s_mine);                         // two tiles: x, dt, z, dy [TOK][CPW], b, c [TOK][N]
    float *s_dt = reinterpret_cast<float *>(s_mine + Sh::RAW_B), *s_dx = s_dt + TOK * CPW, *s_dg = s_dx + TOK * CPW;
    float *s_bc = s_dt + Sh::PREP_F;                                     // b, c [TOK][N] in fp32
    float4 *s_keep = reinterpret_cast<float4 *>(s_bc + Sh::BC_F);        // states before tokens 0, 2, 4, 6: [CH NS / 4][32] each
    constexpr int HAND = Sh::WARP_B - Sh::STATE_F * 4;
    float4 *s_down = reinterpret_cast<float4 *>(s_mine + HAND);          // the gradient handed down

    const int nblk = (p.D + CPW - 1) / CPW;
    __shared__ int s_len[32 * WT + 1];
    const int s = seq_by_length(p.off, p.S, p.T, blockIdx.x / nblk, s_len), cb = blockIdx.x % nblk, c0 = cb * CPW;
    const int q = lane % R, grp = lane / R;
    const int chl = grp * CH + q % CH, ch = c0 + chl, n0 = NS * q;
    const int half = (lane >> 4) * 4;   // of its 8 states, the four that a lane holds first: the lower ones in lanes 0 .. 15
    const int tok0 = (q / CH / DUP) * PT;   // of two tokens, the first whose outputs this lane writes (DUP lanes have the same)
    const bool live = ch < p.D, writer = live && (q / CH) % DUP == 0;
    const SeqRange sr = seq_range(p.off, s, p.S, p.T);
    const int g_ = p.G == 1 ? 0 : c0 / (p.D / p.G);

    if (threadIdx.x < 6) {
        const int w = threadIdx.x;
        const void *base = w == 0 ? p.x : w == 1 ? p.dt : w == 2 ? p.z : w == 3 ? q_.dy : w == 4 ? p.b : p.c;
        const long long stride = w == 0 ? p.xs : w == 1 ? p.dts : w == 2 ? p.zs : w == 3 ? q_.dys : w == 4 ? p.bs : p.cs;
        const long long at = (long long)sr.start * stride + (w < 4 ? c0 : g_ * N);
        s_src[w] = base ? make_longlong2((long long)base + at * (long long)sizeof(TI), stride * (long long)sizeof(TI)) : make_longlong2(0, 0);
    }
    auto states_from = [&](const float *from, float2 (&v)[CH][NP]) {   // this lane's states of a [D][N] array
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float4 u = zero4(), w = u;
            if ((ch ^ j) < p.D) {
                const float *o = from + (size_t)(ch ^ j) * N + n0;
                u = *reinterpret_cast<const float4 *>(o + half);
                w = *reinterpret_cast<const float4 *>(o + (half ^ 4));
            }
            v[j][0] = make_float2(u.x, u.y); v[j][1] = make_float2(u.z, u.w);
            v[j][2] = make_float2(w.x, w.y); v[j][3] = make_float2(w.z, w.w);
        }
    };
    auto states_to = [&](float *to, const float2 (&v)[CH][NP]) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if ((ch ^ j) < p.D) {
                float *o = to + (size_t)(ch ^ j) * N + n0;
                *reinterpret_cast<float4 *>(o + half) = make_float4(v[j][0].x, v[j][0].y, v[j][1].x, v[j][1].y);
                *reinterpret_cast<float4 *>(o + (half ^ 4)) = make_float4(v[j][2].x, v[j][2].y, v[j][3].x, v[j][3].y);
            }
        }
    };
    auto put = [&](float4 *to, const float2 (&v)[CH][NP]) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int k = 0; k < NP; k += 2) to[(j * NP / 2 + k / 2) * 32 + lane] = make_float4(v[j][k].x, v[j][k].y, v[j][k + 1].x, v[j][k + 1].y);
    };
    auto take = [&](const float4 *from, float2 (&v)[CH][NP]) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int k = 0; k < NP; k += 2) {
                const float4 u = from[(j * NP / 2 + k / 2) * 32 + lane];
                v[j][k] = make_float2(u.x, u.y);
                v[j][k + 1] = make_float2(u.z, u.w);
            }
    };
    auto clear = [&](float2 (&v)[CH][NP]) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int k = 0; k < NP; ++k) v[j][k] = make_float2(0.f, 0.f);
    };
    float2 a[CH][NP], da[CH][NP];   // decay rates a log2(e); gradient of a
    states_from(p.a, a);
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int k = 0; k < NP; ++k) a[j][k] = make_float2(decay_rate(a[j][k].x), decay_rate(a[j][k].y));
    clear(da);
    DecayShift shift[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) shift[j].set(a[j]);
    const float bias = live && p.bias ? p.bias[ch] : 0.f, skip = live && p.dsk ? p.dsk[ch] : 0.f;
    float sum_skip = 0.f, sum_bias = 0.f, lost_skip = 0.f, lost_bias = 0.f;
    __syncthreads();

    const int ntile = (sr.len + TOK - 1) / TOK;
    const size_t ck0 = (size_t)(sr.start / kCkptTok) + s;
    auto fetch = [&](int tile, TI *to) {   // raw operands of a tile
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            int id = lane + 32 * i;
            if (id < Sh::CHUNKS) {
                TI *at = to + id * E16;
                const bool in_x = id < 4 * TOK * XC;
                const int which = in_x ? id / (TOK * XC) : 4 + (id - 4 * TOK * XC) / (TOK * BC);
                id = in_x ? id % (TOK * XC) : (id - 4 * TOK * XC) % (TOK * BC);
                const int per = in_x ? XC : BC, t = tile * TOK + id / per;
                const longlong2 from = s_src[which];
                const bool ok = from.x && t < sr.len && (!in_x || c0 + (id % per) * E16 < p.D);
                const char *src = reinterpret_cast<const char *>(ok ? from.x + (long long)t * from.y + (id % per) * 16 : (long long)p.x);
                copy16(at, src, ok);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // the tile's checkpoint into the first of the kept states; the forward kernel's order of states in a lane
    auto fetch_state = [&](int tile) {
        const float4 *from = ckpt_at(p.ckpt, ck0 + tile, nblk, cb, CH * NP / 2) + lane;
#pragma unroll
        for (int i = 0; i < CH * NP / 2; ++i) copy16(s_keep + i * 32 + lane, from + (i ^ (half >> 2)) * 32, (ch ^ (i / 2)) < p.D);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int stage = 0;
    if (ntile - 1 - warp >= 0) {
        fetch(ntile - 1 - warp, s_raw2);
        fetch_state(ntile - 1 - warp);
    }
    for (int tile = ntile - 1 - warp; tile >= 0; tile -= WT) {
        const int t0 = tile * TOK;
        const TI *s_raw = s_raw2 + stage * Sh::RAW_E;
        asm volatile("cp.async.wait_group 1;" ::: "memory");   // the operands; the checkpoint may still be under way
        __syncwarp();
#pragma unroll
        for (int i = 0; i < (Sh::BC_F / 4 + 31) / 32; ++i)
            if (lane + 32 * i < Sh::BC_F / 4) reinterpret_cast<float4 *>(s_bc)[lane + 32 * i] = load4(s_raw + 4 * TOK * CPW + 4 * (lane + 32 * i));
        // time step, input and gated gradient of every token and channel
#pragma unroll
        for (int i0 = 0; i0 < TOK / LPC; i0 += 2) {
            float d[2];
            int at[2], tt[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                tt[k] = q / CH + LPC * (i0 + k < TOK / LPC ? i0 + k : i0);
                at[k] = tt[k] * CPW + chl;
                d[k] = load1(s_raw + TOK * CPW + at[k]) + bias;
            }
            if (p.softplus) {
                const float2 v = softplus_acc(make_float2(d[0], d[1]));
                d[0] = v.x;
                d[1] = v.y;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (t0 + tt[k] >= sr.len) d[k] = 0.f;   // past the end: decay 1, no input
                float dg = load1(s_raw + 3 * TOK * CPW + at[k]);
                if (p.z) dg *= gate_f(load1(s_raw + 2 * TOK * CPW + at[k]));
                s_dt[at[k]] = d[k];
                s_dx[at[k]] = d[k] * load1(s_raw + at[k]);
                s_dg[at[k]] = dg;
            }
        }
        __syncwarp();
        auto row_of = [&](const float *m, float2 (&o)[NP]) {
            const float4 u = *reinterpret_cast<const float4 *>(m + half), v = *reinterpret_cast<const float4 *>(m + (half ^ 4));
            o[0] = make_float2(u.x, u.y); o[1] = make_float2(u.z, u.w);
            o[2] = make_float2(v.x, v.y); o[3] = make_float2(v.z, v.w);
        };
        const float *s_b = s_bc + n0, *s_c = s_b + TOK * N;

        asm volatile("cp.async.wait_group 0;" ::: "memory");
        float2 h[CH][NP];
        take(s_keep, h);
        if (tile >= WT) {
            stage ^= 1;
            fetch(tile - WT, s_raw2 + stage * Sh::RAW_E);
            if (lane < CH * NP) asm volatile("prefetch.global.L2 [%0];" ::"l"(ckpt_at(p.ckpt, ck0 + tile - WT, nblk, cb, CH * NP / 2) + lane * 8));
        }
        // forwards: states; what the tile adds to the gradient before it
        float2 add[CH][NP], whole[CH][NP];
        clear(add);
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int k = 0; k < NP; ++k) whole[j][k] = make_float2(1.f, 1.f);
        float time[CH] = {};
        float2 near[CH];
#pragma unroll
        for (int u = 0; u < TOK; u += SUB) {
            if (u) put(s_keep + u / SUB * (Sh::STATE_F / 4), h);
#pragma unroll
            for (int i = 0; i < SUB; ++i) {
                float2 bv[NP], cv[NP];
                row_of(s_b + (u + i) * N, bv);
                row_of(s_c + (u + i) * N, cv);
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    const int at = (u + i) * CPW + (chl ^ j);
                    const float2 d = splat2(s_dt[at]), x = splat2(s_dx[at]), y = splat2(s_dg[at]);
                    if (u == 0 && i == 0) near[j] = shift[j].at(d.x);
                    time[j] += d.x;
#pragma unroll
                    for (int k = 0; k < NP; ++k) {
                        const float2 v = fma2v(a[j][k], d, near[j]), e = make_float2(ex2(v.x), ex2(v.y));
                        h[j][k] = fma2v(e, h[j][k], mul2v(x, bv[k]));
                        whole[j][k] = mul2v(whole[j][k], e);
                        add[j][k] = fma2v(whole[j][k], mul2v(cv[k], y), add[j][k]);
                    }
                }
            }
        }
        // The tile's whole decay, from its time.  As a product it would lose k l 2^-48 at each step from (1 - k 2^-24)(1 - l
        // 2^-24) whenever that is less than half a step, always to the same side: 0.16 steps a token at exponents of 2^-14.
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            near[j] = shift[j].at(time[j]);
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const float2 v = fma2v(a[j][k], splat2(time[j]), near[j]);
                whole[j][k] = make_float2(ex2(v.x), ex2(v.y));
            }
        }
        // the gradient behind the tile comes in, the one before it goes on
        float2 g[CH][NP];
        if (tile < ntile - 1) {
            const int from = (warp + WT - 1) % WT;
            named_sync(1 + from);
            take(reinterpret_cast<const float4 *>(smem + from * Sh::WARP_B + HAND), g);
        } else if (q_.d_state_out) {
            states_from(q_.d_state_out + (size_t)s * p.D * N, g);
        } else {
            clear(g);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int k = 0; k < NP; ++k) add[j][k] = fma2v(whole[j][k], g[j][k], add[j][k]);
        if (tile > 0) {
            put(s_down, add);
            named_arrive(1 + warp);
        } else if (q_.d_state_in) {
            states_to(q_.d_state_in + (size_t)s * p.D * N, add);
        }

        // backwards, two tokens at a time
        float tile_skip = 0.f, tile_bias = 0.f;
        float *part = q_.part_bc + ((size_t)cb * p.T + sr.start + t0) * (2 * N);   // [token][dB N | dC N]
#pragma unroll 1
        for (int u = TOK - SUB; u >= 0; u -= SUB) {
            take(s_keep + u / SUB * (Sh::STATE_F / 4), h);
            auto fold_channels = [&](const float2 (&w)[NP], float *to) {
                // this lane's 8 states summed over the 32 / R lanes of other channels; 8 values halve three times at most.
                // Lanes 16 .. 31 hold the upper four first, so the first halving sends the last four everywhere.
                float v[4];
                v[0] = w[0].x + __shfl_xor_sync(0xffffffffu, w[2].x, 16);
                v[1] = w[0].y + __shfl_xor_sync(0xffffffffu, w[2].y, 16);
                v[2] = w[1].x + __shfl_xor_sync(0xffffffffu, w[3].x, 16);
                v[3] = w[1].y + __shfl_xor_sync(0xffffffffu, w[3].y, 16);
                int first = 0, n = 4;
#pragma unroll
                for (int o = 8; o >= R; o >>= 1) {
                    if (n > 1) {
                        n >>= 1;
                        const bool up = lane & o;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            if (k < n) {
                                const float send = up ? v[k] : v[k + n], keep = up ? v[k + n] : v[k];
                                v[k] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                            }
                        }
                        if (up) first += n;
                    } else {
                        v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
                    }
                }
                constexpr int GR = 32 / R, KEEP = GR >= 8 ? 1 : 8 / GR;
                if (to && (GR <= 8 || grp % (GR > 8 ? GR / 8 : 1) == 0)) {
#pragma unroll
                    for (int k = 0; k < KEEP; ++k) to[n0 + half + first + k] = v[k];
                }
            };
            float2 e[SUB][CH][NP], h0[CH][NP];   // decays; the state behind the first token
            float dts[SUB][CH], dxs[SUB][CH], dgs[SUB][CH];
            float yh[SUB], gb[SUB], ga[SUB];     // of this lane's channel: sum_n c h, g b, e h_prev a
            {
                float2 hh[CH][NP];
#pragma unroll
                for (int i = 0; i < SUB; ++i) {
                    float2 bv[NP], cv[NP];
                    row_of(s_b + (u + i) * N, bv);
                    row_of(s_c + (u + i) * N, cv);
                    float own[CH];
                    float2 v[NP];
#pragma unroll
                    for (int j = 0; j < CH; ++j) {
                        const int at = (u + i) * CPW + (chl ^ j);
                        dts[i][j] = s_dt[at];
                        dxs[i][j] = s_dx[at];
                        dgs[i][j] = s_dg[at];
                        float2 sum = make_float2(0.f, 0.f);
                        if (i == 0) near[j] = shift[j].at(dts[i][j]);
#pragma unroll
                        for (int k = 0; k < NP; ++k) {
                            const float2 w = fma2v(a[j][k], splat2(dts[i][j]), near[j]);
                            e[i][j][k] = make_float2(ex2(w.x), ex2(w.y));
                            hh[j][k] = fma2v(e[i][j][k], i ? h0[j][k] : h[j][k], mul2v(splat2(dxs[i][j]), bv[k]));
                            if (i == 0) h0[j][k] = hh[j][k];
                            sum = k ? fma2v(cv[k], hh[j][k], sum) : mul2v(cv[k], hh[j][k]);
                            v[k] = j ? fma2v(splat2(dgs[i][j]), hh[j][k], v[k]) : mul2v(splat2(dgs[i][j]), hh[j][k]);
                        }
                        own[j] = sum.x + sum.y;
                    }
                    yh[i] = CH == 1 ? own[0] : own[0] + __shfl_xor_sync(0xffffffffu, own[CH - 1], 1);
                    fold_channels(v, t0 + u + i < sr.len ? part + (size_t)(u + i) * 2 * N + N : nullptr);
                }
            }
#pragma unroll
            for (int i = SUB - 1; i >= 0; --i) {
                float2 bv[NP], cv[NP];
                row_of(s_b + (u + i) * N, bv);
                row_of(s_c + (u + i) * N, cv);
                float ogb[CH], oga[CH];
                float2 v[NP];
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    float2 ub = make_float2(0.f, 0.f), ua = ub;
#pragma unroll
                    for (int k = 0; k < NP; ++k) {
                        g[j][k] = fma2v(cv[k], splat2(dgs[i][j]), g[j][k]);
                        ub = k ? fma2v(g[j][k], bv[k], ub) : mul2v(g[j][k], bv[k]);
                        v[k] = j ? fma2v(splat2(dxs[i][j]), g[j][k], v[k]) : mul2v(splat2(dxs[i][j]), g[j][k]);
                        g[j][k] = mul2v(g[j][k], e[i][j][k]);   // e_t
                        const float2 through = mul2v(g[j][k], i ? h0[j][k] : h[j][k]);
                        ua = k ? fma2v(through, a[j][k], ua) : mul2v(through, a[j][k]);
                        da[j][k] = fma2v(through, splat2(dts[i][j]), da[j][k]);
                    }
                    ogb[j] = ub.x + ub.y;
                    oga[j] = ua.x + ua.y;
                }
                gb[i] = CH == 1 ? ogb[0] : ogb[0] + __shfl_xor_sync(0xffffffffu, ogb[CH - 1], 1);
                ga[i] = CH == 1 ? oga[0] : oga[0] + __shfl_xor_sync(0xffffffffu, oga[CH - 1], 1);
                fold_channels(v, t0 + u + i < sr.len ? part + (size_t)(u + i) * 2 * N : nullptr);
            }
            // the other lanes of a channel hold other states: halve the tokens at the first exchange, then add
            if (R > CH) {
                int n = SUB;
#pragma unroll
                for (int o = R / 2; o >= CH; o >>= 1) {
                    const bool up = lane & o;
                    if (n > 1) {
                        n >>= 1;
                        auto turn = [&](float (&w)[SUB]) {
                            const float send = up ? w[0] : w[1], mine = up ? w[1] : w[0];
                            w[0] = mine + __shfl_xor_sync(0xffffffffu, send, o);
                        };
                        turn(yh);
                        turn(gb);
                        turn(ga);
                    } else {
                        yh[0] += __shfl_xor_sync(0xffffffffu, yh[0], o);
                        gb[0] += __shfl_xor_sync(0xffffffffu, gb[0], o);
                        ga[0] += __shfl_xor_sync(0xffffffffu, ga[0], o);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                const int t = u + tok0 + i, at = t * CPW + chl;
                if (writer && t0 + t < sr.len) {
                    const float x = load1(s_raw + at), dy = load1(s_raw + 3 * TOK * CPW + at), dg = s_dg[at];
                    const size_t o = (size_t)(sr.start + t0 + t) * p.D + ch;
                    if (p.z) {
                        const float z = load1(s_raw + 2 * TOK * CPW + at), sg = sigmoid_acc(z);
                        store1(static_cast<TG *>(q_.d_z) + o, dy * fmaf(skip, x, yh[i]) * (sg * fmaf(z, 1.f - sg, 1.f)));
                    }
                    store1(static_cast<TG *>(q_.d_x) + o, fmaf(s_dt[at], gb[i], skip * dg));
                    float ddt = fmaf(x, gb[i], 0.6931471805599453f * ga[i]);   // the rates are a log2(e)
                    if (p.softplus) ddt *= sigmoid_acc(load1(s_raw + TOK * CPW + at) + bias);
                    store1(static_cast<TG *>(q_.d_dt) + o, ddt);
                    tile_skip = fmaf(dg, x, tile_skip);
                    tile_bias += ddt;
                }
            }
        }
        compensated(sum_skip, lost_skip, tile_skip);
        compensated(sum_bias, lost_bias, tile_bias);
        __syncwarp();   // done with the tile's shared memory
        if (tile >= WT) fetch_state(tile - WT);
    }
    if (ntile == 0 && q_.d_state_in && warp == 0) {
        float2 g[CH][NP];
        clear(g);
        if (q_.d_state_out) states_from(q_.d_state_out + (size_t)s * p.D * N, g);
        states_to(q_.d_state_in + (size_t)s * p.D * N, g);
    }
    // this sequence's share of the parameters' gradients: over the warps, then over a channel's lanes
    __syncthreads();
    put(s_keep, da);
    float *s_sum = reinterpret_cast<float *>(s_down);
    s_sum[lane] = sum_skip;
    s_sum[32 + lane] = sum_bias;
    __syncthreads();
    if (warp == 0) {
#pragma unroll 1
        for (int w = 1; w < WT; ++w) {
            const unsigned char *other = smem + w * Sh::WARP_B;
            float2 v[CH][NP];
            take(reinterpret_cast<const float4 *>(other + Sh::RAW_B + (Sh::PREP_F + Sh::BC_F) * 4), v);
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int k = 0; k < NP; ++k) da[j][k] = add2v(da[j][k], v[j][k]);
            const float *o = reinterpret_cast<const float *>(other + HAND);
            sum_skip += o[lane];
            sum_bias += o[32 + lane];
        }
        states_to(q_.part_a + (size_t)s * p.D * N, da);
#pragma unroll
        for (int o = CH; o < R; o <<= 1) {
            sum_skip += __shfl_xor_sync(0xffffffffu, sum_skip, o);
            sum_bias += __shfl_xor_sync(0xffffffffu, sum_bias, o);
        }
        if (live && q < CH) {
            q_.part_d[((size_t)s * 2) * p.D + ch] = sum_skip;
            q_.part_d[((size_t)s * 2 + 1) * p.D + ch] = sum_bias;
        }
    }
}

// Zeros in the rows of [T, D] tensors (the last two nullable) that belong to no sequence
template <typename T_>
__device__ __forceinline__ void zero_rest(void *a, void *b, void *c, const int *off, int S, int T, int D)
{
    const size_t first = (size_t)seq_start(off, S, S, T) * D;
    for (size_t i = first + 4 * (blockIdx.x * (size_t)blockDim.x + threadIdx.x); i < (size_t)T * D; i += 4 * (size_t)gridDim.x * blockDim.x) {
        store4(static_cast<T_ *>(a) + i, zero4());
        if (b) store4(static_cast<T_ *>(b) + i, zero4());
        if (c) store4(static_cast<T_ *>(c) + i, zero4());
    }
}
template <typename TO>
__global__ void __launch_bounds__(256) selscan_rest_kernel(void *y, const int *off, int S, int T, int D)
{
    zero_rest<TO>(y, nullptr, nullptr, off, S, T, D);
}

// dB, dC: sum of the channel blocks' partial sums, rounded once; zeros where there is no sequence, in the other gradients too
template <typename TG, int N>
__global__ void __launch_bounds__(256) selscan_bc_kernel(const ScanBwdParams q, void *d_b, void *d_c, int blocks_per_group)
{
    const float *part = q.part_bc;
    const int *off = q.f.off, S = q.f.S, T = q.f.T, G = q.f.G;
    const size_t per_tok = (size_t)G * (2 * N / 4);
    const size_t end = seq_start(off, S, S, T);
    for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < (size_t)T * per_tok; i += (size_t)gridDim.x * blockDim.x) {
        const size_t t = i / per_tok;
        const int rest = (int)(i % per_tok), g = rest / (2 * N / 4), v = rest % (2 * N / 4);
        float4 o = zero4();
        for (int k = 0; k < (t < end ? blocks_per_group : 0); ++k) {
            const float4 u = *reinterpret_cast<const float4 *>(part + ((size_t)(g * blocks_per_group + k) * T + t) * (2 * N) + 4 * v);
            o.x += u.x; o.y += u.y; o.z += u.z; o.w += u.w;
        }
        const bool is_c = v >= N / 4;
        store4(static_cast<TG *>(is_c ? d_c : d_b) + (t * G + g) * N + 4 * (v - (is_c ? N / 4 : 0)), o);
    }
    if (off) zero_rest<TG>(q.d_x, q.d_dt, q.d_z, off, S, T, q.f.D);
}

// The parameters' gradients: sums over the sequences of part_a and part_d, the former's elements first
__global__ void __launch_bounds__(256) selscan_sum_kernel(const float *part_a, const float *part_d, float *d_a, float *d_skip, float *d_bias, int S,
                                                          int D, int N)
{
    const size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x, na = (size_t)D * N;
    if (i >= na + 2 * (size_t)D) return;
    const bool in_a = i < na;
    const size_t k = in_a ? i : i - na;   // for the rest [skip | bias][D]
    float *out = in_a ? d_a + k : (k < (size_t)D ? (d_skip ? d_skip + k : nullptr) : (d_bias ? d_bias + (k - D) : nullptr));
    if (!out) return;
    const float *part = in_a ? part_a : part_d;
    const size_t stride = in_a ? na : 2 * (size_t)D;
    float o = 0.f;
    for (int s = 0; s < S; ++s) o += part[(size_t)s * stride + k];
    *out = o;
}

// ------------------------------------------------------------------------------------------------ launches

// Tokens of a segment, 0 = whole sequences.  A split costs a second pass over x, dt, b (their decays evaluated twice, 1.9
// times the exponentials), so for sequences of equal length it pays only where the chains leave more than half of the SMs
// without work.  The host does not know the lengths and takes the mean: one long sequence among many short ones is not split
// (30000 tokens among 39 of 51, 512 channels: 1700 us).
int fwd_segment(int T, int S, int D, int N)
{
    const int cpw = chain_channels(N);
    const long long cols = (D + cpw - 1) / cpw, chains = cols * S;
    if (chains * 2 > 148 || T / S < 512) return 0;
    // k segments a sequence of average length: as many rounds of two CTAs an SM as it takes, each as long as a segment and
    // what it costs to begin one (about 100 tokens).  A segment too many is a round more: one sequence of 32768 x 512
    // takes 255 us in 18 segments, 390 in 22, 262 in 37.
    const long long len = T / S;
    long long best = 0, best_seg = 0;
    for (long long k = 1; k <= 1024 && (k == 1 || len / k >= 256); ++k) {
        const long long seg = ((len + k - 1) / k + 31) / 32 * 32, rounds = (k * chains + 2 * 148 - 1) / (2 * 148), cost = rounds * (seg + 100);
        if (k == 1 || cost < best) {
            best = cost;
            best_seg = seg;
        }
    }
    return (int)best_seg;
}

template <typename TI, typename TO, int N, int CH, int TOK, int WT, int OCC>
chela_status_t fwd_launch(ScanParams p, cudaStream_t stream)
{
    using Sh = FwdShape<TI, N, CH, TOK>;
    constexpr size_t smem = (size_t)WT * Sh::WARP_B;
    const auto kern = selscan_fwd_kernel<TI, TO, N, CH, TOK, WT, OCC>;
    if (smem > 40 * 1024) {   // with the static part, past the 48 KB that need no asking
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return cuda_status(e);
    }
    const long long chains = p.seg ? (long long)packed_blocks(p.T, p.S, p.seg) : p.S;
    const long long blocks = chains * ((p.D + Sh::CPW - 1) / Sh::CPW);
    if (blocks > 0x7fffffffLL) return CHELA_ERR_UNSUPPORTED;
    if (p.seg) {
        ScanParams q = p;
        q.y = nullptr;
        q.c = q.z = nullptr;
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

// Half as many channels a chain and twice the tokens a slice (one channel a lane): twice the chains, half the steps of each.
// Every b and c is then read for one channel instead of two, so it pays while the SM with the most chains has fewer half
// ones than whole ones' halves: up to one and a half chains of the full width per SM (4 x 4096 x 1024, 128 chains: 152 us
// against 226; 8 x 8192 x 1024, 256 chains: 581 against 553).
bool fwd_narrow(const ScanParams &p, int N) { return !p.seg && (long long)p.S * ((p.D + chain_channels(N) - 1) / chain_channels(N)) <= 222; }

template <typename TI, typename TO>
chela_status_t fwd_n(const ScanParams &p, int N, cudaStream_t stream)
{
    switch (N) {
    case 8: return fwd_launch<TI, TO, 8, 1, 8, 8, 2>(p, stream);
    case 16: return fwd_narrow(p, N) ? fwd_launch<TI, TO, 16, 1, 8, 8, 2>(p, stream) : fwd_launch<TI, TO, 16, 2, 4, 8, 2>(p, stream);
    case 32: return fwd_narrow(p, N) ? fwd_launch<TI, TO, 32, 1, 8, 8, 2>(p, stream) : fwd_launch<TI, TO, 32, 2, 4, 8, 2>(p, stream);
    default: return fwd_launch<TI, TO, 64, 2, 4, 8, 2>(p, stream);
    }
}

template <typename TI, typename TO>
chela_status_t step_n(const ScanParams &p, int N, cudaStream_t stream)
{
    const size_t threads = (size_t)p.S * p.D * (N / 8);
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

template <typename TI, typename TG, int N>
chela_status_t bwd_launch(const ScanBwdParams &q, void *d_b, void *d_c, float *d_a, float *d_skip, float *d_bias, cudaStream_t stream)
{
    const ScanParams &p = q.f;
    using Sh = BwdShape<TI, N, chain_ch(N)>;
    constexpr int DC = Sh::CPW;
    constexpr size_t smem = Sh::SMEM;
    const auto kern = selscan_bwd_kernel<TI, TG, N, chain_ch(N)>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return cuda_status(e);
    const int nblk = (p.D + DC - 1) / DC;
    const long long blocks = (long long)p.S * nblk;
    if (blocks > 0x7fffffffLL) return CHELA_ERR_UNSUPPORTED;
    kern<<<(unsigned)blocks, 32 * Sh::WT, smem, stream>>>(q);
    chela_status_t st = last_launch_status();
    if (st != CHELA_OK) return st;
    const size_t items = (size_t)p.T * p.G * (2 * N / 4);
    const size_t grid = (items + 255) / 256;
    selscan_bc_kernel<TG, N><<<(unsigned)(grid < 148 * 32 ? grid : 148 * 32), 256, 0, stream>>>(q, d_b, d_c, nblk / p.G);
    st = last_launch_status();
    if (st == CHELA_OK) {
        selscan_sum_kernel<<<(unsigned)(((size_t)p.D * (N + 2) + 255) / 256), 256, 0, stream>>>(q.part_a, q.part_d, d_a, d_skip, d_bias, p.S, p.D, N);
        st = last_launch_status();
    }
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
    p.S = a.S; p.T = a.T; p.D = a.D; p.G = a.G; p.softplus = a.softplus & 1;
    return p;
}

struct ScanBwdPlan {
    size_t off_ckpt, off_fwd, off_bc, off_a, off_d, total;
};
ScanBwdPlan bwd_plan(int T, int S, int D, int N, bool have_ckpt)
{
    ScanBwdPlan p;
    const int dc = chain_channels(N);
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
    const int cpw = chain_channels(N);
    return packed_blocks(T, S, kCkptTok) * ((D + cpw - 1) / cpw) * cpw * N * sizeof(float);
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
    if (y && a.seq_offsets && (a.softplus & CHELA_ZERO_REST)) {   // mostly no rows or few: one CTA an SM
        const auto rest = out_dtype == CHELA_F32 ? selscan_rest_kernel<float> : selscan_rest_kernel<__nv_bfloat16>;
        rest<<<148, 256, 0, stream>>>(y, a.seq_offsets, a.S, a.T, a.D);
        const chela_status_t st = last_launch_status();
        if (st != CHELA_OK) return st;
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
