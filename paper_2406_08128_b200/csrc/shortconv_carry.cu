// Short depthwise causal convolution over packed sequences with the last width - 1 inputs carried between calls, its
// single-token form and its backward pass.  u_t = bias + sum_j w_j x_{t-j}, y = act(u).
//
// Bound by HBM: 2 bytes in and 2 out per bf16 element for 2 width flops.  A thread owns 4 channels (one 8-byte access
// for bf16, a warp reads 256 contiguous bytes of a token) and kTok consecutive tokens of one sequence with the taps and the
// previous inputs in registers, so every input is read once plus a halo of width - 1 rows per kTok.
#include <type_traits>

#include "packed.cuh"

namespace chela {
namespace {

constexpr int kTok = 32;      // tokens of one forward work item
constexpr int kBwdTok = 64;   // tokens of one backward work item

struct ConvParams {
    const void *x;
    long long xs;
    const float *w, *bias;
    void *y;
    const void *state_in;
    void *state_out;
    const int *off;
    int S, T, D, width, act;
    int rest;   // 1: the rows of tokens of no sequence become zeros
};

__device__ __forceinline__ float4 fma4(float4 a, float4 b, float4 c)
{
    return make_float4(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y), fmaf(a.z, b.z, c.z), fmaf(a.w, b.w, c.w));
}
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 zero4() { return make_float4(0.f, 0.f, 0.f, 0.f); }
__device__ __forceinline__ float silu_acc(float u) { return u * sigmoid_acc(u); }
__device__ __forceinline__ float d_silu(float u)
{
    const float s = sigmoid_acc(u);
    return s * fmaf(u, 1.f - s, 1.f);
}

// Input row at position t of a sequence that starts at row `start`: carried rows stand before position 0.
template <typename T>
__device__ __forceinline__ float4 row_at(const ConvParams &p, int s, int start, int len, int t, int c)
{
    if (t >= 0) return t < len ? load4(static_cast<const T *>(p.x) + (size_t)(start + t) * p.xs + c) : zero4();
    const int r = p.width - 1 + t;
    if (!p.state_in || r < 0) return zero4();
    return load4(static_cast<const T *>(p.state_in) + ((size_t)s * (p.width - 1) + r) * p.D + c);
}

// The last width - 1 inputs of (carried rows | sequence).  Called by the one thread that owns these channels of the
// sequence's first work item, after all its own reads of state_in, so both states may be the same buffer: state_out row r
// comes from a row of state_in with an index >= r, so going upwards no row is written before it is read.
template <typename T>
__device__ __forceinline__ void store_state(const ConvParams &p, int s, const SeqRange &sr, int c)
{
    const int n = p.width - 1;
    for (int r = 0; r < n; ++r) {
        const float4 v = row_at<T>(p, s, sr.start, sr.len, sr.len - n + r, c);
        store4(static_cast<T *>(p.state_out) + ((size_t)s * n + r) * p.D + c, v);
    }
}

// Zeros in four channels of the rows of a block of K tokens behind the last sequence
template <typename T>
__device__ __forceinline__ void zero_rest(const ConvParams &p, void *rows, long long blk, int K, int c)
{
    const int end = seq_start(p.off, p.S, p.S, p.T);
    const long long first = end + (blk - (end / K + p.S)) * K, last = first + K < p.T ? first + K : p.T;
#pragma unroll 1
    for (long long t = first; t < last; ++t) store4(static_cast<T *>(rows) + (size_t)t * p.D + c, zero4());
}

// taps[j] = (w[c][j], w[c+1][j], w[c+2][j], w[c+3][j]).  Four channels' taps are 4 width contiguous floats from a multiple
// of 16 bytes on, read as vectors where the width is a template argument.
template <int W>
__device__ __forceinline__ void load_taps(const float *w, int width, int c, float4 (&taps)[W])
{
    if (width == W) {
        float f[4 * W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const float4 v = reinterpret_cast<const float4 *>(w + (size_t)c * W)[j];
            f[4 * j] = v.x; f[4 * j + 1] = v.y; f[4 * j + 2] = v.z; f[4 * j + 3] = v.w;
        }
#pragma unroll
        for (int j = 0; j < W; ++j) taps[j] = make_float4(f[j], f[W + j], f[2 * W + j], f[3 * W + j]);
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            taps[j] = j < width ? make_float4(w[(size_t)c * width + j], w[(size_t)(c + 1) * width + j], w[(size_t)(c + 2) * width + j],
                                              w[(size_t)(c + 3) * width + j])
                                : zero4();
    }
}

// (item / nvec, item % nvec) without a 64-bit division where 32 bits do
__device__ __forceinline__ void split_item(long long item, long long items, int nvec, long long &blk, int &cv)
{
    if (items <= 0x7fffffffLL) {
        blk = (unsigned)item / (unsigned)nvec;
        cv = (int)((unsigned)item % (unsigned)nvec);
    } else {
        blk = item / nvec;
        cv = (int)(item % nvec);
    }
}

// W: taps held in registers (the width itself up to 4; 8 and 16 for the widths up to those, whose extra taps are skipped:
// zero times an infinity that lies further back than the width would be NaN).
// The tokens of a work item are copied to shared memory in groups of SUB, two groups ahead of the arithmetic, every thread
// the 8 or 16 bytes that it will use itself: nothing but its own copies has to be waited for, and the loads in flight
// cost no registers.  (65536 x 1024, bf16: four loads a thread in registers 140 us, eight 68 us, this way 58 us; groups of
// eight or two CTAs an SM 64 and 68 us.)
template <typename T, int W>
__global__ void __launch_bounds__(256, W <= 4 ? 3 : 1) conv_carry_kernel(const ConvParams p, long long items)
{
    constexpr int SUB = 4;
    extern __shared__ __align__(16) unsigned char smem[];
    Raw4<T> *ring = reinterpret_cast<Raw4<T> *>(smem) + threadIdx.x;   // [2][SUB][256]
    const int nvec = p.D / 4;
    for (long long idx = blockIdx.x * (long long)blockDim.x + threadIdx.x; idx < items; idx += (long long)gridDim.x * blockDim.x) {
        long long blk;
        int cv;
        split_item(idx, items, nvec, blk, cv);
        const int c = 4 * cv;
        const int s = packed_block_seq(p.off, p.S + p.rest, p.T, kTok, blk);
        if (s == p.S) {
            zero_rest<T>(p, p.y, blk, kTok, c);
            continue;
        }
        const SeqRange sr = seq_range(p.off, s, p.S, p.T);
        const int b = (int)(blk - (sr.start / kTok + s));
        if (b < 0 || b > sr.len / kTok) continue;
        const int t0 = b * kTok;
        if (t0 < sr.len) {
            const int end = min(t0 + kTok, sr.len);
            const T *px = static_cast<const T *>(p.x) + (size_t)(sr.start + t0) * p.xs + c;
            T *py = static_cast<T *>(p.y) + (size_t)(sr.start + t0) * p.D + c;
            auto fetch = [&](int t, int half) {
#pragma unroll
                for (int i = 0; i < SUB; ++i) copy_raw4(ring + (half * SUB + i) * 256, t + i < end ? px + (size_t)i * p.xs : px, t + i < end);
                px += t + SUB < end ? (size_t)SUB * p.xs : 0;
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            fetch(t0, 0);
            fetch(t0 + SUB, 1);
            float4 taps[W], in[W];   // in[j] = x_{t-j}
            load_taps<W>(p.w, p.width, c, taps);
            const float4 bias = p.bias ? load4(p.bias + c) : zero4();
#pragma unroll
            for (int j = 1; j < W; ++j) in[j - 1] = row_at<T>(p, s, sr.start, sr.len, t0 - j, c);
            int half = 0;
#pragma unroll 1
            for (int t = t0; t < end; t += SUB) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
                for (int i = 0; i < SUB; ++i) {
#pragma unroll
                    for (int j = W - 1; j > 0; --j) in[j] = in[j - 1];
                    in[0] = ring[(half * SUB + i) * 256].get();
                    float4 u = bias;
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        if (W <= 4 || j < p.width) u = fma4(taps[j], in[j], u);
                    if (p.act) u = make_float4(silu_acc(u.x), silu_acc(u.y), silu_acc(u.z), silu_acc(u.w));
                    if (t + i < end) store4(py + (size_t)i * p.D, u);
                }
                py += (size_t)SUB * p.D;
                fetch(t + 2 * SUB, half);
                half ^= 1;
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        if (b == 0 && p.state_out) store_state<T>(p, s, sr, c);
    }
}

// One token per sequence: a thread reads its channels' carried rows and the new one, writes the output and the rows moved on.
template <typename T, int W>
__global__ void __launch_bounds__(128) conv_step_kernel(const ConvParams p)
{
    const int nvec = p.D / 4;
    const long long idx = blockIdx.x * (long long)blockDim.x + threadIdx.x;
    if (idx >= (long long)p.S * nvec) return;
    long long row;
    int cv;
    split_item(idx, (long long)p.S * nvec, nvec, row, cv);
    const int c = 4 * cv, s = (int)row, n = p.width - 1;
    float4 in[W], taps[W];
    in[0] = load4(static_cast<const T *>(p.x) + (size_t)s * p.xs + c);
    const T *held = static_cast<const T *>(p.state_in) + ((size_t)s * n) * p.D + c;
#pragma unroll
    for (int j = 1; j < W; ++j) in[j] = j <= n ? load4(held + (size_t)(n - j) * p.D) : zero4();
    load_taps<W>(p.w, p.width, c, taps);
    float4 u = p.bias ? load4(p.bias + c) : zero4();
#pragma unroll
    for (int j = 0; j < W; ++j) u = fma4(taps[j], in[j], u);
    if (p.act) u = make_float4(silu_acc(u.x), silu_acc(u.y), silu_acc(u.z), silu_acc(u.w));
    store4(static_cast<T *>(p.y) + (size_t)s * p.D + c, u);
    T *keep = static_cast<T *>(p.state_out) + ((size_t)s * n) * p.D + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
        if (j < n) store4(keep + (size_t)(n - 1 - j) * p.D, in[j]);
}

// ------------------------------------------------------------------------------------------------ backward

struct ConvBwdParams {
    ConvParams f;
    const void *dy;
    long long dys;
    const void *d_state_out;
    void *d_x, *d_state_in;
    float *part;   // [gridDim.y][width + 1][D]: taps, bias
};

// A CTA: 32 lanes x 4 channels, 8 warps that walk work items of kBwdTok tokens; the taps' gradients stay in registers until
// the end, are added over the warps in shared memory and leave as one partial sum per CTA row (a fixed order, no atomics).
// d_x_t = sum_j w_j d_u_{t+j}: a thread evaluates the d_u of its tokens and of the W - 1 behind them.  x and d_y are
// copied to shared memory two groups of SUB tokens ahead, as in the forward kernel.
template <typename T, typename TG, int W>
__global__ void __launch_bounds__(256, W <= 4 ? 2 : 1) conv_bwd_kernel(const ConvBwdParams q, long long nblocks)
{
    constexpr int SUB = 4;
    const ConvParams &p = q.f;
    extern __shared__ __align__(16) unsigned char smem[];
    Raw4<T> *ring = reinterpret_cast<Raw4<T> *>(smem) + threadIdx.x;   // [2][SUB][x, d_y][256]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = (blockIdx.x * 32 + lane) * 4;
    const bool live = c < p.D;
    float4 taps[W], dw[W], db = zero4(), bias = zero4();
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j] = zero4();
    if (live) {
        load_taps<W>(p.w, p.width, c, taps);
        if (p.bias) bias = load4(p.bias + c);
        for (long long blk = (long long)blockIdx.y * 8 + warp; blk < nblocks; blk += (long long)gridDim.y * 8) {
            const int s = packed_block_seq(p.off, p.S + p.rest, p.T, kBwdTok, blk);
            if (s == p.S) {
                zero_rest<TG>(p, q.d_x, blk, kBwdTok, c);
                continue;
            }
            const SeqRange sr = seq_range(p.off, s, p.S, p.T);
            const int b = (int)(blk - (sr.start / kBwdTok + s));
            if (b < 0 || sr.len == 0 || b > (sr.len - 1) / kBwdTok) continue;
            const int t0 = b * kBwdTok;
            const int end = min(t0 + kBwdTok, sr.len), stop = end + W - 1;
            const T *px = static_cast<const T *>(p.x) + (size_t)(sr.start + t0) * p.xs + c;
            const T *pd = static_cast<const T *>(q.dy) + (size_t)(sr.start + t0) * q.dys + c;
            const int last = min(sr.len, stop);   // d_u is zero behind the sequence
            auto fetch = [&](int t, int half) {
#pragma unroll
                for (int i = 0; i < SUB; ++i) {
                    const bool ok = t + i < last;
                    Raw4<T> *to = ring + (half * SUB + i) * 512;
                    copy_raw4(to, ok ? px + (size_t)i * p.xs : px, ok);
                    copy_raw4(to + 256, ok ? pd + (size_t)i * q.dys : pd, ok);
                }
                px += t + SUB < last ? (size_t)SUB * p.xs : 0;
                pd += t + SUB < last ? (size_t)SUB * q.dys : 0;
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            fetch(t0, 0);
            fetch(t0 + SUB, 1);
            int half = 0;
            float4 in[W], du[W];   // in[j] = x_{t-j}; du[j] = d_u_{t-j}
#pragma unroll
            for (int j = 0; j < W; ++j) du[j] = zero4();
#pragma unroll
            for (int j = 1; j < W; ++j) in[j - 1] = row_at<T>(p, s, sr.start, sr.len, t0 - j, c);
            TG *pdx = static_cast<TG *>(q.d_x) + (size_t)(sr.start + t0) * p.D + c;   // of position tg
            // kEdge: some of the group's tokens, or of the positions whose d_x they complete, lie outside the work item or
            // pass a gradient on from state_out
            auto group = [&](auto edge, int tg) {
                constexpr bool kEdge = decltype(edge)::value;
#pragma unroll
                for (int i = 0; i < SUB; ++i) {
                    const int t = tg + i;
#pragma unroll
                    for (int j = W - 1; j > 0; --j) {
                        in[j] = in[j - 1];
                        du[j] = du[j - 1];
                    }
                    in[0] = ring[(half * SUB + i) * 512].get();
                    float4 d = ring[(half * SUB + i) * 512 + 256].get();
                    if (p.act) {
                        float4 u = bias;
#pragma unroll
                        for (int j = 0; j < W; ++j)
                            if (W <= 4 || j < p.width) u = fma4(taps[j], in[j], u);
                        d = make_float4(d.x * d_silu(u.x), d.y * d_silu(u.y), d.z * d_silu(u.z), d.w * d_silu(u.w));
                    }
                    du[0] = !kEdge || t < sr.len ? d : zero4();
                    if (!kEdge || t < end) {
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[j] = fma4(du[0], in[j], dw[j]);
                        db = add4(db, du[0]);
                    }
                    const int tx = t - (W - 1);   // all terms of d_x at this position are there now
                    if (!kEdge || (tx >= t0 && tx < end)) {
                        float4 dx = zero4();
#pragma unroll
                        for (int j = 0; j < W; ++j)
                            if (W <= 4 || j < p.width) dx = fma4(taps[j], du[W - 1 - j], dx);
                        if (kEdge) {
                            const int r = tx - (sr.len - (p.width - 1));
                            if (q.d_state_out && r >= 0)
                                dx = add4(dx, load4(static_cast<const T *>(q.d_state_out) + ((size_t)s * (p.width - 1) + r) * p.D + c));
                        }
                        store4(pdx + (long long)(i - (W - 1)) * p.D, dx);
                    }
                }
            };
#pragma unroll 1
            for (int tg = t0; tg < stop; tg += SUB) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                if (tg >= t0 + W - 1 && tg + SUB <= end && (!q.d_state_out || tg + SUB <= sr.len - p.width))
                    group(std::false_type(), tg);
                else
                    group(std::true_type(), tg);
                pdx += (size_t)SUB * p.D;
                fetch(tg + 2 * SUB, half);
                half ^= 1;
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
    }
    if (!q.part) return;
    __shared__ float4 red[8][32];
#pragma unroll 1
    for (int j = 0; j <= p.width; ++j) {
        float4 v = db;
#pragma unroll
        for (int k = 0; k < W; ++k)
            if (k == j && j < p.width) v = dw[k];
        __syncthreads();
        red[warp][lane] = v;
        __syncthreads();
        if (warp == 0 && live) {
            float4 o = zero4();
#pragma unroll
            for (int k = 0; k < 8; ++k) o = add4(o, red[k][lane]);
            *reinterpret_cast<float4 *>(q.part + ((size_t)blockIdx.y * (p.width + 1) + j) * p.D + c) = o;
        }
    }
}

// d_state_in row r is position r - (width - 1): sum_j w_j d_u of the tokens it reached, plus what passes straight through
// to state_out where the sequence is shorter than the state.
template <typename T, typename TG>
__global__ void __launch_bounds__(128) conv_bwd_state_kernel(const ConvBwdParams q)
{
    const ConvParams &p = q.f;
    const int n = p.width - 1, nvec = p.D / 4;
    const long long idx = blockIdx.x * (long long)blockDim.x + threadIdx.x;
    if (idx >= (long long)p.S * n * nvec) return;
    const int c = 4 * (int)(idx % nvec), r = (int)(idx / nvec % n), s = (int)(idx / nvec / n);
    const SeqRange sr = seq_range(p.off, s, p.S, p.T);
    const int pos = r - n;
    float4 acc = zero4();
    const float4 bias = p.bias ? load4(p.bias + c) : zero4();
    auto tap = [&](int j) {
        return make_float4(p.w[(size_t)c * p.width + j], p.w[(size_t)(c + 1) * p.width + j], p.w[(size_t)(c + 2) * p.width + j],
                           p.w[(size_t)(c + 3) * p.width + j]);
    };
    for (int t = 0; t <= pos + n && t < sr.len; ++t) {
        float4 d = load4(static_cast<const T *>(q.dy) + (size_t)(sr.start + t) * q.dys + c);
        if (p.act) {
            float4 u = bias;
            for (int j = 0; j < p.width; ++j) u = fma4(tap(j), row_at<T>(p, s, sr.start, sr.len, t - j, c), u);
            d = make_float4(d.x * d_silu(u.x), d.y * d_silu(u.y), d.z * d_silu(u.z), d.w * d_silu(u.w));
        }
        acc = fma4(tap(t - pos), d, acc);
    }
    const int k = pos - (sr.len - n);
    if (q.d_state_out && k >= 0) acc = add4(acc, load4(static_cast<const T *>(q.d_state_out) + ((size_t)s * n + k) * p.D + c));
    store4(static_cast<TG *>(q.d_state_in) + ((size_t)s * n + r) * p.D + c, acc);
}

// Partial sums of the CTA rows in a fixed order: 8 warps take every eighth, then meet in shared memory.
__global__ void __launch_bounds__(256) conv_bwd_sum_kernel(const float *part, float *d_w, float *d_bias, int nparts, int D, int width)
{
    __shared__ float red[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, j = blockIdx.y;
    float o = 0.f;
    if (c < D)
        for (int k = warp; k < nparts; k += 8) o += part[((size_t)k * (width + 1) + j) * D + c];
    red[warp][lane] = o;
    __syncthreads();
    if (warp != 0 || c >= D) return;
    o = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) o += red[k][lane];
    if (j < width) {
        if (d_w) d_w[(size_t)c * width + j] = o;
    } else if (d_bias) {
        d_bias[c] = o;
    }
}

int conv_bwd_rows(int T, int D)
{
    // CTA rows that walk the work items: about two CTAs per SM (as many as are resident) over all channel columns, no
    // more than there are items
    const int cols = (D / 4 + 31) / 32;
    const int want = (148 * 2 + cols - 1) / cols, most = (T / kBwdTok + 8) / 8;
    return want < most ? want : (most < 1 ? 1 : most);
}

template <typename T, int W>
chela_status_t fwd_launch(const ConvParams &p, cudaStream_t stream)
{
    constexpr size_t smem = 2 * 4 * 256 * sizeof(Raw4<T>);
    static_assert(smem <= 48 * 1024, "more has to be asked for");
    const long long items = (long long)packed_blocks(p.T, p.S + p.rest, kTok) * (p.D / 4);
    const long long need = (items + 255) / 256;
    conv_carry_kernel<T, W><<<(unsigned)(need < 148 * 64 ? need : 148 * 64), 256, smem, stream>>>(p, items);
    return last_launch_status();
}

template <typename T>
chela_status_t fwd_w(const ConvParams &p, cudaStream_t stream)
{
    switch (p.width) {
    case 1: return fwd_launch<T, 1>(p, stream);
    case 2: return fwd_launch<T, 2>(p, stream);
    case 3: return fwd_launch<T, 3>(p, stream);
    case 4: return fwd_launch<T, 4>(p, stream);
    case 5: case 6: case 7: case 8: return fwd_launch<T, 8>(p, stream);
    default: return fwd_launch<T, 16>(p, stream);
    }
}

template <typename T>
chela_status_t step_w(const ConvParams &p, cudaStream_t stream)
{
    const long long need = ((long long)p.S * (p.D / 4) + 127) / 128;
    if (need > 0x7fffffffLL) return CHELA_ERR_UNSUPPORTED;
    const unsigned grid = (unsigned)need;
    switch (p.width) {
    case 1: conv_step_kernel<T, 1><<<grid, 128, 0, stream>>>(p); break;
    case 2: conv_step_kernel<T, 2><<<grid, 128, 0, stream>>>(p); break;
    case 3: conv_step_kernel<T, 3><<<grid, 128, 0, stream>>>(p); break;
    case 4: conv_step_kernel<T, 4><<<grid, 128, 0, stream>>>(p); break;
    case 5: case 6: case 7: case 8: conv_step_kernel<T, 8><<<grid, 128, 0, stream>>>(p); break;
    default: conv_step_kernel<T, 16><<<grid, 128, 0, stream>>>(p); break;
    }
    return last_launch_status();
}

template <typename T, typename TG>
chela_status_t bwd_w(const ConvBwdParams &q, float *d_w, float *d_bias, cudaStream_t stream)
{
    const ConvParams &p = q.f;
    const long long nblocks = (long long)packed_blocks(p.T, p.S + p.rest, kBwdTok);
    const int rows = conv_bwd_rows(p.T, p.D);
    const dim3 grid((p.D / 4 + 31) / 32, rows);
    constexpr size_t smem = 2 * 4 * 2 * 256 * sizeof(Raw4<T>);
    auto launch = [&](auto kern) {
        if (smem > 40 * 1024) {   // with the static part, past the 48 KB that need no asking
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return cuda_status(e);
        }
        kern<<<grid, 256, smem, stream>>>(q, nblocks);
        return last_launch_status();
    };
    chela_status_t st;
    switch (p.width) {
    case 1: st = launch(conv_bwd_kernel<T, TG, 1>); break;
    case 2: st = launch(conv_bwd_kernel<T, TG, 2>); break;
    case 3: st = launch(conv_bwd_kernel<T, TG, 3>); break;
    case 4: st = launch(conv_bwd_kernel<T, TG, 4>); break;
    case 5: case 6: case 7: case 8: st = launch(conv_bwd_kernel<T, TG, 8>); break;
    default: st = launch(conv_bwd_kernel<T, TG, 16>); break;
    }
    if (st == CHELA_OK && q.part) {
        conv_bwd_sum_kernel<<<dim3((p.D + 31) / 32, p.width + 1), 256, 0, stream>>>(q.part, d_w, d_bias, rows, p.D, p.width);
        st = last_launch_status();
    }
    if (st == CHELA_OK && q.d_state_in) {
        const long long n = (long long)p.S * (p.width - 1) * (p.D / 4);
        conv_bwd_state_kernel<T, TG><<<(unsigned)((n + 127) / 128), 128, 0, stream>>>(q);
        st = last_launch_status();
    }
    return st;
}

}  // namespace

chela_status_t launch_shortconv_carry(const void *x, long long x_stride, const float *w, const float *bias, void *y,
                                      const void *state_in, void *state_out, const int *seq_offsets, int S, int T, int D, int width,
                                      int act, chela_dtype_t io_dtype, cudaStream_t stream)
{
    const bool held = width > 1;
    const ConvParams p = {x, x_stride, w, bias, y, held ? state_in : nullptr, held ? state_out : nullptr, seq_offsets, S, T, D, width,
                          act & 1, seq_offsets && (act & CHELA_ZERO_REST)};
    return io_dtype == CHELA_F32 ? fwd_w<float>(p, stream) : fwd_w<__nv_bfloat16>(p, stream);
}

chela_status_t launch_shortconv_step(const void *x, long long x_stride, const float *w, const float *bias, void *y, const void *state_in,
                                     void *state_out, int S, int D, int width, int act, chela_dtype_t io_dtype, cudaStream_t stream)
{
    const ConvParams p = {x, x_stride, w, bias, y, state_in, state_out, nullptr, S, S, D, width, act & 1, 0};
    return io_dtype == CHELA_F32 ? step_w<float>(p, stream) : step_w<__nv_bfloat16>(p, stream);
}

size_t shortconv_bwd_workspace_bytes(int T, int D, int width)
{
    return align_up((size_t)conv_bwd_rows(T, D) * (width + 1) * D * sizeof(float), 256);
}

chela_status_t launch_shortconv_bwd(const void *x, long long x_stride, const float *w, const float *bias, const void *d_y,
                                    long long d_y_stride, const void *state_in, const void *d_state_out, void *d_x, float *d_w,
                                    float *d_bias, void *d_state_in, const int *seq_offsets, int S, int T, int D, int width, int act,
                                    chela_dtype_t io_dtype, chela_dtype_t grad_dtype, void *workspace, cudaStream_t stream)
{
    const bool held = width > 1;
    ConvBwdParams q = {};
    q.f = ConvParams{x, x_stride, w, bias, nullptr, held ? state_in : nullptr, nullptr, seq_offsets, S, T, D, width, act & 1, seq_offsets != nullptr};
    q.dy = d_y;
    q.dys = d_y_stride;
    q.d_state_out = held ? d_state_out : nullptr;
    q.d_x = d_x;
    q.d_state_in = held ? d_state_in : nullptr;
    q.part = d_w || d_bias ? static_cast<float *>(workspace) : nullptr;
    if (io_dtype == CHELA_F32)
        return grad_dtype == CHELA_F32 ? bwd_w<float, float>(q, d_w, d_bias, stream) : bwd_w<float, __nv_bfloat16>(q, d_w, d_bias, stream);
    return grad_dtype == CHELA_F32 ? bwd_w<__nv_bfloat16, float>(q, d_w, d_bias, stream)
                                   : bwd_w<__nv_bfloat16, __nv_bfloat16>(q, d_w, d_bias, stream);
}

}  // namespace chela
