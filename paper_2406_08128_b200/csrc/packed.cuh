// Helpers of the operators over packed sequences (short convolution with carried inputs, selective scan, block norms).
#pragma once
#include "common.cuh"

namespace chela {

// Tokens of one sequence.  Offsets come from the device unchecked by the host, so they are clamped to [0, T] here:
// a bad array then gives wrong results, never an access outside the tensors.
struct SeqRange {
    int start, len;
};
__device__ __forceinline__ int seq_start(const int *off, int s, int S, int T)
{
    return off ? min(max(off[s], 0), T) : (int)((long long)T / S * s);
}
__device__ __forceinline__ SeqRange seq_range(const int *off, int s, int S, int T)
{
    SeqRange r;
    r.start = seq_start(off, s, S, T);
    r.len = max(seq_start(off, s + 1, S, T) - r.start, 0);
    return r;
}

// Blocks of K tokens that do not cross sequences, numbered without knowing the lengths on the host: sequence s owns the
// blocks start_s / K + s ... start_{s+1} / K + s.  That is at least one and at least ceil(len / K) blocks, and there are
// at most T / K + S in all.
inline size_t packed_blocks(int T, int S, int K) { return (size_t)T / K + S; }
__device__ __forceinline__ int packed_block_seq(const int *off, int S, int T, int K, long long block)
{
    int lo = 0, hi = S - 1;   // the last s with start_s / K + s <= block
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((long long)(seq_start(off, mid, S, T) / K) + mid <= block) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// (With S + 1 for S the tokens behind the last sequence count as one more.)

// The sequence with the `rank`-th most tokens, for kernels whose CTAs walk whole sequences: the CTAs that start first get
// the long ones, so that none of those is left for the end.  Packed sequences only, and no more of them than the CTA has
// threads (else rank itself: the order of the array).  All threads call it; s_len has blockDim.x + 1 ints.
__device__ __forceinline__ int seq_by_length(const int *off, int S, int T, int rank, int *s_len)
{
    if (!off || S == 1 || S > (int)blockDim.x) return rank;
    const int tid = threadIdx.x;
    if (tid < S) s_len[tid] = seq_range(off, tid, S, T).len;
    __syncthreads();
    if (tid < S) {
        const int mine = s_len[tid];
        int longer = 0;
        for (int j = 0; j < S; ++j) longer += s_len[j] > mine || (s_len[j] == mine && j < tid);
        if (longer == rank) s_len[blockDim.x] = tid;
    }
    __syncthreads();
    return s_len[blockDim.x];
}

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Added to the exponent x of a decay 2^x that a recurrence multiplies up.  Over the tokens that a slow state remembers the
// mean error of the approximate exponential adds up where the rest of it does not.  Mean errors measured over a million
// arguments an octave, in steps of 2^-24:
//     -x                      2^-19 .. 2^-8    2^-8 .. 2^-1    2^-1 .. 1    above 1
//     as it is                -0.17 .. -0.09   -0.44 .. -0.26  -0.42        -0.83 .. -0.85
//     kDecayShift             +0.13 .. +0.22   -0.14 .. +0.04  -0.11        -0.53
//     kSlowDecayShift         -0.05 .. +0.03   -0.33 .. -0.15  -0.30        -0.72
// so exponents closer to zero than kSlowExponent get the smaller one.  Closer to zero than 2^-19 the mean errors with that
// one are -0.12 (2^-20), -0.06 (2^-21), -0.22 (2^-22); below 2^-23 the exponential is 1.  Growing states (x > 0, errors of
// +0.12 and more as it is) get none.  2^x at x = 0 stays 1.
constexpr float kDecayShift = 2.6e-8f, kSlowDecayShift = 1.0e-8f, kSlowExponent = 0x1p-8f;
__device__ __forceinline__ float decay(float rate, float dt)
{
    const float x = rate * dt, shift = x < -kSlowExponent ? kDecayShift : kSlowDecayShift;
    return ex2(fmaf(rate, dt, x < 0.f ? shift : 0.f));
}
// The same for the states that a lane holds of one channel and for a few tokens in a row, with one choice for all of them:
// that of the slowest state at the first of the tokens.  A fast state forgets the error; and where the first token is a
// fast one, every state forgets within a few hundred groups of tokens what the larger shift does to the slower ones.  (8 x
// 8192 x 1024, N = 16: 550 us, with a choice for every token 556 to 612, with one constant for all exponents 537.)  No shift where one of the rates is above zero; a time step below zero is not
// looked for.
struct DecayShift {
    float slow_below, slow;   // time steps below the first: the second, others kDecayShift
    template <int NP>
    __device__ __forceinline__ void set(const float2 (&rates)[NP])
    {
        float least = fabsf(rates[0].x), most = rates[0].x;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            least = fminf(least, fminf(fabsf(rates[k].x), fabsf(rates[k].y)));
            most = fmaxf(most, fmaxf(rates[k].x, rates[k].y));
        }
        slow_below = most > 0.f ? INFINITY : kSlowExponent / least;
        slow = most > 0.f ? 0.f : kSlowDecayShift;
    }
    __device__ __forceinline__ float2 at(float dt) const
    {
        const float v = dt < slow_below ? slow : kDecayShift;
        return make_float2(v, v);
    }
};
__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// sigmoid; for u far below zero the reciprocal of infinity is 0
__device__ __forceinline__ float sigmoid_acc(float u) { return rcp_approx(1.0f + ex2(-u * kLog2e)); }

// pairs of fp32 values in one instruction
__device__ __forceinline__ float2 mul2v(float2 a, float2 b)
{
    float2 d;
    asm("{ .reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mul.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2v(float2 a, float2 b)
{
    float2 d;
    asm("{ .reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2v(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{ .reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 x, x, y, z;"
        " mov.b64 {%0, %1}, x; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 splat2(float a) { return make_float2(a, a); }

// log(1 + e^v) = max(v, 0) + log1p(e^-|v|).  log1p(e)/e on [0, 1] is a polynomial of degree 9 fitted for this file
// (weighted least squares iterated to equal ripple, relative error 5e-9; 1.6e-7 with fp32 Horner steps): the logarithm
// of the rounded sum 1 + e would lose the small time steps (e = 1e-3 .. 1e-1) that these models work with.  The
// exponential's argument |v| log2(e) is rounded to p; what p lost, |v| - p ln 2, is put back to first order.
__device__ __forceinline__ float2 softplus_acc(float2 v)
{
    // NaN stays; above 100 the exponential is below every normal number
    const float2 x = make_float2(fabsf(v.x) > 100.f ? 100.f : fabsf(v.x), fabsf(v.y) > 100.f ? 100.f : fabsf(v.y));
    const float2 t = mul2v(x, splat2(kLog2e)), r = fma2v(t, splat2(0.6931471805599453f), make_float2(-x.x, -x.y));
    float2 e = make_float2(ex2(-t.x), ex2(-t.y));
    e = fma2v(e, r, e);
    float2 p = splat2(-3.244025400e-03f);
    p = fma2v(p, e, splat2(1.985146478e-02f));
    p = fma2v(p, e, splat2(-5.695954338e-02f));
    p = fma2v(p, e, splat2(1.060365662e-01f));
    p = fma2v(p, e, splat2(-1.530559361e-01f));
    p = fma2v(p, e, splat2(1.967594028e-01f));
    p = fma2v(p, e, splat2(-2.495413423e-01f));
    p = fma2v(p, e, splat2(3.332996368e-01f));
    p = fma2v(p, e, splat2(-4.999990165e-01f));
    p = fma2v(p, e, splat2(1.0f));
    return fma2v(p, e, make_float2(fmaxf(v.x, 0.f), fmaxf(v.y, 0.f)));
}
__device__ __forceinline__ float softplus_acc(float v) { return softplus_acc(splat2(v)).x; }

// Four consecutive elements as they lie in memory: loads that are issued ahead wait in half the registers.
template <typename T>
struct Raw4;
template <>
struct Raw4<float> {
    float4 v;
    __device__ __forceinline__ void load(const float *p) { v = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void zero() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ float4 get() const { return v; }
};
template <>
struct Raw4<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint2 *>(p); }
    __device__ __forceinline__ void zero() { v = make_uint2(0u, 0u); }
    __device__ __forceinline__ float4 get() const
    {
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                           __uint_as_float(v.y & 0xffff0000u));
    }
};

// 16 bytes from global to shared memory, asynchronously; zeros where ok is false (the address is then not read)
__device__ __forceinline__ void copy16(void *dst, const void *src, bool ok)
{
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(ok ? 16 : 0) : "memory");
}

// Four elements (8 or 16 bytes) of one lane, asynchronously; zeros where ok is false.  The lane that copied reads them.
template <typename T>
__device__ __forceinline__ void copy_raw4(Raw4<T> *dst, const T *src, bool ok)
{
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if (sizeof(T) == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(ok ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(d), "l"(src), "r"(ok ? 8 : 0) : "memory");
}

}  // namespace chela
