// The vocabulary's cross entropy and its gradients for a few tokens (up to 16; bf16 while the weights are few): the weights are
// read once in each pass, on the plain fp32 pipes.  A tile of 256 rows of tensor-core operands would be nearly empty; the
// backward pass needs the logits of a weight row, its own gradient and its share of d_h while the row is in shared memory, where
// the tensor-core path reads the weights twice and passes dz through memory.  fp32 operands keep all their bits without being
// split.
//
// A persistent CTA walks tiles of weight rows, copied two tiles ahead by bulk copies.  Few rows are bound by the instructions that
// they take, so the sums are two-wide (one instruction a pair of columns).  A warp takes 32 / kTokens rows and a share of the
// columns: 32 sums a lane, transposed and added over the lanes in 31 exchanges, after which lane i has the logit of row
// i / kTokens and token i % kTokens.  Backward, a thread then owns columns: with the tokens' values of its columns in registers
// it writes the rows' gradients and keeps its share of d_h.  (6 x 91800 x 352 fp32: 35 us forward, 88 backward, where the weights
// take 20 once and their gradients as long again; 467 us for both on the tensor cores.)
#include "packed.cuh"
#include "sm100_ptx.cuh"
#include "vocabloss.cuh"

namespace chela {
namespace {

using sm100::griddep_launch_dependents;
using sm100::griddep_wait;

constexpr int kThreads = 256, kWarps = 8;
constexpr int kSmemMost = 200 << 10, kSmemTwo = 108 << 10;   // of one CTA an SM, of two
// Two CTAs an SM wherever the registers allow it: one waits while the other adds.
constexpr bool two_ctas(int tokens, int quads, bool grad) { return !grad || tokens * quads <= 8; }

struct Few {
    const void *h, *w, *targets;
    long long h_stride, w_stride;
    int T, V, D, wide_ids, groups;      // groups: of 32 / kTokens rows in a tile (1, 2, 4 or 8)
    float c2, scale;                    // scale log2 e, scale
    int *head;                          // asynchronous status
    float2 *part;                       // [CTAs][16]
    float *zt;                          // [16]
    const float *lse, *d_loss, *d_lse;
    const void *dw_in;
    void *dw;
    float *dhp;                         // [CTAs][kTokens][D]
    WaitCtl wc;
};

__device__ __forceinline__ long long target_of(const Few &p, int t)
{
    return t >= p.T ? -1 : p.wide_ids ? reinterpret_cast<const long long *>(p.targets)[t] : reinterpret_cast<const int *>(p.targets)[t];
}

__device__ __forceinline__ void copy_bulk(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// The sum over the lanes of a[i], in lane i.
__device__ __forceinline__ float transpose_sum(float (&a)[32], int lane)
{
#pragma unroll
    for (int n = 16; n >= 1; n >>= 1)
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const bool upper = lane & n;
            const float keep = upper ? a[i + n] : a[i], send = upper ? a[i] : a[i + n];
            a[i] = keep + __shfl_xor_sync(0xffffffffu, send, n);
        }
    return a[0];
}

// Weight rows v0 ... into a tile, by one thread; the barrier completes when they are there.  Rows past the vocabulary are not copied:
// what the tile holds there is multiplied and then left out.
template <typename TW>
__device__ __forceinline__ void load_tile(TW *tile, uint32_t bar, const Few &p, long long v0, int rows)
{
    const int there = (int)min((long long)rows, p.V - v0);
    const uint32_t bytes = p.D * (uint32_t)sizeof(TW), dst = sm100::smem_u32(tile);
    const TW *src = reinterpret_cast<const TW *>(p.w) + v0 * p.w_stride;
    sm100::mbar_expect_tx(bar, there * bytes);
    if (p.w_stride == p.D) copy_bulk(dst, src, there * bytes, bar);
    else
        for (int r = 0; r < there; ++r) copy_bulk(dst + r * bytes, src + r * p.w_stride, bytes, bar);
}

__device__ __forceinline__ float2 lo2(const float4 &v) { return make_float2(v.x, v.y); }
__device__ __forceinline__ float2 hi2(const float4 &v) { return make_float2(v.z, v.w); }

// kGrad = false: running maximum and sum of each token over the CTA's rows, and the targets' logits.
// kGrad = true: d_w's rows (TG) and this CTA's share of d_h; a thread owns kQuads groups of four columns.
template <typename TW, typename TG, int kTokens, int kQuads, bool kGrad>
__global__ void __launch_bounds__(kThreads, two_ctas(kTokens, kQuads, kGrad) ? 2 : 1) few_kernel(const Few p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int kRows = 32 / kTokens;
    __shared__ float s_part[kWarps * 32];
    __shared__ __align__(16) float2 s_dz[kWarps * 32];   // each value twice
    __shared__ __align__(8) unsigned long long s_bar[2];
    __shared__ int s_gave_up;
    __shared__ float s_lse[kTokens], s_g1[kTokens], s_g0[kTokens];
    __shared__ long long s_target[kTokens];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, D = p.D;
    const int rows = kRows * p.groups, slices = kWarps / p.groups, group = warp % p.groups, slice = warp / p.groups;
    float *s_h = reinterpret_cast<float *>(smem);
    TW *tiles = reinterpret_cast<TW *>(s_h + kTokens * D);
    const unsigned count = (unsigned)((p.V + (long long)rows - 1) / rows);
    griddep_launch_dependents();
    const uint32_t bars = sm100::smem_u32(s_bar);
    if (tid == 0) {
        if (blockIdx.x == 0) p.head[0] = 0;
        s_gave_up = 0;
        sm100::mbar_init(bars, 1);
        sm100::mbar_init(bars + 8, 1);
        sm100::fence_barrier_init();
        sm100::fence_proxy_async();
        // (test hook: the first copy of CTA 0 left out, so that the wait for it runs out)
        for (int k = p.wc.skip_arrival && blockIdx.x == 0; k < 2 && blockIdx.x + k * gridDim.x < count; ++k)
            load_tile(tiles + (size_t)k * rows * D, bars + 8 * k, p, (blockIdx.x + (long long)k * gridDim.x) * rows, rows);
    }
    if (tid < kTokens) {
        const long long y = target_of(p, tid);
        const bool kept = y >= 0 && y < p.V;
        s_target[tid] = kept ? y : -1;
        if (kGrad) {
            const float g = kept && p.d_loss ? p.d_loss[tid] : 0.f, gl = kept && p.d_lse ? p.d_lse[tid] : 0.f;
            s_lse[tid] = kept ? p.lse[tid] * kLog2e : 0.f;
            s_g1[tid] = p.scale * (g + gl), s_g0[tid] = p.scale * g;
        }
    }
    __syncthreads();
    for (int i = tid; i < kTokens * D / 4; i += kThreads) {
        const int t = i * 4 / D, c = i * 4 - t * D;
        const float4 x = s_target[t] >= 0 ? load4(reinterpret_cast<const TW *>(p.h) + t * p.h_stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        store4(s_h + i * 4, x);
    }
    float run_m = -INFINITY, run_s = 0.f;
    // columns of this thread in the gradients: quads of a group of threads, the groups take rows in turn
    const int quads = D / 4, sets = kQuads == 1 ? max(1, kThreads / quads) : 1, set = kQuads == 1 ? tid / quads : 0, quad = kQuads == 1 ? tid % quads : tid;
    constexpr int kOwn = kGrad ? kQuads : 1;
    float2 acc_lo[kOwn][kTokens], acc_hi[kOwn][kTokens], h_lo[kOwn][kTokens], h_hi[kOwn][kTokens];
    if (kGrad) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kQuads; ++j)
#pragma unroll
            for (int t = 0; t < kTokens; ++t) {
                acc_lo[j][t] = acc_hi[j][t] = splat2(0.f);
                const int c = (quad + j * kThreads) * 4;
                const float4 x = c < D ? load4(s_h + t * D + c) : make_float4(0.f, 0.f, 0.f, 0.f);
                h_lo[j][t] = lo2(x), h_hi[j][t] = hi2(x);
            }
    }
    int step = 0;
    for (unsigned i = blockIdx.x; i < count; i += gridDim.x, ++step) {
        TW *tile = tiles + (size_t)(step & 1) * rows * D;
        if (!sm100::mbar_wait(bars + 8 * (step & 1), step >> 1 & 1, nullptr, p.wc.limit)) s_gave_up = 1;
        __syncthreads();
        if (s_gave_up) break;
        // (backward the columns' registers leave no room for two sums each)
        float2 a2[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) a2[e] = make_float2(0.f, 0.f);
        const TW *mine = tile + (size_t)group * kRows * D + lane * 4;
        const float *tokens = s_h + lane * 4;
#pragma unroll 1
        for (int c = slice * 128; c + lane * 4 < D; c += slices * 128) {
            float4 w[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) w[r] = load4(mine + r * D + c);
#pragma unroll
            for (int t = 0; t < kTokens; ++t) {
                const float4 x = load4(tokens + t * D + c);
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    float2 &s = a2[r * kTokens + t];
                    if (kGrad) s.x = fmaf(w[r].w, x.w, fmaf(w[r].z, x.z, fmaf(w[r].y, x.y, fmaf(w[r].x, x.x, s.x))));
                    else s = fma2v(hi2(w[r]), hi2(x), fma2v(lo2(w[r]), lo2(x), s));
                }
            }
        }
        float a[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) a[e] = kGrad ? a2[e].x : a2[e].x + a2[e].y;
        s_part[slice * p.groups * 32 + group * 32 + lane] = transpose_sum(a, lane);
        __syncthreads();
        if (tid < 32 * p.groups) {
            float z = 0.f;
            for (int s = 0; s < slices; ++s) z += s_part[s * p.groups * 32 + tid];
            z *= p.c2;
            const long long v = (long long)i * rows + tid / kTokens;
            const int t = tid % kTokens;
            if (!kGrad) {
                if (v < p.V) {
                    const float m = fmaxf(run_m, z);
                    run_s = run_s * rescale(run_m, m) + ex2(z - (m == -INFINITY ? 0.f : m));
                    run_m = m;
                    if (v == s_target[t]) p.zt[t] = z;
                }
            } else {
                float dz = s_g1[t] * ex2(z - s_lse[t]);
                if (v == s_target[t]) dz -= s_g0[t];
                // (a token that is left out by choice, not by its factor of zero: the weights may hold infinities)
                s_dz[tid] = v < p.V && s_target[t] >= 0 ? splat2(dz) : splat2(0.f);
            }
        }
        if (kGrad) {
            __syncthreads();
            if (set < sets)
#pragma unroll 2
                for (int r = set; r < rows && (long long)i * rows + r < p.V; r += sets) {
                    const long long v = (long long)i * rows + r;
#pragma unroll
                    for (int j = 0; j < kQuads; ++j) {
                        const int c = (quad + j * kThreads) * 4;
                        if (c >= D) continue;
                        const float4 w = load4(tile + (size_t)r * D + c);
                        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (p.dw_in) o = load4(reinterpret_cast<const TG *>(p.dw_in) + v * D + c);
                        float2 o_lo = lo2(o), o_hi = hi2(o);
#pragma unroll
                        for (int t = 0; t < kTokens; t += 2) {
                            const float4 pair = *reinterpret_cast<const float4 *>(s_dz + r * kTokens + t);   // two tokens
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float2 dz = e ? hi2(pair) : lo2(pair);
                                o_lo = fma2v(dz, h_lo[j][t + e], o_lo), o_hi = fma2v(dz, h_hi[j][t + e], o_hi);
                                acc_lo[j][t + e] = fma2v(dz, lo2(w), acc_lo[j][t + e]), acc_hi[j][t + e] = fma2v(dz, hi2(w), acc_hi[j][t + e]);
                            }
                        }
                        store4(reinterpret_cast<TG *>(p.dw) + v * D + c, make_float4(o_lo.x, o_lo.y, o_hi.x, o_hi.y));
                    }
                }
            __syncthreads();   // the tile has been read
        }
        if (tid == 0 && i + 2 * gridDim.x < count) {
            sm100::fence_proxy_async();   // ... before the copy engine writes it
            load_tile(tile, bars + 8 * (step & 1), p, (i + 2LL * gridDim.x) * rows, rows);
        }
    }
    __syncthreads();
    if (s_gave_up) {
        if (tid == 0) {
            atomicExch(p.head, (int)CHELA_ERR_TIMEOUT);
            for (int k = 0; k < 2; ++k) sm100::mbar_wait(bars + 8 * ((step + k) & 1), (step + k) >> 1 & 1, nullptr, p.wc.limit);   // copies in flight
        }
        return;
    }
    if (!kGrad) {
        s_part[tid] = run_m, s_dz[tid] = splat2(run_s);
        __syncthreads();
        if (tid < kTokens) {
            float m = -INFINITY, s = 0.f;
            for (int e = tid; e < 32 * p.groups; e += kTokens) m = fmaxf(m, s_part[e]);
            for (int e = tid; e < 32 * p.groups; e += kTokens) s += s_dz[e].x * rescale(s_part[e], m);
            p.part[blockIdx.x * 16 + tid] = make_float2(m, s);
        }
    } else if (kQuads > 1 || sets == 1) {
#pragma unroll
        for (int j = 0; j < kQuads; ++j)
#pragma unroll
            for (int t = 0; t < kTokens; ++t) {
                const int c = (quad + j * kThreads) * 4;
                if (c < D && set < sets) store4(p.dhp + ((size_t)blockIdx.x * kTokens + t) * D + c, make_float4(acc_lo[j][t].x, acc_lo[j][t].y, acc_hi[j][t].x, acc_hi[j][t].y));
            }
    } else {
        // the sets' shares in order, through the tokens' place in shared memory
        for (int s = 0; s < sets; ++s) {
            if (set == s)
#pragma unroll
                for (int t = 0; t < kTokens; ++t) {
                    float *to = s_h + t * D + quad * 4;
                    const float4 b = s ? load4(to) : make_float4(0.f, 0.f, 0.f, 0.f);
                    store4(to, make_float4(b.x + acc_lo[0][t].x, b.y + acc_lo[0][t].y, b.z + acc_hi[0][t].x, b.w + acc_hi[0][t].y));
                }
            __syncthreads();
        }
        for (int e = tid; e < kTokens * D / 4; e += kThreads) store4(p.dhp + (size_t)blockIdx.x * kTokens * D + e * 4, load4(s_h + e * 4));
    }
}

// lse and loss of a token, a CTA each, from the parts of the CTAs before; zero where it is left out.
__global__ void __launch_bounds__(kThreads) few_join_kernel(const Few p, int ctas, float *loss, float *lse)
{
    __shared__ float2 s_warp[kWarps];
    const int t = blockIdx.x, tid = threadIdx.x;
    const long long y = target_of(p, t);
    griddep_wait();
    float m = -INFINITY, s = 0.f;
    for (int q = tid; q < ctas; q += kThreads) {
        const float2 v = p.part[q * 16 + t];
        const float mm = fmaxf(m, v.x);
        s = s * rescale(m, mm) + v.y * rescale(v.x, mm), m = mm;
    }
    for (int o = 16; o; o >>= 1) {
        const float mo = __shfl_xor_sync(0xffffffffu, m, o), so = __shfl_xor_sync(0xffffffffu, s, o), mm = fmaxf(m, mo);
        s = s * rescale(m, mm) + so * rescale(mo, mm), m = mm;
    }
    if ((tid & 31) == 0) s_warp[tid >> 5] = make_float2(m, s);
    __syncthreads();
    if (tid == 0) {
        float mm = m, sum = 0.f;
        for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, s_warp[w].x);
        for (int w = 0; w < kWarps; ++w) sum += s_warp[w].y * rescale(s_warp[w].x, mm);
        const bool kept = y >= 0 && y < p.V;
        const float log_s = log1pf(sum - 1.f);   // the largest term is 1
        lse[t] = kept ? fmaf(mm, 0.6931471805599453f, log_s) : 0.f;
        loss[t] = kept ? fmaf(mm - p.zt[t], 0.6931471805599453f, log_s) : 0.f;
    }
}

// d_h: the CTAs' shares added up, 32 columns of a token a CTA, 32 shares side by side and then in order; zero where it is left out
// (its shares are sums of zeros, but of zeros times the weights).
template <typename TG>
__global__ void __launch_bounds__(kThreads) few_spread_kernel(const Few p, int ctas, int tokens, TG *d_h)
{
    __shared__ float4 s_sum[32][8];
    const int t = blockIdx.y, quad = threadIdx.x & 7, lot = threadIdx.x >> 3, c = blockIdx.x * 32 + quad * 4;
    const long long y = target_of(p, t);
    griddep_wait();
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < p.D && y >= 0 && y < p.V)
#pragma unroll 4
        for (int q = lot; q < ctas; q += 32) {
            const float4 x = load4(p.dhp + ((size_t)q * tokens + t) * p.D + c);
            s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
        }
    s_sum[lot][quad] = s;
    __syncthreads();
    if (lot == 0 && c < p.D) {
        for (int l = 1; l < 32; ++l) {
            const float4 x = s_sum[l][quad];
            s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
        }
        store4(d_h + (size_t)t * p.D + c, s);
    }
}

struct Plan {
    int tokens, quads, groups, ctas, smem;
    size_t part, zt, dhp, bytes;
};

bool make_plan(Plan &q, int T, int V, int D, chela_dtype_t in_dtype, bool grad)
{
    // fp32: 91800 x 352, forward and backward, 14 tokens 226 us here and 20 tokens 443 us on the tensor cores.  bf16: the tensor
    // cores' path takes 60 us and 1.5 us for a million weights, this one 15 us and 1.9 (up to 4 tokens), 2.7 (8) or 7 (16).
    const long long weights = (long long)V * D, most = T <= 4 ? 128LL << 20 : T <= 8 ? 32LL << 20 : 4LL << 20;
    if (T > 16 || (in_dtype != CHELA_F32 && weights > most)) return false;
    q.tokens = T <= 4 ? 4 : T <= 8 ? 8 : 16;
    q.quads = D <= 1024 ? 1 : D <= 2048 ? 2 : 4;
    if (D > 4096 || q.quads * q.tokens > 16) return false;   // 64 registers of sums and 64 of tokens a thread
    const long long es = (long long)dtype_size(in_dtype), tokens = 4LL * q.tokens * D, tile = 2LL * (32 / q.tokens) * D * es;   // two tiles of one group
    if (tokens + tile > kSmemMost) return false;
    const int sms = current_sm_count();
    // as many rows a tile as fit, but a tile for each CTA
    const bool two = two_ctas(q.tokens, q.quads, grad) && tokens + tile <= kSmemTwo;
    const int slots = two ? 2 * sms : sms, most_smem = two ? kSmemTwo : kSmemMost;
    q.groups = 8;
    while (q.groups > 1 && (tokens + tile * q.groups > most_smem || V < (long long)slots * q.groups * (32 / q.tokens))) q.groups >>= 1;
    q.smem = (int)(tokens + tile * q.groups);
    const long long rows = (long long)q.groups * (32 / q.tokens), count = (V + rows - 1) / rows;
    q.ctas = (int)(count < slots ? count : slots);
    q.zt = 256;
    q.part = 512;
    q.dhp = q.part + align_up((size_t)q.ctas * 16 * 8, 256);
    q.bytes = q.dhp + (grad ? (size_t)q.ctas * q.tokens * D * 4 : 0);
    return true;
}

template <typename... P, typename... A>
chela_status_t launch_after(void (*kernel)(P...), dim3 grid, cudaStream_t stream, const A &...args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid, cfg.blockDim = dim3(kThreads), cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr, cfg.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
}

template <typename TW, typename TG, int kTokens, int kQuads, bool kGrad>
chela_status_t launch_few(const Few &p, const Plan &q, cudaStream_t stream)
{
    auto kern = few_kernel<TW, TG, kTokens, kQuads, kGrad>;
    // (the limit is the function's, not the thread's: set to what this call takes, it would refuse another thread's wider rows)
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost) != cudaSuccess) return CHELA_ERR_CUDA;
    kern<<<q.ctas, kThreads, q.smem, stream>>>(p);
    return last_launch_status();
}
template <typename TW, typename TG>
chela_status_t launch_few_bwd(const Few &p, const Plan &q, cudaStream_t stream)
{
    if (q.tokens == 4) return q.quads == 1 ? launch_few<TW, TG, 4, 1, true>(p, q, stream) : q.quads == 2 ? launch_few<TW, TG, 4, 2, true>(p, q, stream) : launch_few<TW, TG, 4, 4, true>(p, q, stream);
    if (q.tokens == 8) return q.quads == 1 ? launch_few<TW, TG, 8, 1, true>(p, q, stream) : launch_few<TW, TG, 8, 2, true>(p, q, stream);
    return launch_few<TW, TG, 16, 1, true>(p, q, stream);
}
template <typename TW>
chela_status_t launch_few_fwd(const Few &p, const Plan &q, cudaStream_t stream)
{
    if (q.tokens == 4) return launch_few<TW, TW, 4, 1, false>(p, q, stream);
    if (q.tokens == 8) return launch_few<TW, TW, 8, 1, false>(p, q, stream);
    return launch_few<TW, TW, 16, 1, false>(p, q, stream);
}

Few make_few(const chela_vocabloss_args_t &a, const Plan &q, uint8_t *ws)
{
    Few p{};
    p.h = a.h, p.w = a.w, p.targets = a.targets, p.h_stride = a.h_stride, p.w_stride = a.w_stride;
    p.T = a.T, p.V = a.V, p.D = a.D, p.wide_ids = a.wide_ids, p.groups = q.groups, p.c2 = a.scale * kLog2e, p.scale = a.scale;
    p.head = (int *)ws, p.part = (float2 *)(ws + q.part), p.zt = (float *)(ws + q.zt), p.dhp = (float *)(ws + q.dhp);
    p.wc = current_wait_ctl();
    return p;
}

}  // namespace

size_t vocabloss_few_workspace_bytes(int T, int V, int D, chela_dtype_t in_dtype, bool grad)
{
    Plan q{};
    return make_plan(q, T, V, D, in_dtype, grad) ? q.bytes : 0;
}

chela_status_t launch_vocabloss_few_fwd(const chela_vocabloss_args_t &a, float *loss, float *lse, void *workspace, cudaStream_t stream)
{
    Plan q{};
    if (!make_plan(q, a.T, a.V, a.D, a.in_dtype, false)) return CHELA_ERR_UNSUPPORTED;
    const Few p = make_few(a, q, (uint8_t *)workspace);
    const chela_status_t st = a.in_dtype == CHELA_F32 ? launch_few_fwd<float>(p, q, stream) : launch_few_fwd<__nv_bfloat16>(p, q, stream);
    return st != CHELA_OK ? st : launch_after(few_join_kernel, dim3(a.T), stream, p, q.ctas, loss, lse);
}

chela_status_t launch_vocabloss_few_bwd(const chela_vocabloss_args_t &a, const float *lse, const float *d_loss, const float *d_lse, void *d_h, const void *d_w_in, void *d_w,
                                        chela_dtype_t grad_dtype, void *workspace, cudaStream_t stream)
{
    Plan q{};
    if (!make_plan(q, a.T, a.V, a.D, a.in_dtype, true)) return CHELA_ERR_UNSUPPORTED;
    Few p = make_few(a, q, (uint8_t *)workspace);
    p.lse = lse, p.d_loss = d_loss, p.d_lse = d_lse, p.dw_in = d_w_in, p.dw = d_w;
    const bool f32 = grad_dtype == CHELA_F32;
    const chela_status_t st = a.in_dtype == CHELA_F32 ? (f32 ? launch_few_bwd<float, float>(p, q, stream) : launch_few_bwd<float, __nv_bfloat16>(p, q, stream))
                                                      : (f32 ? launch_few_bwd<__nv_bfloat16, float>(p, q, stream) : launch_few_bwd<__nv_bfloat16, __nv_bfloat16>(p, q, stream));
    if (st != CHELA_OK) return st;
    const dim3 grid((a.D + 31) / 32, a.T);
    return f32 ? launch_after(few_spread_kernel<float>, grid, stream, p, q.ctas, q.tokens, (float *)d_h)
               : launch_after(few_spread_kernel<__nv_bfloat16>, grid, stream, p, q.ctas, q.tokens, (__nv_bfloat16 *)d_h);
}

}  // namespace chela
