// Token embedding and the gradient of its table:
//   out[t] = scale w[ids[t]],        d_w[v] = d_w_in[v] + scale sum_{t : ids[t] = v} d_out[t].
// Both are bound by HBM: the rows that are read and written, and for the gradient the whole table.
//
// The gradient sorts (id, t) by id, stably, in passes of up to 9 bits (counts, their sums, placing), so that the tokens of a
// row lie together in their order; no sum depends on the order of atomics.  The sorted tokens are cut into blocks of kBlock, a
// warp each for 256 columns: rows whose tokens lie inside a block are finished there, those that cross its ends leave a
// partial sum that a second kernel adds up in order.  However often one id occurs, no warp reads more than kBlock rows.
// Rows of ids that do not occur are filled by a third kernel, which knows them from a bitmap.
#include "packed.cuh"

namespace chela {
namespace {

constexpr int kBlock = 64;
constexpr int kSortTile = 4096, kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kMaxBits = 9, kMaxBins = 1 << kMaxBits;

struct Vec8 {
    float v[8];
    __device__ __forceinline__ void load(const float *p)
    {
        const float4 a = load4(p), b = load4(p + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p)
    {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    __device__ __forceinline__ void store(float *p) const
    {
        store4(p, make_float4(v[0], v[1], v[2], v[3]));
        store4(p + 4, make_float4(v[4], v[5], v[6], v[7]));
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// A warp takes a row and 256 columns at a time.
template <typename Idx, typename TI, typename TO>
__global__ void __launch_bounds__(256) embed_kernel(const Idx *ids, const TI *w, long long w_stride, TO *out, int T, int V, int D, float scale)
{
    const int lane = threadIdx.x & 31;
    const int chunks = (D + 255) / 256;
    const long long items = (long long)T * chunks, step = (long long)gridDim.x * 8;
    for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < items; i += step) {
        const long long t = i / chunks;
        const int c = (int)(i % chunks) * 256 + lane * 8;
        const Idx id = ids[t];
        if (c >= D) continue;
        Vec8 x;
        if (id >= 0 && id < (Idx)V) {
            x.load(w + (long long)id * w_stride + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[e] *= scale;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[e] = 0.f;
        }
        x.store(out + t * D + c);
    }
}

// ---- stable sort of (id, t) -----------------------------------------------------------------------------------------

// The key of a token: its id, or V for tokens that are left out, which the sort puts last.
template <typename Idx>
__device__ __forceinline__ int key_of(Idx id, int V) { return id >= 0 && id < (Idx)V ? (int)id : V; }

// Counts of a tile's digits to counts[digit][tile]; the first pass (ids given) also marks the ids that occur.
template <typename Idx>
__global__ void __launch_bounds__(kSortThreads) count_kernel(const Idx *ids, const int *keys, int T, int V, int shift, int bins, int tiles, int *counts, unsigned *present)
{
    __shared__ int s_count[kMaxBins];
    for (int b = threadIdx.x; b < bins; b += kSortThreads) s_count[b] = 0;
    __syncthreads();
    const long long begin = (long long)blockIdx.x * kSortTile;
    for (int i = threadIdx.x; i < kSortTile && begin + i < T; i += kSortThreads) {
        const int key = ids ? key_of(ids[begin + i], V) : keys[begin + i];
        atomicAdd(&s_count[key >> shift & (bins - 1)], 1);
        if (ids && key < V) atomicOr(&present[key >> 5], 1u << (key & 31));
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kSortThreads) counts[(long long)b * tiles + blockIdx.x] = s_count[b];
}

// counts -> the number of all entries before each, in one CTA.
__global__ void __launch_bounds__(1024) sums_kernel(int *counts, long long n)
{
    __shared__ int s_warp[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int before = 0;
    for (long long at = 0; at < n; at += 1024) {
        const int mine = at + tid < n ? counts[at + tid] : 0;
        int sum = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) s_warp[warp] = sum;
        __syncthreads();
        int total = 0, ahead = 0;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) ahead += s_warp[w];
            total += s_warp[w];
        }
        if (at + tid < n) counts[at + tid] = before + ahead + sum - mine;
        before += total;
        __syncthreads();
    }
}

// Places a tile's entries: base of the digit and tile, entries of the digit in the warps before, rank inside the warp.
template <typename Idx>
__global__ void __launch_bounds__(kSortThreads) place_kernel(const Idx *ids, const int *keys, const int *from, int T, int V, int shift, int bins, int tiles, const int *counts, int *keys_out, int *from_out)
{
    __shared__ unsigned short s_off[kSortWarps][kMaxBins];
    __shared__ int s_base[kMaxBins];
    constexpr int kPerWarp = kSortTile / kSortWarps;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    for (int b = tid; b < kSortWarps * kMaxBins; b += kSortThreads) (&s_off[0][0])[b] = 0;
    for (int b = tid; b < bins; b += kSortThreads) s_base[b] = counts[(long long)b * tiles + blockIdx.x];
    __syncthreads();
    const long long begin = (long long)blockIdx.x * kSortTile + warp * kPerWarp;
    int key[kPerWarp / 32], src[kPerWarp / 32];
#pragma unroll
    for (int i = 0; i < kPerWarp / 32; ++i) {
        const long long t = begin + i * 32 + lane;
        key[i] = t >= T ? -1 : ids ? key_of(ids[t], V) : keys[t];
        src[i] = t >= T ? 0 : ids ? (int)t : from[t];
        const int digit = key[i] < 0 ? -1 : key[i] >> shift & (bins - 1);
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        if (digit >= 0 && lane == __ffs(same) - 1) s_off[warp][digit] += (unsigned short)__popc(same);
        __syncwarp();
    }
    __syncthreads();
    for (int b = tid; b < bins; b += kSortThreads) {
        int sum = 0;
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = s_off[w][b];
            s_off[w][b] = (unsigned short)sum;
            sum += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPerWarp / 32; ++i) {
        const int digit = key[i] < 0 ? -1 : key[i] >> shift & (bins - 1);
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        if (digit >= 0) {
            const int at = s_base[digit] + s_off[warp][digit] + __popc(same & ((1u << lane) - 1u));
            keys_out[at] = key[i];
            from_out[at] = src[i];
        }
        __syncwarp();
        if (digit >= 0 && lane == __ffs(same) - 1) s_off[warp][digit] += (unsigned short)__popc(same);
        __syncwarp();
    }
}

// ---- sums over the sorted tokens ------------------------------------------------------------------------------------

template <typename TO>
__device__ __forceinline__ void finish_row(const Vec8 &sum, float scale, const TO *d_w_in, TO *d_w, long long at)
{
    Vec8 o;
    if (d_w_in) {
        o.load(d_w_in + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = fmaf(sum.v[e], scale, o.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = sum.v[e] * scale;
    }
    o.store(d_w + at);
}

// partial[2 b]: the sum of block b's first tokens where their row began in an earlier block; partial[2 b + 1]: of its last
// tokens where their row began in this block and goes on in the next.
template <typename TI, typename TO>
__global__ void __launch_bounds__(256) block_sums_kernel(const int *keys, const int *from, const TI *d_out, long long d_out_stride, const TO *d_w_in, TO *d_w, float *partial,
                                                         int T, int V, int D, float scale)
{
    const int lane = threadIdx.x & 31, chunks = (D + 255) / 256;
    const long long blocks = (T + kBlock - 1LL) / kBlock, items = blocks * chunks, step = (long long)gridDim.x * 8;
    for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < items; i += step) {
        const long long b = i / chunks, begin = b * kBlock, end = min(begin + kBlock, (long long)T);
        const int c = (int)(i % chunks) * 256 + lane * 8;
        const bool in = c < D;
        Vec8 sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum.v[e] = 0.f;
        bool from_left = begin > 0 && keys[begin - 1] == keys[begin];
        for (long long e0 = begin; e0 < end; e0 += 32) {
            // this group's keys and the one behind it
            const int key = e0 + lane < end ? keys[e0 + lane] : V, src = e0 + lane < end ? from[e0 + lane] : 0;
            const int behind = e0 + 32 < T ? keys[e0 + 32] : V;
            int next = __shfl_down_sync(0xffffffffu, key, 1);
            if (lane == 31) next = behind;
            const int count = (int)min(32LL, end - e0);
#pragma unroll 1
            for (int q = 0; q < count; q += 8) {
                Vec8 x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const long long row = __shfl_sync(0xffffffffu, src, q + k);
                    const int now = __shfl_sync(0xffffffffu, key, q + k);
                    if (q + k < count && in && now < V) x[k].load(d_out + row * d_out_stride + c);
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[k].v[e] = 0.f;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int now = __shfl_sync(0xffffffffu, key, q + k), after = __shfl_sync(0xffffffffu, next, q + k);
                    if (q + k >= count || now >= V) continue;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum.v[e] += x[k].v[e];
                    const bool last = e0 + q + k + 1 == end, to_right = last && e0 + q + k + 1 < T && after == now;
                    if (after != now || last) {
                        if (in) {
                            if (from_left || to_right) sum.store(partial + (2 * b + (from_left ? 0 : 1)) * (long long)D + c);
                            else finish_row(sum, scale, d_w_in, d_w, (long long)now * D + c);
                        }
                        from_left = false;
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum.v[e] = 0.f;
                    }
                }
            }
        }
    }
}

// Rows that cross blocks, by the block they begin in: its last tokens' sum and those of the blocks behind it, in order.
template <typename TO>
__global__ void __launch_bounds__(256) join_blocks_kernel(const int *keys, const float *partial, const TO *d_w_in, TO *d_w, int T, int V, int D, float scale)
{
    const int lane = threadIdx.x & 31, chunks = (D + 255) / 256;
    const long long blocks = (T + kBlock - 1LL) / kBlock, items = blocks * chunks, step = (long long)gridDim.x * 8;
    for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < items; i += step) {
        const long long b = i / chunks, begin = b * kBlock, end = begin + kBlock;
        if (end >= T) continue;
        const int key = keys[end - 1];
        if (key >= V || keys[end] != key) continue;                                  // nothing crosses this block's end
        if (begin > 0 && keys[begin - 1] == key) continue;                           // it began in an earlier block
        const int c = (int)(i % chunks) * 256 + lane * 8;
        // the last block with tokens of this row
        long long last = b + 1;
        for (;;) {
            const long long q = last + lane;   // does the row go on behind block q?
            const bool on = (q + 1) * kBlock < T && keys[(q + 1) * kBlock] == key;
            const unsigned votes = __ballot_sync(0xffffffffu, !on);
            if (votes) {
                last += __ffs(votes) - 1;
                break;
            }
            last += 32;
        }
        if (c >= D) continue;
        Vec8 sum;
        sum.load(partial + (2 * b + 1) * (long long)D + c);
        for (long long q = b + 1; q <= last; q += 8) {
            Vec8 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (q + k <= last) x[k].load(partial + 2 * (q + k) * (long long)D + c);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (q + k <= last)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum.v[e] += x[k].v[e];
        }
        finish_row(sum, scale, d_w_in, d_w, (long long)key * D + c);
    }
}

// Rows of ids that do not occur: d_w_in's, or zero.
template <typename TO>
__global__ void __launch_bounds__(256) other_rows_kernel(const unsigned *present, const TO *d_w_in, TO *d_w, int V, int D)
{
    constexpr int kVec = 16 / sizeof(TO);
    const long long per_row = D / kVec, items = per_row * V, step = gridDim.x * 256LL;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < items; i += step) {
        const int v = (int)(i / per_row);
        if (present[v >> 5] >> (v & 31) & 1u) continue;
        const uint4 x = d_w_in ? reinterpret_cast<const uint4 *>(d_w_in)[i] : make_uint4(0u, 0u, 0u, 0u);
        reinterpret_cast<uint4 *>(d_w)[i] = x;
    }
}

int sm_count()
{
    int sms = 0, dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) sms = 148;
    return sms;
}
int grid_for(long long items, long long per_cta, int most) { const long long g = (items + per_cta - 1) / per_cta; return (int)(g < most ? g : most); }

struct Plan {
    int passes, bits, tiles;
    size_t keys[2], from[2], counts, present, partial, bytes;
};
Plan make_plan(int T, int V, int D)
{
    Plan q{};
    int bits = 1;
    while (bits < 31 && (1LL << bits) <= V) ++bits;   // keys 0 ... V
    q.passes = (bits + kMaxBits - 1) / kMaxBits;
    q.bits = (bits + q.passes - 1) / q.passes;
    q.tiles = (int)((T + kSortTile - 1LL) / kSortTile);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes, 256);
        return here;
    };
    for (int i = 0; i < 2; ++i) q.keys[i] = take((size_t)T * 4), q.from[i] = take((size_t)T * 4);
    q.counts = take(((size_t)1 << q.bits) * q.tiles * 4);
    q.present = take(((size_t)V + 31) / 32 * 4);
    q.partial = take((size_t)2 * ((T + kBlock - 1LL) / kBlock) * D * 4);
    q.bytes = at;
    return q;
}

template <typename Idx>
chela_status_t sort_ids(const Idx *ids, int T, int V, const Plan &q, uint8_t *ws, cudaStream_t stream)
{
    int *counts = (int *)(ws + q.counts);
    unsigned *present = (unsigned *)(ws + q.present);
    if (cudaMemsetAsync(present, 0, ((size_t)V + 31) / 32 * 4, stream) != cudaSuccess) return CHELA_ERR_CUDA;
    const int bins = 1 << q.bits;
    for (int i = 0; i < q.passes; ++i) {
        const int *keys = (const int *)(ws + q.keys[(i + 1) & 1]), *from = (const int *)(ws + q.from[(i + 1) & 1]);
        count_kernel<Idx><<<q.tiles, kSortThreads, 0, stream>>>(i ? nullptr : ids, keys, T, V, i * q.bits, bins, q.tiles, counts, present);
        sums_kernel<<<1, 1024, 0, stream>>>(counts, (long long)bins * q.tiles);
        place_kernel<Idx><<<q.tiles, kSortThreads, 0, stream>>>(i ? nullptr : ids, keys, from, T, V, i * q.bits, bins, q.tiles, counts, (int *)(ws + q.keys[i & 1]), (int *)(ws + q.from[i & 1]));
    }
    return last_launch_status();
}

template <typename TI, typename TO>
chela_status_t sum_rows(const TI *d_out, long long d_out_stride, const TO *d_w_in, TO *d_w, int T, int V, int D, float scale, const Plan &q, uint8_t *ws, cudaStream_t stream)
{
    const int sms = sm_count(), at = (q.passes - 1) & 1;
    const int *keys = (const int *)(ws + q.keys[at]), *from = (const int *)(ws + q.from[at]);
    float *partial = (float *)(ws + q.partial);
    const long long items = (T + kBlock - 1LL) / kBlock * ((D + 255) / 256);
    if (d_w_in != d_w) other_rows_kernel<TO><<<grid_for((long long)V * D / 8, 256, 8 * sms), 256, 0, stream>>>((const unsigned *)(ws + q.present), d_w_in, d_w, V, D);
    block_sums_kernel<TI, TO><<<grid_for(items, 8, 4 * sms), 256, 0, stream>>>(keys, from, d_out, d_out_stride, d_w_in, d_w, partial, T, V, D, scale);
    if (T > kBlock) join_blocks_kernel<TO><<<grid_for(items, 8, 8 * sms), 256, 0, stream>>>(keys, partial, d_w_in, d_w, T, V, D, scale);
    return last_launch_status();
}

template <typename Idx, typename TI>
void embed_to(const void *ids, const void *w, long long w_stride, void *out, int T, int V, int D, float scale, chela_dtype_t out_dtype, cudaStream_t stream)
{
    const int grid = grid_for((long long)T * ((D + 255) / 256), 8, 16 * sm_count());
    if (out_dtype == CHELA_F32) embed_kernel<Idx, TI, float><<<grid, 256, 0, stream>>>((const Idx *)ids, (const TI *)w, w_stride, (float *)out, T, V, D, scale);
    else embed_kernel<Idx, TI, __nv_bfloat16><<<grid, 256, 0, stream>>>((const Idx *)ids, (const TI *)w, w_stride, (__nv_bfloat16 *)out, T, V, D, scale);
}

}  // namespace

chela_status_t launch_embed_fwd(const void *ids, bool wide_ids, const void *w, long long w_stride, void *out, int T, int V, int D, float scale, chela_dtype_t w_dtype,
                                chela_dtype_t out_dtype, cudaStream_t stream)
{
    if (w_dtype == CHELA_F32) {
        if (wide_ids) embed_to<long long, float>(ids, w, w_stride, out, T, V, D, scale, out_dtype, stream);
        else embed_to<int, float>(ids, w, w_stride, out, T, V, D, scale, out_dtype, stream);
    } else {
        if (wide_ids) embed_to<long long, __nv_bfloat16>(ids, w, w_stride, out, T, V, D, scale, out_dtype, stream);
        else embed_to<int, __nv_bfloat16>(ids, w, w_stride, out, T, V, D, scale, out_dtype, stream);
    }
    return last_launch_status();
}

size_t embed_bwd_workspace_bytes(int T, int V, int D) { return make_plan(T, V, D).bytes; }

chela_status_t launch_embed_bwd(const void *ids, bool wide_ids, const void *d_out, long long d_out_stride, const void *d_w_in, void *d_w, int T, int V, int D, float scale,
                                chela_dtype_t d_out_dtype, chela_dtype_t grad_dtype, void *workspace, cudaStream_t stream)
{
    const Plan q = make_plan(T, V, D);
    uint8_t *ws = reinterpret_cast<uint8_t *>(workspace);
    const chela_status_t st = wide_ids ? sort_ids((const long long *)ids, T, V, q, ws, stream) : sort_ids((const int *)ids, T, V, q, ws, stream);
    if (st != CHELA_OK) return st;
    typedef __nv_bfloat16 bf16;
    if (d_out_dtype == CHELA_F32)
        return grad_dtype == CHELA_F32 ? sum_rows((const float *)d_out, d_out_stride, (const float *)d_w_in, (float *)d_w, T, V, D, scale, q, ws, stream)
                                       : sum_rows((const float *)d_out, d_out_stride, (const bf16 *)d_w_in, (bf16 *)d_w, T, V, D, scale, q, ws, stream);
    return grad_dtype == CHELA_F32 ? sum_rows((const bf16 *)d_out, d_out_stride, (const float *)d_w_in, (float *)d_w, T, V, D, scale, q, ws, stream)
                                   : sum_rows((const bf16 *)d_out, d_out_stride, (const bf16 *)d_w_in, (bf16 *)d_w, T, V, D, scale, q, ws, stream);
}

}  // namespace chela
