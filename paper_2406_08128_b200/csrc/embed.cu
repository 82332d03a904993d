// Token embedding and the gradient of its table:
//   out[t] = scale w[ids[t]],        d_w[v] = d_w_in[v] + scale sum_{t : ids[t] = v} d_out[t].
// Both are bound by HBM: the rows that are read and written, and for the gradient the whole table.
//
// The gradient sorts (id, t) by id, stably, in passes of up to 9 bits, so that the tokens of a row lie together in their
// order; no sum depends on the order of atomics.  Up to kClusterTokens tokens one cluster of eight CTAs sorts in its shared
// memory; more tokens take three launches a pass.
// The sorted tokens are cut into blocks of kBlock, a warp each for 256 columns, all of whose rows are loaded at once: table
// rows whose tokens lie inside a block are finished there, those that cross its ends leave partial sums that another kernel
// adds up in order.  However often one id occurs, no warp reads more than kBlock rows.
//
// Sort and sums are a chain of latencies; the rest of the table, the rows of ids that do not occur, is bound by HBM and needs
// neither.  So the launch behind the sort is a programmatic dependent of one CTA on each SM that the sort leaves: half of its
// warps fill the rest of the table from the start, the others wait for the sort and add up.
#include <cooperative_groups.h>

#include "packed.cuh"
#include "sm100_ptx.cuh"

namespace chela {
namespace {

namespace cg = cooperative_groups;
using sm100::griddep_launch_dependents;
using sm100::griddep_wait;

constexpr int kBlock = 16;
constexpr int kSortTile = 4096, kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kMaxBits = 9, kMaxBins = 1 << kMaxBits;

// Eight elements of a lane, of 256 that a warp takes: four at its column c and four at c + 128, so that every access of a warp
// covers whole sectors whatever the types (two halves of 32 bytes a lane would touch each sector twice).  second: c + 128 < D.
struct Vec8 {
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    template <typename T>
    __device__ __forceinline__ void load(const T *p, bool second)
    {
        a = load4(p);
        b = second ? load4(p + 128) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    template <typename T>
    __device__ __forceinline__ void store(T *p, bool second) const
    {
        store4(p, a);
        if (second) store4(p + 128, b);
    }
    __device__ __forceinline__ void scale(float f) { a.x *= f, a.y *= f, a.z *= f, a.w *= f, b.x *= f, b.y *= f, b.z *= f, b.w *= f; }
    __device__ __forceinline__ void add(float4 u, float4 v) { a.x += u.x, a.y += u.y, a.z += u.z, a.w += u.w, b.x += v.x, b.y += v.y, b.z += v.z, b.w += v.w; }
};
// The same as they lie in memory.
template <typename T>
struct Raw8 {
    Raw4<T> a, b;
    __device__ __forceinline__ void load(const T *p, bool second)
    {
        a.load(p);
        if (second) b.load(p + 128); else b.zero();
    }
    __device__ __forceinline__ void add_to(Vec8 &s) const { s.add(a.get(), b.get()); }
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
        const Idx id = ids[t];
        const bool kept = id >= 0 && id < (Idx)V;
        const TI *row = w + (kept ? (long long)id : 0) * w_stride;
        if (sizeof(TI) == 2 && sizeof(TO) == 2) {   // eight columns in a row: whole sectors, half the accesses
            const int c = (int)(i % chunks) * 256 + lane * 8;
            if (c >= D) continue;
            uint4 u = make_uint4(0u, 0u, 0u, 0u);
            if (kept) {
                u = *reinterpret_cast<const uint4 *>(row + c);
                uint32_t *v = reinterpret_cast<uint32_t *>(&u);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = sm100::pack_bf16(__uint_as_float(v[e] << 16) * scale, __uint_as_float(v[e] & 0xffff0000u) * scale);
            }
            *reinterpret_cast<uint4 *>(out + t * D + c) = u;
            continue;
        }
        const int c = (int)(i % chunks) * 256 + lane * 4;
        const bool second = c + 128 < D;
        if (c >= D) continue;
        Vec8 x;
        x.zero();
        if (kept) {
            x.load(row + c, second);
            x.scale(scale);
        }
        x.store(out + t * D + c, second);
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

// ---- the same by one cluster, in shared memory --------------------------------------------------------------------------

constexpr int kCluster = 8, kPerCta = 8192, kClusterTokens = kCluster * kPerCta;
struct SortSmem {
    unsigned long long items[2][kPerCta];   // key and token; a pass reads the one and writes the other
    unsigned short off[kSortWarps][kMaxBins];
    int total[kMaxBins], base[kMaxBins], warp[kSortWarps];
};

// The lanes with this lane's digit, by a vote a bit (__match_any_sync takes a step for each different value).
__device__ __forceinline__ unsigned same_digit(int digit, int bits)
{
    unsigned same = __ballot_sync(0xffffffffu, digit >= 0);
    for (int i = 0; i < bits; ++i) {
        const unsigned votes = __ballot_sync(0xffffffffu, digit >> i & 1);
        same &= digit >> i & 1 ? votes : ~votes;
    }
    return same;
}

// The loops are rolled: a launch of few passes is bound by fetching its instructions, not by running them.
template <typename Idx>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kSortThreads, 1)
    cluster_sort_kernel(const Idx *ids, int T, int V, int passes, int bits, int *keys_out, int *from_out, int *crossing)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    griddep_launch_dependents();
    SortSmem &s = *reinterpret_cast<SortSmem *>(smem);
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = cluster.block_rank();
    const int per_cta = (T + kCluster - 1) / kCluster, per_thread = (per_cta + kSortThreads - 1) / kSortThreads, bins = 1 << bits;
    const int begin = rank * per_cta, mine = max(min(per_cta, T - begin), 0);
    if (rank == 0 && tid == 0) crossing[0] = 0;
#pragma unroll 4
    for (int i = tid; i < mine; i += kSortThreads) s.items[0][i] = (unsigned long long)(unsigned)key_of(ids[begin + i], V) << 32 | (unsigned)(begin + i);
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = 32 + pass * bits;
        const unsigned long long *items = s.items[pass & 1];
        for (int b = tid; b < kSortWarps * kMaxBins / 2; b += kSortThreads) reinterpret_cast<unsigned *>(s.off)[b] = 0;
        __syncthreads();
        // a warp's items are consecutive
        const int first = warp * per_thread * 32;
#pragma unroll 1
        for (int i = 0; i < per_thread; ++i) {
            const int at = first + i * 32 + lane, digit = at < mine ? (int)(items[at] >> shift) & (bins - 1) : -1;
            const unsigned same = same_digit(digit, bits);
            if (digit >= 0 && lane == __ffs(same) - 1) s.off[warp][digit] += (unsigned short)__popc(same);
            __syncwarp();
        }
        __syncthreads();
        if (tid < bins) {
            int sum = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) {
                const int c = s.off[w][tid];
                s.off[w][tid] = (unsigned short)sum;
                sum += c;
            }
            s.total[tid] = sum;
        }
        cluster.sync();   // totals are there
        {
            // entries of smaller digits, and of this one in the CTAs before
            int all = 0, ahead = 0;
            if (tid < bins)
#pragma unroll
                for (int r = 0; r < kCluster; ++r) {
                    const int c = *cluster.map_shared_rank(&s.total[tid], r);
                    ahead += r < rank ? c : 0;
                    all += c;
                }
            int sum = all;
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            if (lane == 31) s.warp[warp] = sum;
            __syncthreads();
            if (tid < bins) {
                for (int w = 0; w < warp; ++w) sum += s.warp[w];
                s.base[tid] = sum - all + ahead;
            }
            __syncthreads();
        }
#pragma unroll 1
        for (int i = 0; i < per_thread; ++i) {
            const int at = first + i * 32 + lane;
            const unsigned long long v = at < mine ? items[at] : 0;
            const int digit = at < mine ? (int)(v >> shift) & (bins - 1) : -1;
            const unsigned same = same_digit(digit, bits);
            if (digit >= 0) {
                const int to = s.base[digit] + s.off[warp][digit] + __popc(same & ((1u << lane) - 1u));
                if (pass + 1 < passes) {
                    const int cta = to / per_cta;
                    *cluster.map_shared_rank(&s.items[(pass & 1) ^ 1][to - cta * per_cta], cta) = v;
                } else {
                    keys_out[to] = (int)(v >> 32), from_out[to] = (int)(unsigned)v;
                }
            }
            __syncwarp();
            if (digit >= 0 && lane == __ffs(same) - 1) s.off[warp][digit] += (unsigned short)__popc(same);
            __syncwarp();
        }
        cluster.sync();   // items have arrived, and no CTA reads another's totals any more
    }
}

// ---- sums over the sorted tokens ------------------------------------------------------------------------------------

template <typename TO>
__device__ __forceinline__ void finish_row(const Vec8 &sum, float f, const TO *d_w_in, TO *d_w, long long at, bool second)
{
    Vec8 o;
    o.zero();
    if (d_w_in) o.load(d_w_in + at, second);
    o.a = make_float4(fmaf(sum.a.x, f, o.a.x), fmaf(sum.a.y, f, o.a.y), fmaf(sum.a.z, f, o.a.z), fmaf(sum.a.w, f, o.a.w));
    o.b = make_float4(fmaf(sum.b.x, f, o.b.x), fmaf(sum.b.y, f, o.b.y), fmaf(sum.b.z, f, o.b.z), fmaf(sum.b.w, f, o.b.w));
    o.store(d_w + at, second);
}

// Rows of ids that do not occur: d_w_in's, or zero.  A CTA's kFillThreads take a stretch of the rows and look through all ids for
// them.
constexpr int kFillThreads = 512, kSumThreads = 512;
constexpr int kFillRows = 8 * 32768;   // rows in a CTA's bitmap at a time
__device__ __forceinline__ void fill_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kFillThreads) : "memory"); }
template <typename Idx, typename TO>
__device__ __forceinline__ void fill_rows(const Idx *ids, const TO *d_w_in, TO *d_w, int T, int V, int D, int tid)
{
    __shared__ unsigned bitmap[kFillRows / 32];
    const int warp = tid >> 5, lane = tid & 31;
    const int first = (int)((long long)V * blockIdx.x / gridDim.x), end = (int)((long long)V * (blockIdx.x + 1) / gridDim.x);
    const unsigned per_row = D / (16 / sizeof(TO));
    for (int v0 = first; v0 < end; v0 += kFillRows) {
        const int rows = min(kFillRows, end - v0);
        for (int i = tid; i < (rows + 31) / 32; i += kFillThreads) bitmap[i] = 0;
        fill_sync();
#pragma unroll 8
        for (int t = tid; t < T; t += kFillThreads) {   // T is at most kClusterTokens
            const long long at = (long long)ids[t] - v0;
            // looked at first: a frequent id's word would be queued for by all
            if (at >= 0 && at < rows && !(*reinterpret_cast<volatile unsigned *>(&bitmap[at >> 5]) >> (at & 31) & 1u)) atomicOr(&bitmap[at >> 5], 1u << (at & 31));
        }
        fill_sync();
        // eight vectors of a lane at once: copies are bound by the loads in flight
        const uint4 *src = reinterpret_cast<const uint4 *>(d_w_in) + (long long)v0 * per_row;
        uint4 *dst = reinterpret_cast<uint4 *>(d_w) + (long long)v0 * per_row;
        const unsigned items = (unsigned)rows * per_row;
        for (unsigned i0 = warp * 256 + lane; i0 < items; i0 += kFillThreads * 8) {
            uint4 x[8];
            bool fill[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const unsigned i = i0 + 32 * k, row = i / per_row;
                fill[k] = i < items && !(bitmap[row >> 5] >> (row & 31) & 1u);
                x[k] = make_uint4(0u, 0u, 0u, 0u);
                if (d_w_in && fill[k]) x[k] = src[i];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (fill[k]) dst[i0 + 32 * k] = x[k];
        }
        fill_sync();
    }
}

// The end of a row's tokens in a block.  Out of line: the unrolled loop that calls it is straight-line code run once or twice a
// launch, and the time to fetch it shows.
template <typename TO>
__device__ __noinline__ void end_of_row(float4 a, float4 b, float scale, const TO *d_w_in, TO *d_w, long long at, float *partial, bool second)
{
    const Vec8 sum = {a, b};
    if (partial) sum.store(partial, second);
    else finish_row(sum, scale, d_w_in, d_w, at, second);
}

// The first kSumThreads: the sums of the blocks.  partial[2 b]: the sum of block b's first tokens where their row began in an
// earlier block; partial[2 b + 1]: of its last tokens where their row began in this block and goes on in the next.  Such rows
// are listed by the block they begin in (crossing[0] counts them); the list's order says nothing.
// The threads behind them (where ids are given): the rows of ids that do not occur.
template <typename Idx, typename TI, typename TO>
__global__ void __launch_bounds__(kSumThreads + kFillThreads, 1) table_kernel(const Idx *ids, const int *keys, const int *from, const TI *d_out, long long d_out_stride, const TO *d_w_in,
                                                                              TO *d_w, float *partial, int *crossing, int T, int V, int D, float scale)
{
    constexpr int kAhead = sizeof(TI) == 2 ? 8 : 4, kWarps = kSumThreads / 32;   // rows in flight
    const int lane = threadIdx.x & 31, chunks = (D + 255) / 256;
    const long long blocks = (T + kBlock - 1LL) / kBlock, items = blocks * chunks;
    griddep_launch_dependents();
    if (threadIdx.x >= kSumThreads) {
        fill_rows(ids, d_w_in, d_w, T, V, D, threadIdx.x - kSumThreads);
        return;
    }
    griddep_wait();
    // consecutive items go to different SMs
    for (long long i = (threadIdx.x >> 5) * (long long)gridDim.x + blockIdx.x; i < items; i += (long long)gridDim.x * kWarps) {
        const long long b = i / chunks, begin = b * kBlock;
        const int count = (int)min((long long)kBlock, T - begin), c = (int)(i % chunks) * 256 + lane * 4;
        const bool in = c < D, second = c + 128 < D;
        // lane l: token begin + l - 1, so that the neighbours on either side are at hand
        const long long at = begin + lane - 1;
        const int key = at >= 0 && lane <= kBlock + 1 && at < T ? keys[at] : V, src = lane >= 1 && lane <= count ? from[at] : 0;
        if (__shfl_sync(0xffffffffu, key, 1) >= V) continue;   // left out from here on
        if (d_w_in && key < V) {   // the table's rows, a cache line at a time
            const TO *row = d_w_in + (long long)key * D + (i % chunks) * 256;
            for (int l = 0; l < 256; l += 128 / sizeof(TO))
                if ((i % chunks) * 256 + l < D) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + l));
        }
        Vec8 sum;
        sum.zero();
        bool from_left = __shfl_sync(0xffffffffu, key, 0) == __shfl_sync(0xffffffffu, key, 1);
#pragma unroll 1
        for (int q = 0; q < count; q += kAhead) {
            Raw8<TI> x[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const long long row = __shfl_sync(0xffffffffu, src, q + k + 1);
                const int now = __shfl_sync(0xffffffffu, key, q + k + 1);
                if (q + k < count && in && now < V) x[k].load(d_out + row * d_out_stride + c, second);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int now = __shfl_sync(0xffffffffu, key, q + k + 1), after = __shfl_sync(0xffffffffu, key, q + k + 2);
                if (q + k >= count || now >= V) continue;
                x[k].add_to(sum);
                const bool to_right = q + k + 1 == kBlock && after == now;
                if (after != now || to_right) {
                    if (in)
                        end_of_row(sum.a, sum.b, scale, d_w_in, d_w, (long long)now * D + c,
                                   from_left || to_right ? partial + (2 * b + (from_left ? 0 : 1)) * (long long)D + c : nullptr, second);
                    if (to_right && !from_left && c == 0) crossing[1 + atomicAdd(crossing, 1)] = (int)b;
                    from_left = false;
                    sum.zero();
                }
            }
        }
    }
}

// The sum of a crossing row's partial sums first ... last - 1.
__device__ __forceinline__ Vec8 sum_partials(const float *partial, long long begin, long long first, long long last, int D, int c)
{
    Vec8 sum;
    sum.zero();
    if (c < D)
        for (long long q = first; q < last; q += 6) {
            Raw8<float> x[6];
#pragma unroll
            for (int k = 0; k < 6; ++k)
                if (q + k < last) x[k].load(partial + (2 * (q + k) + (q + k == begin)) * (long long)D + c, c + 128 < D);
#pragma unroll
            for (int k = 0; k < 6; ++k)
                if (q + k < last) x[k].add_to(sum);
        }
    return sum;
}

// Rows that cross blocks: the last tokens' sum of the block they begin in and the first tokens' sums of those behind it, in
// order.  A warp a row and 256 columns; rows of many blocks go to the CTA's warps together, a stretch of blocks each.
constexpr int kJoinThreads = 256;
template <typename TO>
__global__ void __launch_bounds__(kJoinThreads, 2) join_blocks_kernel(const int *keys, const float *partial, const TO *d_w_in, TO *d_w, const int *crossing, int T, int V, int D, float scale)
{
    constexpr int kAlone = 16, kQueue = 256, kWarps = kJoinThreads / 32;
    __shared__ float s_sum[kWarps][256 + 8];
    __shared__ int s_queue[kQueue], s_blocks[kQueue], s_queued;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunks = (D + 255) / 256;
    griddep_wait();
    const long long items = (long long)crossing[0] * chunks;
    for (long long i0 = blockIdx.x; i0 < items; i0 += (long long)gridDim.x * kQueue) {
        if (threadIdx.x == 0) s_queued = 0;
        __syncthreads();
        for (int j = warp; j < kQueue; j += kWarps) {
            const long long i = i0 + (long long)gridDim.x * j;
            if (i >= items) break;
            const long long b = crossing[1 + i / chunks];
            const int key = keys[(b + 1) * kBlock - 1], c = (int)(i % chunks) * 256 + lane * 4;
            // the last block that begins with this row, among the sorted keys: 32 places at a time
            long long lo = b + 1, left = (T + kBlock - 1LL) / kBlock - lo;   // it is in lo ... lo + left - 1
            bool near = true;                                                 // most rows end soon: the nearest 32 blocks first
            while (left > 1) {
                const long long stride = near ? 1 : (left + 31) / 32, q = lo + lane * stride;
                const int on = __popc(__ballot_sync(0xffffffffu, lane * stride < left && keys[q * kBlock] == key));
                lo += (on - 1) * stride;
                left = stride == 1 && on < 32 ? 1 : min(near ? left : stride, left - (on - 1) * stride);
                near = false;
            }
            const long long count = lo - b + 1;
            if (count > kAlone) {
                if (lane == 0) {
                    const int at = atomicAdd(&s_queued, 1);
                    s_queue[at] = j, s_blocks[at] = (int)count;
                }
                continue;
            }
            const Vec8 sum = sum_partials(partial, b, b, b + count, D, c);
            if (c < D) finish_row(sum, scale, d_w_in, d_w, (long long)key * D + c, c + 128 < D);
        }
        __syncthreads();
        for (int j = 0; j < s_queued; ++j) {
            const long long i = i0 + (long long)gridDim.x * s_queue[j], b = crossing[1 + i / chunks], count = s_blocks[j];
            const int key = keys[(b + 1) * kBlock - 1], c = (int)(i % chunks) * 256 + lane * 4;
            Vec8 sum = sum_partials(partial, b, b + count * warp / kWarps, b + count * (warp + 1) / kWarps, D, c);
            sum.store(&s_sum[warp][lane * 4], true);
            __syncthreads();
            if (warp == 0 && c < D) {
                for (int w = 1; w < kWarps; ++w) sum.add(load4(&s_sum[w][lane * 4]), load4(&s_sum[w][lane * 4 + 128]));
                finish_row(sum, scale, d_w_in, d_w, (long long)key * D + c, c + 128 < D);
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

// Rows of ids that do not occur where the tokens are many, from the bitmap of count_kernel.
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

int grid_for(long long items, long long per_cta, int most) { const long long g = (items + per_cta - 1) / per_cta; return (int)(g < most ? g : most); }

struct Plan {
    int passes, bits, tiles;
    size_t keys[2], from[2], counts, present, crossing, partial, bytes;
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
    const size_t blocks = (T + kBlock - 1LL) / kBlock;
    q.keys[0] = take((size_t)T * 4), q.from[0] = take((size_t)T * 4);
    if (T > kClusterTokens) {
        q.keys[1] = take((size_t)T * 4), q.from[1] = take((size_t)T * 4);
        q.counts = take(((size_t)1 << q.bits) * q.tiles * 4);
        q.present = take(((size_t)V + 31) / 32 * 4);
    }
    q.crossing = take((1 + blocks) * 4);
    q.partial = take(2 * blocks * D * 4);
    q.bytes = at;
    return q;
}

// Launch as a programmatic dependent of the kernel before it in the stream, which it waits for by griddep_wait.
template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), int grid, int threads, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid), cfg.blockDim = dim3(threads), cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// Sorted keys and tokens in keys[0], from[0], and the rows that no token changes.
template <typename Idx, typename TO>
chela_status_t arrange(const Idx *ids, int T, int V, int D, const TO *d_w_in, TO *d_w, const Plan &q, uint8_t *ws, int sms, cudaStream_t stream)
{
    int *crossing = (int *)(ws + q.crossing);
    if (T <= kClusterTokens) {
        auto sort = cluster_sort_kernel<Idx>;
        if (cudaFuncSetAttribute(sort, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortSmem)) != cudaSuccess) return CHELA_ERR_CUDA;
        sort<<<kCluster, kSortThreads, sizeof(SortSmem), stream>>>(ids, T, V, q.passes, q.bits, (int *)(ws + q.keys[0]), (int *)(ws + q.from[0]), crossing);
        return last_launch_status();
    }
    int *counts = (int *)(ws + q.counts);
    unsigned *present = (unsigned *)(ws + q.present);
    if (cudaMemsetAsync(present, 0, ((size_t)V + 31) / 32 * 4, stream) != cudaSuccess || cudaMemsetAsync(crossing, 0, 4, stream) != cudaSuccess) return CHELA_ERR_CUDA;
    const int bins = 1 << q.bits;
    for (int i = 0; i < q.passes; ++i) {
        const int to = (q.passes - 1 - i) & 1;   // the last pass writes keys[0]
        const int *keys = (const int *)(ws + q.keys[to ^ 1]), *from = (const int *)(ws + q.from[to ^ 1]);
        count_kernel<Idx><<<q.tiles, kSortThreads, 0, stream>>>(i ? nullptr : ids, keys, T, V, i * q.bits, bins, q.tiles, counts, present);
        sums_kernel<<<1, 1024, 0, stream>>>(counts, (long long)bins * q.tiles);
        place_kernel<Idx><<<q.tiles, kSortThreads, 0, stream>>>(i ? nullptr : ids, keys, from, T, V, i * q.bits, bins, q.tiles, counts, (int *)(ws + q.keys[to]), (int *)(ws + q.from[to]));
    }
    if (d_w_in != d_w) other_rows_kernel<TO><<<grid_for((long long)V * D / 8, 256, 8 * sms), 256, 0, stream>>>(present, d_w_in, d_w, V, D);
    return last_launch_status();
}

template <typename Idx, typename TI, typename TO>
chela_status_t embed_bwd(const Idx *ids, const TI *d_out, long long d_out_stride, const TO *d_w_in, TO *d_w, int T, int V, int D, float scale, uint8_t *ws, cudaStream_t stream)
{
    const Plan q = make_plan(T, V, D);
    const int sms = current_sm_count();
    const chela_status_t st = arrange(ids, T, V, D, d_w_in, d_w, q, ws, sms, stream);
    if (st != CHELA_OK) return st;
    const int *keys = (const int *)(ws + q.keys[0]), *from = (const int *)(ws + q.from[0]);
    int *crossing = (int *)(ws + q.crossing);
    float *partial = (float *)(ws + q.partial);
    const bool fill = T <= kClusterTokens && d_w_in != d_w;
    const long long items = (T + kBlock - 1LL) / kBlock * ((D + 255) / 256);
    const int most = sms > kCluster ? sms - kCluster : 1;   // one CTA on each SM that the sort leaves
    if (launch_after(table_kernel<Idx, TI, TO>, fill ? most : grid_for(items, 1, most), fill ? kSumThreads + kFillThreads : kSumThreads, stream, ids, keys, from, d_out, d_out_stride, d_w_in,
                     d_w, partial, crossing, T, V, D, scale) != cudaSuccess)
        return CHELA_ERR_CUDA;
    if (T > kBlock && launch_after(join_blocks_kernel<TO>, grid_for(items, 4, 2 * sms), kJoinThreads, stream, keys, partial, d_w_in, d_w, crossing, T, V, D, scale) != cudaSuccess)
        return CHELA_ERR_CUDA;
    return last_launch_status();
}

template <typename TI, typename TO>
chela_status_t embed_bwd(const void *ids, bool wide_ids, const void *d_out, long long d_out_stride, const void *d_w_in, void *d_w, int T, int V, int D, float scale, uint8_t *ws, cudaStream_t stream)
{
    if (wide_ids) return embed_bwd((const long long *)ids, (const TI *)d_out, d_out_stride, (const TO *)d_w_in, (TO *)d_w, T, V, D, scale, ws, stream);
    return embed_bwd((const int *)ids, (const TI *)d_out, d_out_stride, (const TO *)d_w_in, (TO *)d_w, T, V, D, scale, ws, stream);
}

template <typename Idx, typename TI>
void embed_to(const void *ids, const void *w, long long w_stride, void *out, int T, int V, int D, float scale, chela_dtype_t out_dtype, cudaStream_t stream)
{
    const int grid = grid_for((long long)T * ((D + 255) / 256), 8, 16 * current_sm_count());
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
    uint8_t *ws = reinterpret_cast<uint8_t *>(workspace);
    typedef __nv_bfloat16 bf16;
    if (d_out_dtype == CHELA_F32)
        return grad_dtype == CHELA_F32 ? embed_bwd<float, float>(ids, wide_ids, d_out, d_out_stride, d_w_in, d_w, T, V, D, scale, ws, stream)
                                       : embed_bwd<float, bf16>(ids, wide_ids, d_out, d_out_stride, d_w_in, d_w, T, V, D, scale, ws, stream);
    return grad_dtype == CHELA_F32 ? embed_bwd<bf16, float>(ids, wide_ids, d_out, d_out_stride, d_w_in, d_w, T, V, D, scale, ws, stream)
                                   : embed_bwd<bf16, bf16>(ids, wide_ids, d_out, d_out_stride, d_w_in, d_w, T, V, D, scale, ws, stream);
}

}  // namespace chela
