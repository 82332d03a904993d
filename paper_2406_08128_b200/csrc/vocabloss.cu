// Softmax cross entropy of hidden rows against a vocabulary's weight rows, and its gradients, without the T x V logits in
// memory:
//   z[t,v] = scale <h_t, w_v>,  lse_t = log sum_v e^z[t,v],  loss_t = lse_t - z[t,y_t],
//   dz[t,v] = scale ((d_loss_t + d_lse_t) e^(z[t,v] - lse_t) - d_loss_t [v = y_t]),   d_h = dz w,   d_w = dz^T h.
//
// Bound by the tensor cores: T V D multiply-adds a product.  The forward pass is one product whose epilogue keeps a running
// maximum and sum per row.  The backward pass walks the vocabulary in pieces: the logits of a piece once more, their dz to the
// workspace in bf16, and both gradient products of the piece in one launch, so that the few tiles of the one fill the SMs that
// the other leaves idle.  Four products for a training step where storing the logits would take three.
//
// Left-out rows (target outside the vocabulary) cost nothing and are never read: the kept rows are numbered on the device, all
// kernels walk those, and h is copied together only where some are left out.
//
// bf16 operands go to the tensor cores as they are; dz is rounded to bf16 where the gradients are bf16 and their sums have many
// terms (its rounding is as large as theirs and independent between terms), and split in bf16 planes otherwise: two, or three
// (24 bits) where the gradients are fp32.  fp32 operands are split in three planes too, and a product of
// them is the six plane products that reach 2^-24 of the result, the small ones first.  The tensor cores truncate the
// accumulator at every step, so long sums are cut in segments that the epilogue adds up in registers: however long a sum, the
// truncations take no more of it than those of one segment take of that.
#include "packed.cuh"
#include "sm100_pair.cuh"
#include "vocabloss.cuh"

namespace chela {
namespace {

using namespace sm100;

constexpr int kTile = 256;              // rows and columns of a tile: 128 rows of A and 128 columns of B in each CTA's memory
constexpr int kOperand = 128 * 128, kStageBytes = 2 * kOperand;
constexpr int kEpilogueWarps = 8, kThreads = 64 + 32 * kEpilogueWarps;
constexpr int kBox = 32 * 128, kStagingWarp = 2 * kBox;   // two boxes of 32 rows x 128 bytes: one is filled while the other is stored
// K blocks of 64 (four truncated steps of up to 2^-23 each) that the tensor cores add up at most.  fp32 logits and gradients: 2^-19
// of a plane product's segment.  bf16 operands' logits, and bf16 gradients of dz in planes: 2^-17, the same for any D (uncut, the
// logits of 8192 positive products were 3.0e-5 too small, of 524288 3.3e-3; 7e-7 now.  4096 x 50000 x 2048: 558 -> 576 us, with
// gradients 2311 -> 2368).  bf16 gradients of dz in one plane: 2^-13, a sixteenth of half a step of dz and of the result (uncut, 65536
// products of a slice 3.9e-4 too small, 8e-5 now; no difference in time).
constexpr int kSegment = 4, kLongSegment = 16, kWholeSegment = 256;
enum What { kStats, kSlopes, kGrads };

// The ring of operands, and what the epilogue stages; kStats stages nothing and has the room for two stages more (48 tokens
// against 50000 x 1024, bound by the weights that are on their way: the call 34.7 us with five, 33.7 with seven).
template <bool kStaging>
struct Layout {
    static constexpr int stages = kStaging ? 5 : 7, staging = stages * kStageBytes, bar = staging + (kStaging ? kEpilogueWarps * kStagingWarp : 0);
    static constexpr int tmem = bar + 8 * (2 * stages + 4), abort = tmem + 8, bytes = abort + 8;
    static_assert(bytes <= 232448, "shared memory per CTA");
};
static_assert(kBox % 1024 == 0 && kStageBytes % 1024 == 0, "swizzled boxes start on 1024 bytes");

constexpr size_t kHead = 256;           // workspace header: word 0 the asynchronous status, word 1 the number of kept rows
constexpr float kLn2 = 0.6931471805599453f;

// Planes of A and B of the partial products of one product, small ones first, two bits each.
struct Terms {
    int n;
    uint32_t a, b;
};
constexpr Terms kTerms1 = {1, 0, 0};
constexpr Terms kTerms2A = {2, 1 | 0 << 2, 0};                                                                 // A in planes, two of them
constexpr Terms kTerms3B = {3, 0 | 1 << 2 | 0 << 4, 1 | 0 << 2 | 0 << 4};                                      // both, two of them
constexpr Terms kTerms3 = {3, 2 | 1 << 2 | 0 << 4, 0};                                                        // A in planes
constexpr Terms kTerms6 = {6, 2 | 0 << 2 | 1 << 4 | 1 << 6 | 0 << 8 | 0 << 10, 0 | 2 << 2 | 1 << 4 | 0 << 6 | 1 << 8 | 0 << 10};   // both

struct Product {
    CUtensorMap h, hk, w, dz, dz_out, dh_out, dw_out;
    Terms terms;
    int *head;
    const int *target;              // [Tpad] of kept rows, -1 behind them
    const float4 *coef;             // [Tpad] {lse log2 e, factor of the softmax, factor of the target, target}
    float *zt;                      // [Tpad] target's product with h
    float2 *part;                   // [2 * chunks][Tpad] running maximum (log2 e) and sum of a chunk's column halves
    const void *dw_in;
    const int *row_of;              // [Tpad] tokens of the kept rows
    void *d_h;
    const float *dh_before;         // d_h's sum over the pieces before, where dh_last
    int T, Tpad, V, D, v0, vc, w_row, per_chunk, first_part, sh, sv, planes;
    int h_in_planes, dh_add, dh_last, grad_bf16, dw_sliced, segment;
    float c2;                       // scale log2 e
    WaitCtl wc;
};

// One tile of the product that a launch computes.
struct Tile {
    int m0, n0, kb0, kb1, a_boxes, b_boxes;   // boxes of 64 rows of A and columns of B that exist; the others are not loaded
    bool dw;       // d_w's product (A is dz taken by columns)
    int slice;
};

__device__ __forceinline__ int row_tiles(int n) { return (n + kTile - 1) / kTile; }
__device__ __forceinline__ int piece_boxes(const Product &p) { return (min(p.vc, p.V - p.v0) + 63) / 64; }

__device__ __forceinline__ int units_of(const Product &p, int what, int n)
{
    const int mt = row_tiles(n), boxes = piece_boxes(p), nt = (boxes + 3) / 4, nd = (p.D + kTile - 1) / kTile;
    if (what == kStats) return mt * ((boxes + p.per_chunk - 1) / p.per_chunk);
    if (what == kSlopes) return mt * nt;
    return nd * (nt * p.sv + mt * p.sh);
}

// kStats: a unit is a chunk of per_chunk boxes of 64 columns of one row tile, four boxes a tile.  Neighbouring units share their
// columns: the weights of a chunk are read by all row tiles about the same time.
__device__ __forceinline__ Tile tile_of(const Product &p, int what, int n, int u, int j)
{
    Tile t{};
    const int mt = row_tiles(n), nd = (p.D + kTile - 1) / kTile;
    if (what != kGrads) {
        const int at = u / mt;
        t.m0 = u % mt * kTile;
        t.kb1 = (p.D + 63) / 64;
        const int per = what == kSlopes ? 4 : p.per_chunk, box = at * per + 4 * j;
        t.n0 = box * 64;
        t.a_boxes = min(4, (n - t.m0 + 63) / 64);
        t.b_boxes = min(4, min((at + 1) * per, piece_boxes(p)) - box);
        return t;
    }
    // d_w's tiles first: with many tokens they are the longer ones
    const int ndw = (piece_boxes(p) + 3) / 4 * nd * p.sv;
    t.dw = u < ndw;
    const int v = t.dw ? u : u - ndw, tile = v / nd;
    const int slices = t.dw ? p.sv : p.sh, kbs = t.dw ? (n + 63) / 64 : piece_boxes(p);
    t.n0 = (v - tile * nd) * kTile;
    t.m0 = tile / slices * kTile;
    t.slice = tile % slices;
    t.kb1 = kbs;
    if (slices > 1) {
        t.kb0 = (int)((long long)kbs * t.slice / slices);
        t.kb1 = (int)((long long)kbs * (t.slice + 1) / slices);
    }
    t.a_boxes = min(4, t.dw ? piece_boxes(p) - t.m0 / 64 : (n - t.m0 + 63) / 64);
    t.b_boxes = min(4, (p.D - t.n0 + 63) / 64);
    return t;
}
__device__ __forceinline__ int tiles_in_unit(const Product &p, int what, int n, int u)
{
    if (what != kStats) return 1;
    const int at = u / row_tiles(n);
    return (min((at + 1) * p.per_chunk, piece_boxes(p)) - at * p.per_chunk + 3) / 4;
}

// Columns of a tile that a CTA's half of B has: the product is as wide as the boxes that exist, and each CTA brings half of it.
__device__ __forceinline__ int b_half(const Tile &t) { return 32 * t.b_boxes; }

// Half an operand tile: 128 rows of M or N by 64 of K as two boxes of 64 x 64 (or fewer, the rest left as it is).
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap *map, uint32_t bar, bool mn_major, int mn, int kb, int plane, int boxes)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (i >= boxes) break;
        const int at = mn + 64 * i;
        tma_load_3d_pair(dst + i * 8192, map, bar, mn_major ? at : kb * 64, mn_major ? kb * 64 : at, plane);
    }
}

// Two CTAs a tile of 256 x 256, persistent.  Warp 0: TMA producer of its CTA's halves; warp 1 of the even CTA: issuer;
// warps 2-9: epilogue, each 32 rows x 128 columns.  Accumulators double-buffered in TMEM (2 x 256 columns).
template <int kWhat, bool kSegments>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ Product p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    using Smem = Layout<kWhat != kStats>;
    constexpr int kStages = Smem::stages;
    const uint32_t sbase = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t bar_full = sbase + Smem::bar, bar_empty = bar_full + 8 * kStages, bar_tfull = bar_empty + 8 * kStages, bar_tempty = bar_tfull + 16;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + Smem::tmem);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + Smem::abort);
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar_tfull + 8 * b, 1);
            mbar_init(bar_tempty + 8 * b, 2 * kEpilogueWarps);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc_pair(sbase + Smem::tmem, 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    griddep_launch_dependents();
    griddep_wait();   // up to here the kernel before this one may still run
    const int n = min(max(p.head[1], 0), p.T);
    const int units = units_of(p, kWhat, n);
    // h as given when no row is left out, else the kept rows' copy
    const CUtensorMap *map_h = (n == p.T && !p.h_in_planes) ? &p.h : &p.hk;
    bool ok = true;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0) {
            int it = 0;
            for (int u = pair; ok && u < units; u += pairs) {
                const int tiles = tiles_in_unit(p, kWhat, n, u);
                for (int j = 0; ok && j < tiles; ++j) {
                    const Tile t = tile_of(p, kWhat, n, u, j);
                    const bool a_mn = kWhat == kGrads && t.dw, b_mn = kWhat == kGrads;
                    const CUtensorMap *map_a = kWhat == kGrads ? &p.dz : map_h, *map_b = kWhat == kGrads && t.dw ? map_h : &p.w;
                    const Terms terms = p.terms;
                    // weights: rows of the vocabulary are B's columns for logits and its K for d_h
                    const int b_row = kWhat != kGrads ? p.w_row : 0, b_kb = kWhat == kGrads && !t.dw ? p.w_row / 64 : 0;
                    const int seg = kSegments ? p.segment : t.kb1 - t.kb0;
                    for (int kb = t.kb0; ok && kb < t.kb1; kb += seg)
                        for (int i = 0; ok && i < (kSegments ? terms.n : 1); ++i)
                            for (int k = kb; k < min(kb + seg, t.kb1); ++k, ++it) {
                                const int s = it % kStages;
                                ok = mbar_wait(bar_empty + 8 * s, ((it / kStages) & 1) ^ 1, abort_flag, p.wc.limit);
                                if (!ok) break;
                                const uint32_t bar = bar_full + 8 * s, dst = sbase + s * kStageBytes, to = map_to_rank(bar, 0);
                                if (rank == 0) mbar_expect_tx(bar, (t.a_boxes + 2 * ((t.b_boxes + 1) / 2)) * 8192);
                                load_operand(dst, map_a, to, a_mn, t.m0 + (int)rank * 128, k, kSegments ? terms.a >> 2 * i & 3 : 0, t.a_boxes - 2 * (int)rank);
                                load_operand(dst + kOperand, map_b, to, b_mn, t.n0 + b_row + (int)rank * b_half(t), k + b_kb, kSegments ? terms.b >> 2 * i & 3 : 0, (t.b_boxes + 1) / 2);
                            }
                }
            }
            if (!ok) {
                *abort_flag = 1;
                atomicExch(p.head, (int)CHELA_ERR_TIMEOUT);
                // loads in flight land in shared memory: wait for them as far as this CTA can (bounded)
                if (rank == 0)
                    for (int c = it > kStages ? it - kStages : 0; c < it; ++c) mbar_wait(bar_full + 8 * (c % kStages), (c / kStages) & 1, nullptr, p.wc.limit);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (lane == 0 && rank == 0) {
            int it = 0, gs = 0;
            for (int u = pair; ok && u < units; u += pairs) {
                const int tiles = tiles_in_unit(p, kWhat, n, u);
                for (int j = 0; ok && j < tiles; ++j) {
                    const Tile t = tile_of(p, kWhat, n, u, j);
                    const bool a_mn = kWhat == kGrads && t.dw;
                    constexpr bool b_mn = kWhat == kGrads;
                    const int nterms = kSegments ? p.terms.n : 1;
                    const uint32_t idesc = make_idesc(kTile, 64 * t.b_boxes, a_mn, b_mn);
                    // K step of 16: 32 bytes along a K-major row, 16 rows of an MN-major tile (two atoms of 64 columns)
                    const uint32_t a_step = a_mn ? 128 : 2, b_step = b_mn ? 128 : 2;
                    const int seg = kSegments ? p.segment : t.kb1 - t.kb0;
                    for (int kb = t.kb0; ok && kb < t.kb1; kb += seg, ++gs) {
                        const int buf = gs & 1;
                        ok = mbar_wait(bar_tempty + 8 * buf, ((gs >> 1) & 1) ^ 1, abort_flag, p.wc.limit);
                        if (!ok) break;
                        tc_fence_after();
                        const int steps = (min(kb + seg, t.kb1) - kb) * nterms;
                        for (int k = 0; k < steps; ++k, ++it) {
                            const int s = it % kStages;
                            ok = mbar_wait(bar_full + 8 * s, (it / kStages) & 1, abort_flag, p.wc.limit);
                            if (!ok) break;
                            tc_fence_after();
                            const uint32_t st = sbase + s * kStageBytes;
                            const uint32_t a = a_mn ? desc_lo(st, 8192) : desc_lo(st), b = b_mn ? desc_lo(st + kOperand, 8192) : desc_lo(st + kOperand);
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                umma_bf16_pair(tmem + buf * kTile, a + a_step * q, b + b_step * q, idesc, (k > 0 || q > 0) ? 1u : 0u);
                            umma_commit_pair(bar_empty + 8 * s);
                        }
                        if (ok) umma_commit_pair(bar_tfull + 8 * buf);
                    }
                }
            }
            if (!ok) {
                *abort_flag = 1;
                atomicExch(p.head, (int)CHELA_ERR_TIMEOUT);
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue
        // TMEM lanes are a warp's by its number modulo 4; of the two warps of a lane quarter each takes half the columns
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const int row = (int)rank * 128 + quarter * 32 + lane, row0 = (int)rank * 128 + quarter * 32;
        const uint32_t t_at = tmem + ((uint32_t)(quarter * 32) << 16) + half * 128;
        uint8_t *stg = smem + Smem::staging + (warp - 2) * kStagingWarp;
        const uint32_t stg_u32 = sbase + Smem::staging + (warp - 2) * kStagingWarp;
        const uint32_t leader_tempty = map_to_rank(bar_tempty, 0);
        int gs = 0, boxes = 0;
        for (int u = pair; ok && u < units; u += pairs) {
            const int tiles = tiles_in_unit(p, kWhat, n, u);
            float run_m = -INFINITY, run_s = 0.f;
            for (int j = 0; ok && j < tiles; ++j) {
                const Tile t = tile_of(p, kWhat, n, u, j);
                const int seg = kSegments ? p.segment : max(t.kb1 - t.kb0, 1);
                // what the row brings along, asked for before the wait for its products
                int target = -1;
                float4 cf = make_float4(0.f, 0.f, 0.f, 0.f);
                if (kWhat == kStats) target = p.target[t.m0 + row];
                if (kWhat == kSlopes) cf = p.coef[t.m0 + row];
                float z[128];
                if (kWhat == kGrads && t.kb0 == t.kb1) {   // an empty slice
#pragma unroll
                    for (int c = 0; c < 128; ++c) z[c] = 0.f;
                }
                for (int kb = t.kb0; kb < t.kb1; kb += seg, ++gs) {
                    const int buf = gs & 1;
                    ok = __all_sync(0xffffffffu, mbar_wait(bar_tfull + 8 * buf, (gs >> 1) & 1, abort_flag, p.wc.limit));
                    if (!ok) break;
                    tc_fence_after();
                    if (!kSegments || kb == t.kb0) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) tmem_ld32(t_at + buf * kTile + 32 * c, *reinterpret_cast<float(*)[32]>(&z[32 * c]));
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            float more[32];
                            tmem_ld32(t_at + buf * kTile + 32 * c, more);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 32; ++e) z[32 * c + e] += more[e];
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    // (test hook: the first hand-back of CTA 0 left out, so that the issuer's wait for it runs out)
                    if (lane == 0 && !(p.wc.skip_arrival && blockIdx.x == 0 && gs == 0 && warp == 2)) mbar_arrive_cluster(leader_tempty + 8 * buf);
                }
                if (!ok) break;
                if (kWhat != kGrads && row0 >= 64 * t.a_boxes) continue;   // rows of no token, not even loaded
                const int c0 = t.n0 + half * 128;   // first column of this thread's 128, in the piece
                if (kWhat == kStats) {
                    int y = target - p.v0 - c0;
                    if (y + c0 >= t.n0 + 64 * t.b_boxes) y = -1;   // a later chunk's
                    const int end = min(t.n0 + 64 * t.b_boxes, p.V - p.v0);
                    if (c0 + 128 > end) {
#pragma unroll
                        for (int c = 0; c < 128; ++c)
                            if (c0 + c >= end) z[c] = -INFINITY;
                    }
                    float m4[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
                    for (int c = 4; c < 128; ++c) m4[c & 3] = fmaxf(m4[c & 3], z[c]);
                    const float m = fmaxf(run_m, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * p.c2);
                    const float shift = m == -INFINITY ? 0.f : m;
                    float s4[4] = {run_s * rescale(run_m, m), 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < 128; ++c) s4[c & 3] += ex2(fmaf(z[c], p.c2, -shift));
                    run_s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
                    run_m = m;
                    if (__any_sync(0xffffffffu, y >= 0 && y < 128)) {
                        float zy = 0.f;
#pragma unroll
                        for (int c = 0; c < 128; ++c) zy = c == y ? z[c] : zy;
                        if (y >= 0 && y < 128) p.zt[t.m0 + row] = zy;
                    }
                } else if (kWhat == kSlopes) {
                    const int word = __float_as_int(cf.w), y = word - p.v0 - c0;
                    const bool here = __any_sync(0xffffffffu, y >= 0 && y < 128);
#pragma unroll
                    for (int c = 0; c < 128; ++c) z[c] = cf.y * ex2(fmaf(z[c], p.c2, -cf.x));
                    if (here) {
#pragma unroll
                        for (int c = 0; c < 128; ++c) z[c] = c == y ? z[c] - cf.z : z[c];
                    }
                    // rows behind the last token: zero whatever the weights hold (an infinite one times their h of zero is none)
                    if (word < 0 || c0 + 128 > p.V - p.v0) {
#pragma unroll
                        for (int c = 0; c < 128; ++c)
                            if (word < 0 || c0 + c >= p.V - p.v0) z[c] = 0.f;
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        for (int plane = 0;;) {
                            // (every box is a bulk group, stored or not, so that the last but one has left this buffer)
                            const uint32_t buf = (boxes++ & 1) * kBox;
                            if (lane == 0) bulk_wait_read1();
                            __syncwarp();
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float *x = &z[64 * c + 8 * e];
                                *reinterpret_cast<uint4 *>(stg + buf + sw128(lane, e)) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
                            }
                            fence_proxy_async();
                            __syncwarp();
                            if (lane == 0) {
                                if (c0 + 64 * c < p.vc) tma_store_3d(&p.dz_out, stg_u32 + buf, c0 + 64 * c, t.m0 + row0, plane);
                                bulk_commit();
                            }
                            if (++plane == p.planes) break;
#pragma unroll
                            for (int e = 0; e < 64; ++e) z[64 * c + e] -= __bfloat162float(__float2bfloat16_rn(z[64 * c + e]));   // what is left for the next plane
                        }
                } else {
                    // a final gradient, of its type, or a sum in fp32 that goes on
                    const bool final = t.dw ? !p.dw_sliced : p.dh_last, wide = final && p.grad_bf16;   // boxes of 64 bf16 or 32 fp32 columns
                    const int out_row = t.dw && !p.dw_sliced ? p.v0 + t.m0 + row : t.m0 + row;
                    const float *before32 = t.dw ? (const float *)p.dw_in : p.dh_before;
                    if (final && before32 && out_row < (t.dw ? p.V : p.Tpad)) {
                        const size_t at = (size_t)out_row * p.D;
                        const bool half_width = t.dw && p.grad_bf16;
#pragma unroll
                        for (int c = 0; c < 128; c += 4)
                            if (c0 + c < p.D) {
                                const float4 o = half_width ? load4(reinterpret_cast<const __nv_bfloat16 *>(p.dw_in) + at + c0 + c) : load4(before32 + at + c0 + c);
                                z[c] += o.x, z[c + 1] += o.y, z[c + 2] += o.z, z[c + 3] += o.w;
                            }
                    }
                    const int first = out_row - lane, rows = t.dw ? (p.dw_sliced ? p.vc : p.V) : n;
                    const int token = !t.dw && final && t.m0 + row < n ? p.row_of[t.m0 + row] : -1;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (wide && (c & 1)) continue;
                        const uint32_t buf = (boxes++ & 1) * kBox;
                        if (lane == 0) bulk_wait_read1();
                        __syncwarp();
                        if (wide) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                uint32_t v[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) v[i] = pack_bf16(z[(32 * c + 8 * e + 2 * i) & 127], z[(32 * c + 8 * e + 2 * i + 1) & 127]);
                                *reinterpret_cast<uint4 *>(stg + buf + sw128(lane, e)) = make_uint4(v[0], v[1], v[2], v[3]);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                *reinterpret_cast<float4 *>(stg + buf + sw128(lane, e)) = make_float4(z[32 * c + 4 * e], z[32 * c + 4 * e + 1], z[32 * c + 4 * e + 2], z[32 * c + 4 * e + 3]);
                        }
                        if (!t.dw && final) {
                            // rows go to where their tokens are: eight lanes a row of 128 bytes
                            __syncwarp();
                            const int es = wide ? 2 : 4, col = c0 + 32 * c + (lane & 7) * (16 / es);
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int r = e * 4 + (lane >> 3), to = __shfl_sync(0xffffffffu, token, r);
                                const uint4 v = *reinterpret_cast<const uint4 *>(stg + buf + sw128(r, lane & 7));
                                if (to >= 0 && col < p.D) *reinterpret_cast<uint4 *>(reinterpret_cast<uint8_t *>(p.d_h) + ((size_t)to * p.D + col) * es) = v;
                            }
                            __syncwarp();
                            if (lane == 0) bulk_commit();
                            continue;
                        }
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            if (c0 + 32 * c < p.D && first < rows) {
                                if (t.dw) tma_store_3d(&p.dw_out, stg_u32 + buf, c0 + 32 * c, first, p.dw_sliced ? t.slice : 0);
                                else if (p.dh_add) tma_add_3d(&p.dh_out, stg_u32 + buf, c0 + 32 * c, first, t.slice);
                                else tma_store_3d(&p.dh_out, stg_u32 + buf, c0 + 32 * c, first, t.slice);
                            }
                            bulk_commit();
                        }
                    }
                }
            }
            if (ok && kWhat == kStats) {
                const int chunk = p.first_part + u / row_tiles(n), m0 = u % row_tiles(n) * kTile;
                p.part[(size_t)(2 * chunk + half) * p.Tpad + m0 + row] = make_float2(run_m, run_s);
            }
        }
        if (!ok && lane == 0) {
            *abort_flag = 1;
            atomicExch(p.head, (int)CHELA_ERR_TIMEOUT);
        }
        if (lane == 0) bulk_wait0();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();   // the other CTA's arrivals, loads and products that touch this CTA's memory are behind it
    if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

// ---------------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void split3(float x, __nv_bfloat16 (&o)[3])
{
    o[0] = __float2bfloat16_rn(x);
    const float r = x - __bfloat162float(o[0]);
    o[1] = __float2bfloat16_rn(r);
    o[2] = __float2bfloat16_rn(r - __bfloat162float(o[1]));
}
// Eight elements of a row: bf16 as they are, fp32 in three planes `plane` elements apart.
struct Eight16 {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16 *src) { u = *reinterpret_cast<const uint4 *>(src); }
    __device__ __forceinline__ void store(__nv_bfloat16 *dst, size_t) const { *reinterpret_cast<uint4 *>(dst) = u; }
};
struct Eight32 {
    float4 a, b;
    __device__ __forceinline__ void load(const float *src) { a = load4(src), b = load4(src + 4); }
    __device__ __forceinline__ void store(__nv_bfloat16 *dst, size_t plane) const
    {
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        __align__(16) __nv_bfloat16 o[3][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            __nv_bfloat16 t[3];
            split3(x[e], t);
            o[0][e] = t[0], o[1][e] = t[1], o[2][e] = t[2];
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<uint4 *>(dst + i * plane) = *reinterpret_cast<const uint4 *>(o[i]);
    }
};
__device__ __forceinline__ Eight16 eight(const __nv_bfloat16 *) { return Eight16(); }
__device__ __forceinline__ Eight32 eight(const float *) { return Eight32(); }

// A row by a warp, four vectors a lane at once.
template <typename TH>
__device__ __forceinline__ void copy_row(const TH *src, __nv_bfloat16 *dst, size_t plane, int D, int lane)
{
    for (int c = lane * 8; c < D; c += 1024) {
        decltype(eight(src)) x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + 256 * k < D) x[k].load(src + c + 256 * k);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + 256 * k < D) x[k].store(dst + c + 256 * k, plane);
    }
}

struct Rows {
    const void *targets, *h;
    long long h_stride;
    int T, Tpad, V, D, per_cta, planes;
    int *head, *row_of, *pos_of, *target;    // pos_of, target (forward): nullable
    void *d_h;                               // backward without slices: zero for rows that are left out
    int d_h_bytes;                           // of a row
    float4 *coef;                            // backward
    const float *lse, *d_loss, *d_lse;
    float scale;
    float *loss_out, *lse_out;               // forward
    __nv_bfloat16 *hk;
};

constexpr int kRowsThreads = 512, kRowsWarps = kRowsThreads / 32;
// Numbers the kept rows in the order of the tokens, lays out what the products' epilogues read of them, and copies the kept
// rows of h together where some row is left out or h is split in planes.  Every CTA counts the kept rows before its own by
// itself: the targets are few bytes, and a second launch costs more.
template <typename Idx, typename TH>
__global__ void __launch_bounds__(kRowsThreads) rows_kernel(const Rows r)
{
    __shared__ int s_sum[2][kRowsWarps], s_pos[kRowsThreads], s_warp[kRowsWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Idx *targets = reinterpret_cast<const Idx *>(r.targets);
    const TH *h = reinterpret_cast<const TH *>(r.h);
    const long long begin = (long long)blockIdx.x * r.per_cta, end = min(begin + r.per_cta, (long long)r.T);
    int before = 0, total = 0;
    griddep_launch_dependents();
    const auto count = [&](long long t, Idx y) {
        const int kept = y >= 0 && y < (Idx)r.V;
        total += kept;
        before += kept && t < begin;
    };
    // 16 bytes at a time between the ends that are not aligned to them
    constexpr int kVec = 16 / sizeof(Idx);
    const long long head = min((long long)r.T, (long long)((16 - ((uintptr_t)targets & 15)) % 16 / sizeof(Idx))), vecs = (r.T - head) / kVec;
#pragma unroll 4
    for (long long i = tid; i < vecs; i += kRowsThreads) {
        const uint4 u = *reinterpret_cast<const uint4 *>(targets + head + i * kVec);
        const Idx *y = reinterpret_cast<const Idx *>(&u);
#pragma unroll
        for (int e = 0; e < kVec; ++e) count(head + i * kVec + e, y[e]);
    }
    if (tid < head) count(tid, targets[tid]);
    for (long long t = head + vecs * kVec + tid; t < r.T; t += kRowsThreads) count(t, targets[t]);
    for (int o = 16; o; o >>= 1) {
        before += __shfl_xor_sync(0xffffffffu, before, o);
        total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    if (lane == 0) s_sum[0][warp] = before, s_sum[1][warp] = total;
    __syncthreads();
    int base = 0, n = 0;
    for (int w = 0; w < kRowsWarps; ++w) base += s_sum[0][w], n += s_sum[1][w];
    const bool copy = n < r.T || r.planes > 1;
    const size_t plane = (size_t)r.Tpad * r.D;
    if (blockIdx.x == 0 && tid == 0) r.head[0] = 0, r.head[1] = n;
    for (long long t0 = begin; t0 < end; t0 += kRowsThreads) {
        const long long t = t0 + tid;
        const Idx y = t < end ? targets[t] : (Idx)-1;
        const bool kept = y >= 0 && y < (Idx)r.V;
        const unsigned votes = __ballot_sync(0xffffffffu, kept);
        if (lane == 0) s_warp[warp] = __popc(votes);
        __syncthreads();
        int pos = base + __popc(votes & ((1u << lane) - 1u));
        for (int w = 0; w < kRowsWarps; ++w) {
            if (w < warp) pos += s_warp[w];
            base += s_warp[w];
        }
        s_pos[tid] = kept ? pos : -1;
        if (t < end) {
            if (r.pos_of) r.pos_of[t] = kept ? pos : -1;
            if (kept) {
                r.row_of[pos] = (int)t;
                if (r.target) r.target[pos] = (int)y;
                if (r.coef) {
                    const float g = r.d_loss ? r.d_loss[t] : 0.f;
                    r.coef[pos] = make_float4(r.lse[t] * kLog2e, r.scale * (g + (r.d_lse ? r.d_lse[t] : 0.f)), r.scale * g, __int_as_float((int)y));
                }
            } else {
                if (r.loss_out) r.loss_out[t] = 0.f;
                if (r.lse_out) r.lse_out[t] = 0.f;
            }
        }
        __syncthreads();
        if (copy || r.d_h)
            for (int i = warp; i < kRowsThreads && t0 + i < end; i += kRowsWarps) {
                const int at = s_pos[i];
                if (at < 0) {
                    if (r.d_h)
                        for (int c = lane * 16; c < r.d_h_bytes; c += 512) *reinterpret_cast<uint4 *>(reinterpret_cast<uint8_t *>(r.d_h) + (size_t)(t0 + i) * r.d_h_bytes + c) = make_uint4(0u, 0u, 0u, 0u);
                    continue;
                }
                if (!copy) continue;
                copy_row(h + (size_t)(t0 + i) * r.h_stride, r.hk + (size_t)at * r.D, plane, r.D, lane);
            }
        __syncthreads();
    }
    // behind the last kept row: no targets to the end of its tile, zeros of h to the end of its 64 (d_w's sums read so many)
    // (counted in 64 bits: a CTA's place behind a number of tokens near 2^31 is past it)
    for (long long i = n + (long long)blockIdx.x * kRowsThreads + tid; i < min(r.Tpad, (n + kTile - 1) / kTile * kTile); i += gridDim.x * kRowsThreads) {
        if (r.target) r.target[i] = -1;
        if (r.coef) r.coef[i] = make_float4(0.f, 0.f, 0.f, __int_as_float(-1));
    }
    if (copy)
        for (long long i = n + (long long)blockIdx.x * kRowsWarps + warp; i < (n + 63) / 64 * 64; i += gridDim.x * kRowsWarps)
            for (int pl = 0; pl < r.planes; ++pl)
                for (int c = lane * 8; c < r.D; c += 256) *reinterpret_cast<uint4 *>(r.hk + pl * plane + (size_t)i * r.D + c) = make_uint4(0u, 0u, 0u, 0u);
}

// Rows v0 ... v0 + vc of fp32 weights as three bf16 planes [3][vc][D], zero past V.
__global__ void __launch_bounds__(256) planes_kernel(const float *w, long long w_stride, __nv_bfloat16 *out, int v0, int vc, int V, int D)
{
    griddep_launch_dependents();
    griddep_wait();
    const long long per_row = D / 8, items = per_row * vc;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < items; i += gridDim.x * 256LL) {
        const int v = (int)(i / per_row), c = (int)(i % per_row) * 8;
        __nv_bfloat16 *dst = out + (size_t)v * D + c;
        if (v0 + v < V) {
            Eight32 x;
            x.load(w + (size_t)(v0 + v) * w_stride + c);
            x.store(dst, (size_t)vc * D);
        } else
            for (int pl = 0; pl < 3; ++pl) *reinterpret_cast<uint4 *>(dst + (size_t)pl * vc * D) = make_uint4(0u, 0u, 0u, 0u);
    }
}

// lse = (m + log2 s) ln 2 over a row's parts; the loss from the differences to the largest logit, so that it keeps its digits
// where the target has nearly all the weight.
// A CTA's 256 threads are `groups` threads a row, next to one another rows of one part.
__global__ void __launch_bounds__(256) join_kernel(const int *head, const int *row_of, const float *zt, const float2 *part, int parts, int T, int Tpad, int groups, float c2, float *loss, float *lse)
{
    __shared__ float2 s_part[256];
    const int rows = 256 / groups, lane = threadIdx.x % rows, group = threadIdx.x / rows;
    const long long i = (long long)blockIdx.x * rows + lane;
    griddep_wait();
    const int n = min(max(head[1], 0), T);
    if ((long long)blockIdx.x * rows >= n) return;
    float m = -INFINITY, s = 0.f;
    if (i < n)
#pragma unroll 4
        for (int q = group; q < parts; q += groups) {
            const float2 v = part[(size_t)q * Tpad + i];
            const float mm = fmaxf(m, v.x);
            s = s * rescale(m, mm) + v.y * rescale(v.x, mm), m = mm;
        }
    s_part[threadIdx.x] = make_float2(m, s);
    __syncthreads();
    if (group == 0 && i < n) {
        float mm = m;
        for (int g = 1; g < groups; ++g) mm = fmaxf(mm, s_part[g * rows + lane].x);
        float sum = 0.f;
        for (int g = 0; g < groups; ++g) {
            const float2 v = s_part[g * rows + lane];
            sum += v.y * rescale(v.x, mm);
        }
        const int t = row_of[i];
        const float log_s = log1pf(sum - 1.f);   // the largest term is 1
        lse[t] = fmaf(mm, kLn2, log_s);
        // (the product with c2 unrounded, as in the exponents: where the target has the largest logit, what rounding took from
        // the maximum is in log_s and cancels)
        loss[t] = fmaf(fmaf(-zt[i], c2, mm), kLn2, log_s);
    }
}

__device__ __forceinline__ void add4(float4 &a, const float4 b) { a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w; }

// d_h: the slices of a kept row added up in their order and laid where the row came from; zero for rows that were left out.
template <typename TO>
__global__ void __launch_bounds__(256) spread_kernel(const int *pos_of, const float *dh, int slices, int T, int Tpad, int D, TO *d_h)
{
    griddep_wait();
    const long long per_row = D / 4, items = per_row * T;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < items; i += gridDim.x * 256LL) {
        const long long t = i / per_row;
        const int c = (int)(i % per_row) * 4, at = pos_of[t];
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at >= 0)
            for (int s = 0; s < slices; ++s) add4(v, load4(dh + ((size_t)s * Tpad + at) * D + c));
        store4(d_h + t * D + c, v);
    }
}

// d_w's rows v0 ... : its slices added up in their order, on top of dw_in.
template <typename TO>
__global__ void __launch_bounds__(256) add_slices_kernel(const float *part, int slices, int vc, int rows, int D, const TO *dw_in, TO *d_w)
{
    griddep_wait();
    const long long items = (long long)rows * D / 4, slice = (long long)vc * D;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < items; i += gridDim.x * 256LL) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < slices; ++s) add4(v, load4(part + s * slice + 4 * i));
        if (dw_in) add4(v, load4(dw_in + 4 * i));
        store4(d_w + 4 * i, v);
    }
}

// ---------------------------------------------------------------------------------------------------------------------

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// How a call is cut, from its sizes alone, and where its parts lie in the workspace.
struct Plan {
    int pairs, Tpad, vc, pieces, per_chunk, chunks, sh, sv, planes_in, planes_dz;   // per_chunk: boxes of 64 columns
    size_t row_of, pos_of, target, coef, zt, part, hk, wk, dz, dhp, dwp, bytes;
};

constexpr size_t kPieceBytes = (size_t)512 << 20;    // dz (or the weights' planes) of one piece of the vocabulary
constexpr size_t kSliceBytes = (size_t)256 << 20;    // the gradients' slices

// Time of the gradient launch in K blocks: pairs take the units in turn, d_w's before d_h's, and a round lasts as long as its
// longest unit, its K blocks and about eight for the epilogue.
long long grad_rounds(long long ndw, long long kdw, long long ndh, long long kdh, int pairs)
{
    const long long mixed = ndw % pairs ? pairs - ndw % pairs : 0;   // units of d_h in d_w's last round
    long long sum = ndw / pairs * (8 + kdw);
    if (mixed) sum += 8 + (kdh > kdw && ndh ? kdh : kdw);
    if (ndh > mixed) sum += (ndh - mixed + pairs - 1) / pairs * (8 + kdh);
    return sum;
}

Plan make_plan(int T, int V, int D, chela_dtype_t in_dtype, chela_dtype_t grad_dtype, bool bwd)
{
    Plan q{};
    q.pairs = current_sm_count() / 2;
    q.Tpad = ceil_div(T, kTile) * kTile;
    q.planes_in = in_dtype == CHELA_F32 ? 3 : 1;
    // bf16 gradients: one plane of dz, but two beside fp32 operands, and for up to 64 tokens and 2^25 weights, where the launches
    // bound the call: sums of few terms keep the whole of dz's rounding (21 tokens: relative error of d_w 0.0028 with one plane,
    // 0.0017 with two; 42 x 197413 x 1328: 253 us for the gradients with one, 411 with two)
    q.planes_dz = grad_dtype == CHELA_F32 ? 3 : q.planes_in > 1 || (T <= 64 && (long long)V * D <= 1LL << 25) ? 2 : 1;
    const int nt = ceil_div(V, kTile), mt = q.Tpad / kTile, nd = ceil_div(D, kTile);
    size_t tile_bytes = 0;   // of the piece-wise buffers, by column tile
    if (bwd) tile_bytes = (size_t)q.Tpad * kTile * 2 * q.planes_dz;
    if (q.planes_in > 1 && tile_bytes < (size_t)3 * kTile * D * 2) tile_bytes = (size_t)3 * kTile * D * 2;
    long long most = tile_bytes ? (long long)(kPieceBytes / tile_bytes) : nt;
    if (most < 1) most = 1;
    q.pieces = ceil_div(nt, most);
    const int tiles = ceil_div(nt, q.pieces);
    q.pieces = ceil_div(nt, tiles);
    q.vc = tiles * kTile;
    size_t at = kHead;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes, 1024);
        return here;
    };
    q.row_of = take((size_t)q.Tpad * 4);
    q.hk = take((size_t)q.planes_in * q.Tpad * D * 2);
    if (q.planes_in > 1) q.wk = take((size_t)3 * q.vc * D * 2);
    if (!bwd) {
        // chunks of which the pairs get about the same number of boxes, each a box's worth of overhead; more than two row tiles
        // are bound by whole tiles of four boxes, fewer by the weights that are read
        const int boxes = ceil_div(q.pieces > 1 ? q.vc : V, 64);
        long long best = -1;
        for (int rounds = 1; rounds <= 64; ++rounds) {
            long long chunks = (long long)rounds * q.pairs / mt;
            if (chunks < 1) continue;
            if (chunks > boxes) chunks = boxes;
            int per = ceil_div(boxes, chunks);
            if (mt > 2) per = ceil_div(per, 4) * 4;
            const long long cost = ceil_div((long long)mt * ceil_div(boxes, per), q.pairs) * (long long)(per + 1);
            if (best < 0 || cost < best) best = cost, q.per_chunk = per;
            if (chunks == boxes) break;
        }
        if (best < 0) q.per_chunk = boxes < 64 ? boxes : 64;   // many row tiles
        q.chunks = ceil_div(boxes, q.per_chunk);
        q.target = take((size_t)q.Tpad * 4);
        q.zt = take((size_t)q.Tpad * 4);
        q.part = take((size_t)2 * q.chunks * q.pieces * q.Tpad * 8);
    } else {
        // slices of the gradients' sums: the cheapest launch by grad_rounds, with as few slices as it takes
        long long best = -1;
        for (int sv = 1; sv == 1 || (sv <= 64 && sv <= T / 64); sv *= 2)
            for (int sh = 1; sh == 1 || (sh <= 64 && sh <= q.vc / 64); sh *= 2) {
                if (sv > 1 && (size_t)sv * q.vc * D * 4 > kSliceBytes) continue;
                if (sh > 1 && (size_t)sh * q.Tpad * D * 4 > kSliceBytes) continue;
                const long long kdw = ceil_div(ceil_div(T, 64), sv), kdh = ceil_div(q.vc / 64, sh);
                long long cost = grad_rounds((long long)tiles * nd * sv, kdw, (long long)mt * nd * sh, kdh, q.pairs);
                // the slices' own traffic, in K blocks of a pair (0.27 us) at 6 TB/s: written, read, and a launch
                if (sv > 1) cost += (long long)sv * q.vc * D / 200000 + 8;
                if (sh > 1) cost += ((long long)sh * q.Tpad * D / 200000 + 8) / q.pieces;
                if (best < 0 || cost < best) best = cost, q.sv = sv, q.sh = sh;
            }
        if (q.sh > 1) q.pos_of = take((size_t)T * 4);
        q.coef = take((size_t)q.Tpad * 16);
        q.dz = take((size_t)q.planes_dz * q.Tpad * q.vc * 2);
        if (q.sh > 1 || q.pieces > 1) q.dhp = take((size_t)q.sh * q.Tpad * D * 4);
        if (q.sv > 1) q.dwp = take((size_t)q.sv * q.vc * D * 4);
    }
    q.bytes = at;
    return q;
}

bool map_3d(CUtensorMap *map, const void *ptr, bool f32, long long cols, long long rows, long long planes, long long row_bytes, long long plane_bytes, int box_cols, int box_rows)
{
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)row_bytes, (cuuint64_t)plane_bytes};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
    return make_map_sw128(map, ptr, f32, 3, dims, strides, box);
}

// Launch as a programmatic dependent of the kernel before it in the stream, which it waits for by griddep_wait.
template <typename... P, typename... A>
chela_status_t launch_after(void (*kernel)(P...), int grid, int threads, int smem, cudaStream_t stream, const A &...args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr, cfg.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
}

// Shared memory for a product.  Before the tensor maps: this runtime call also makes the device's context the thread's, which
// the driver's call that encodes them needs and a new thread does not have yet.
template <int kWhat, bool kSegments>
bool prepare_product()
{
    return cudaFuncSetAttribute(product_kernel<kWhat, kSegments>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<kWhat != kStats>::bytes) == cudaSuccess;
}
template <int kWhat, bool kSegments>
chela_status_t launch_product(const Product &p, int pairs, cudaStream_t stream)
{
    return launch_after(product_kernel<kWhat, kSegments>, 2 * pairs, kThreads, Layout<kWhat != kStats>::bytes, stream, p);
}

chela_status_t launch_rows(Rows &r, chela_dtype_t in_dtype, bool wide_ids, int sms, cudaStream_t stream)
{
    int grid = ceil_div(r.T, 16);   // a row or more a warp
    if (grid > 2 * sms) grid = 2 * sms;
    r.per_cta = ceil_div(r.T, grid);
    if (in_dtype == CHELA_F32) {
        if (wide_ids) rows_kernel<long long, float><<<grid, kRowsThreads, 0, stream>>>(r);
        else rows_kernel<int, float><<<grid, kRowsThreads, 0, stream>>>(r);
    } else {
        if (wide_ids) rows_kernel<long long, __nv_bfloat16><<<grid, kRowsThreads, 0, stream>>>(r);
        else rows_kernel<int, __nv_bfloat16><<<grid, kRowsThreads, 0, stream>>>(r);
    }
    return last_launch_status();
}

// The products' operands that both passes share.
bool set_operands(Product &p, const chela_vocabloss_args_t &a, const Plan &q, uint8_t *ws)
{
    const size_t hk_plane = (size_t)q.Tpad * a.D * 2;
    p.head = reinterpret_cast<int *>(ws);
    p.T = a.T, p.Tpad = q.Tpad, p.V = a.V, p.D = a.D, p.vc = q.vc;
    p.h_in_planes = q.planes_in > 1;
    p.c2 = a.scale * kLog2e;
    p.wc = current_wait_ctl();
    p.per_chunk = q.per_chunk, p.sh = q.sh, p.sv = q.sv, p.planes = q.planes_dz;
    if (!map_3d(&p.hk, ws + q.hk, false, a.D, q.Tpad, q.planes_in, (long long)a.D * 2, (long long)hk_plane, 64, 64)) return false;
    if (q.planes_in > 1) {
        p.h = p.hk;
        return map_3d(&p.w, ws + q.wk, false, a.D, q.vc, 3, (long long)a.D * 2, (long long)q.vc * a.D * 2, 64, 64);
    }
    return map_3d(&p.h, a.h, false, a.D, a.T, 1, a.h_stride * 2, a.h_stride * 2, 64, 64) &&
           map_3d(&p.w, a.w, false, a.D, a.V, 1, a.w_stride * 2, a.w_stride * 2, 64, 64);
}

// Logits whose sums are cut: those of fp32 operands, and of bf16 ones over more columns than one segment takes.
int logit_segment(const Plan &q) { return q.planes_in > 1 ? kSegment : kLongSegment; }
bool logits_cut(const Plan &q, int D) { return q.planes_in > 1 || ceil_div(D, 64) > kLongSegment; }

// The weights of the piece that starts at v0: rows of w's map, or planes of them.
chela_status_t set_piece(Product &p, const chela_vocabloss_args_t &a, const Plan &q, uint8_t *ws, int v0, int sms, cudaStream_t stream)
{
    p.v0 = v0;
    p.w_row = q.planes_in > 1 ? 0 : v0;
    if (q.planes_in > 1) {
        return launch_after(planes_kernel, 4 * sms, 256, 0, stream, (const float *)a.w, a.w_stride, (__nv_bfloat16 *)(ws + q.wk), v0, q.vc, a.V, a.D);
    }
    return CHELA_OK;
}

}  // namespace

size_t vocabloss_workspace_bytes(int T, int V, int D, chela_dtype_t in_dtype)
{
    const size_t few = vocabloss_few_workspace_bytes(T, V, D, in_dtype, false);
    return few ? few : make_plan(T, V, D, in_dtype, CHELA_BF16, false).bytes;
}
size_t vocabloss_bwd_workspace_bytes(int T, int V, int D, chela_dtype_t in_dtype, chela_dtype_t grad_dtype)
{
    const size_t few = vocabloss_few_workspace_bytes(T, V, D, in_dtype, true);
    return few ? few : make_plan(T, V, D, in_dtype, grad_dtype, true).bytes;
}

chela_status_t launch_vocabloss_fwd(const chela_vocabloss_args_t &a, float *loss, float *lse, void *workspace, cudaStream_t stream)
{
    if (vocabloss_few_workspace_bytes(a.T, a.V, a.D, a.in_dtype, false)) return launch_vocabloss_few_fwd(a, loss, lse, workspace, stream);
    const Plan q = make_plan(a.T, a.V, a.D, a.in_dtype, CHELA_BF16, false);
    uint8_t *ws = reinterpret_cast<uint8_t *>(workspace);
    const int sms = 2 * q.pairs;
    const bool cut = logits_cut(q, a.D);
    Product p{};
    if (!(cut ? prepare_product<kStats, true>() : prepare_product<kStats, false>()) || !set_operands(p, a, q, ws)) return CHELA_ERR_CUDA;
    Rows r{};
    r.targets = a.targets, r.h = a.h, r.h_stride = a.h_stride, r.T = a.T, r.Tpad = q.Tpad, r.V = a.V, r.D = a.D, r.planes = q.planes_in;
    r.head = p.head, r.row_of = (int *)(ws + q.row_of), r.target = (int *)(ws + q.target), r.loss_out = loss, r.lse_out = lse, r.hk = (__nv_bfloat16 *)(ws + q.hk);
    chela_status_t st = launch_rows(r, a.in_dtype, a.wide_ids != 0, sms, stream);
    p.target = r.target, p.zt = (float *)(ws + q.zt), p.part = (float2 *)(ws + q.part);
    p.terms = q.planes_in > 1 ? kTerms6 : kTerms1;
    p.segment = logit_segment(q);
    int parts = 0;
    for (int i = 0; st == CHELA_OK && i < q.pieces; ++i) {
        const int v0 = i * q.vc, boxes = ceil_div((a.V - v0 < q.vc ? a.V - v0 : q.vc), 64);
        st = set_piece(p, a, q, ws, v0, sms, stream);
        if (st != CHELA_OK) return st;
        p.first_part = parts;
        parts += ceil_div(boxes, q.per_chunk);
        st = cut ? launch_product<kStats, true>(p, q.pairs, stream) : launch_product<kStats, false>(p, q.pairs, stream);
    }
    if (st != CHELA_OK) return st;
    const int groups = parts <= 2 ? 1 : parts <= 32 ? 8 : 32;   // threads a row, by the parts (two a chunk)
    return launch_after(join_kernel, q.Tpad / (256 / groups), 256, 0, stream, p.head, r.row_of, p.zt, p.part, 2 * parts, a.T, q.Tpad, groups, p.c2, loss, lse);
}

chela_status_t launch_vocabloss_bwd(const chela_vocabloss_args_t &a, const float *lse, const float *d_loss, const float *d_lse, void *d_h, const void *d_w_in, void *d_w,
                                    chela_dtype_t grad_dtype, void *workspace, cudaStream_t stream)
{
    if (vocabloss_few_workspace_bytes(a.T, a.V, a.D, a.in_dtype, true)) return launch_vocabloss_few_bwd(a, lse, d_loss, d_lse, d_h, d_w_in, d_w, grad_dtype, workspace, stream);
    const Plan q = make_plan(a.T, a.V, a.D, a.in_dtype, grad_dtype, true);
    uint8_t *ws = reinterpret_cast<uint8_t *>(workspace);
    const int sms = 2 * q.pairs;
    const bool f32 = grad_dtype == CHELA_F32;
    Product p{};
    const Terms terms = q.planes_in > 1 ? (f32 ? kTerms6 : kTerms3B) : f32 ? kTerms3 : q.planes_dz > 1 ? kTerms2A : kTerms1;   // of the gradients
    // gradients whose sums are cut: those of several terms, and those over more tokens or words than one segment takes
    const bool cut = logits_cut(q, a.D), cut_grads = terms.n > 1 || ceil_div(ceil_div(a.T, 64), q.sv) > kWholeSegment || ceil_div(q.vc / 64, q.sh) > kWholeSegment;
    if (!(cut ? prepare_product<kSlopes, true>() : prepare_product<kSlopes, false>()) || !(cut_grads ? prepare_product<kGrads, true>() : prepare_product<kGrads, false>()) ||
        !set_operands(p, a, q, ws))
        return CHELA_ERR_CUDA;
    const long long dz_row = (long long)q.vc * 2, es = f32 ? 4 : 2;
    const bool sums = q.sh > 1 || q.pieces > 1;   // d_h passes through fp32 sums
    if (!map_3d(&p.dz, ws + q.dz, false, q.vc, q.Tpad, q.planes_dz, dz_row, dz_row * q.Tpad, 64, 64) ||
        !map_3d(&p.dz_out, ws + q.dz, false, q.vc, q.Tpad, q.planes_dz, dz_row, dz_row * q.Tpad, 64, 32) ||
        (sums && !map_3d(&p.dh_out, ws + q.dhp, true, a.D, q.Tpad, q.sh, a.D * 4LL, (long long)q.Tpad * a.D * 4, 32, 32)))
        return CHELA_ERR_CUDA;
    if (q.sv > 1 ? !map_3d(&p.dw_out, ws + q.dwp, true, a.D, q.vc, q.sv, a.D * 4LL, (long long)q.vc * a.D * 4, 32, 32)
                 : !map_3d(&p.dw_out, d_w, f32, a.D, a.V, 1, a.D * es, a.D * es, f32 ? 32 : 64, 32))
        return CHELA_ERR_CUDA;
    Rows r{};
    r.targets = a.targets, r.h = a.h, r.h_stride = a.h_stride, r.T = a.T, r.Tpad = q.Tpad, r.V = a.V, r.D = a.D, r.planes = q.planes_in;
    r.head = p.head, r.row_of = (int *)(ws + q.row_of), r.pos_of = q.sh > 1 ? (int *)(ws + q.pos_of) : nullptr, r.coef = (float4 *)(ws + q.coef), r.hk = (__nv_bfloat16 *)(ws + q.hk);
    r.lse = lse, r.d_loss = d_loss, r.d_lse = d_lse, r.scale = a.scale;
    if (q.sh == 1) r.d_h = d_h, r.d_h_bytes = a.D * (int)es;
    chela_status_t st = launch_rows(r, a.in_dtype, a.wide_ids != 0, sms, stream);
    p.coef = r.coef;
    p.row_of = r.row_of, p.d_h = d_h, p.dw_in = d_w_in, p.grad_bf16 = !f32, p.dw_sliced = q.sv > 1;
    for (int i = 0; st == CHELA_OK && i < q.pieces; ++i) {
        const int v0 = i * q.vc, rows = a.V - v0 < q.vc ? a.V - v0 : q.vc;
        st = set_piece(p, a, q, ws, v0, sms, stream);
        if (st != CHELA_OK) return st;
        p.terms = q.planes_in > 1 ? kTerms6 : kTerms1;
        p.segment = logit_segment(q);
        st = cut ? launch_product<kSlopes, true>(p, q.pairs, stream) : launch_product<kSlopes, false>(p, q.pairs, stream);
        if (st != CHELA_OK) return st;
        p.terms = terms;
        p.segment = f32 ? kSegment : terms.n > 1 ? kLongSegment : kWholeSegment;
        p.dh_add = i > 0;
        p.dh_last = q.sh == 1 && i + 1 == q.pieces;
        p.dh_before = i > 0 ? (const float *)(ws + q.dhp) : nullptr;
        st = cut_grads ? launch_product<kGrads, true>(p, q.pairs, stream) : launch_product<kGrads, false>(p, q.pairs, stream);
        if (st == CHELA_OK && q.sv > 1) {
            const size_t off = (size_t)v0 * a.D;
            const float *part = (const float *)(ws + q.dwp);
            if (f32) st = launch_after(add_slices_kernel<float>, 4 * sms, 256, 0, stream, part, q.sv, q.vc, rows, a.D, d_w_in ? (const float *)d_w_in + off : nullptr, (float *)d_w + off);
            else st = launch_after(add_slices_kernel<__nv_bfloat16>, 4 * sms, 256, 0, stream, part, q.sv, q.vc, rows, a.D, d_w_in ? (const __nv_bfloat16 *)d_w_in + off : nullptr, (__nv_bfloat16 *)d_w + off);
        }
    }
    if (st != CHELA_OK || q.sh == 1) return st;
    const float *dhp = (const float *)(ws + q.dhp);
    if (f32) return launch_after(spread_kernel<float>, 8 * sms, 256, 0, stream, (const int *)(ws + q.pos_of), dhp, q.sh, a.T, q.Tpad, a.D, (float *)d_h);
    return launch_after(spread_kernel<__nv_bfloat16>, 8 * sms, 256, 0, stream, (const int *)(ws + q.pos_of), dhp, q.sh, a.T, q.Tpad, a.D, (__nv_bfloat16 *)d_h);
}

}  // namespace chela
