// Attention of one new token, or of a block of L new positions, of each sequence over a paged key-value cache
// (dare_attn_paged): o = softmax(scale q k^T) v over the keys [0, n) of the sequence, the block's own among them, or over those
// of them that lie within a sliding window or among the first `sinks`.
//
// What bounds it is reading K and V once (4 d Hkv bytes per key against 4 d Hq L flops), so the kernel is organised around that
// stream:
//   * the work is cut by keys, not by sequences: the 64-key tiles of all (sequence, KV head, chunk of query rows) units are one
//     list, and each of the CTAs that the GPU holds at once takes an equal stretch of it.  A single long sequence, a full batch
//     and a ragged one all keep every SM reading until the end.  A unit that lies in several stretches is joined by whichever
//     of its CTAs comes last, in the order of the keys, so that results do not depend on the order of arrival;
//   * the query rows of all Hq / Hkv heads that share a KV head are one tile: a key is read once for them;
//   * a producer warp looks up pages two tiles ahead and streams the tiles through a shared-memory ring with TMA (128-byte
//     swizzle; a lane per page piece; pieces that nobody may see are read at a row behind the pool, which TMA fills with zeros);
//   * consumer warps own 16 query rows and, where few rows share a KV head, a slice of each tile's keys: QK^T and PV on
//     warp-level MMAs (m16n8k16), the online softmax in registers.
// Probabilities are rounded to bf16 for the second product (relative 2^-9, averaged over the keys); maximum, sum, products and
// the joined parts are fp32; the output is rounded once.
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace dare {
namespace {

constexpr float LOG2E_F = 1.4426950408889634f;
constexpr float LN2_F = 0.6931471805599453f;

constexpr int PG_KT = 64;          // keys per tile
constexpr int PG_AHEAD = 2;        // tiles whose pages are looked up before their turn
constexpr int PG_INFOS = 16;       // descriptors of tiles in flight

struct PagedParams {
    int B, L, Hq, Hkv, g, R, chunks;      // R = L * g packed query rows per (sequence, KV head), in `chunks` of NW * 16
    int page_shift, n_pages, max_pages;
    int window, sinks;                    // window 0: all keys
    float scale_log2;
    const __nv_bfloat16* q;
    const int32_t *table, *kv_lens;
    __nv_bfloat16* out;
    float* lse;
    float* part_o;                        // [CTAs][2][NW * 16][D]: a CTA's first and last unit, where others share them
    float* part_ml;                       // [CTAs][2][NW * 16][2]: maximum (log2 domain) and sum
    uint32_t* counters;
    uint32_t* dev_status;
};

enum { TILE_FIRST = 1, TILE_LAST = 2, TILE_END = 4, TILE_MASKED = 8, TILE_NONE = 16 };

// A tile, as the producer hands it to the consumers.
struct TileDesc {
    int flags;                // TILE_*: first / last of its unit in this CTA, last of the CTA, some row must not see some key
    int b, kvh, chunk;
    int key0, n;              // first key, keys of the sequence
    int first_cta, n_parts;   // the CTAs that share the unit
    int first_slot;           // the slot of first_cta's part
};

template <int STAGES>
struct PagedBarriers {
    uint64_t full[STAGES];
    uint64_t empty[STAGES];
    uint64_t merge;
    TileDesc tile[PG_INFOS];
    uint32_t abort_flag;
    uint32_t arrived;
};

template <int D, int NW, int KS>
struct PagedShape {
    static constexpr int STAGE = 2 * PG_KT * D * 2;
    static constexpr int STAGES = D == 128 ? 3 : 6;
    // (when the descriptor of tile i + PG_AHEAD is written, tile i - 1 - STAGES has been consumed)
    static_assert(PG_INFOS >= STAGES + PG_AHEAD + 1, "descriptors");
    static constexpr int ROUNDS = KS > 1 ? 2 : 1;                                     // of the merge
    static constexpr int NBK = D / 8 / KS;                                            // column blocks a warp finishes
    static constexpr int XCH = KS > 1 ? KS * (KS - 1) * NW * NBK / ROUNDS * 512 : 0;  // bytes a round exchanges
    static constexpr int ML = KS * NW * 16 * 8;
    static constexpr int SMEM = STAGES * STAGE + XCH + ML + static_cast<int>(sizeof(PagedBarriers<STAGES>)) + 1024;
};

// The tiles of a sequence of n keys: those of the first positions (window only), then those of the window.
struct SeqTiles {
    int n, w0;                // keys; the first key that the block's first query sees in its window
    int n_sink, win_tile;     // tiles before the window's first one, and that one
    int n_tiles;              // at least 1: an empty sequence has a tile without keys, so that somebody writes its rows
    __device__ __forceinline__ SeqTiles(int n_, const PagedParams& p) : n(n_) {
        w0 = p.window > 0 ? max(0, n - p.L - p.window + 1) : 0;
        win_tile = w0 / PG_KT;
        n_sink = min(win_tile, (min(p.sinks, n) + PG_KT - 1) / PG_KT);
        n_tiles = max(1, n_sink + (n + PG_KT - 1) / PG_KT - win_tile);
    }
    __device__ __forceinline__ int key0(int t) const { return (t < n_sink ? t : win_tile + t - n_sink) * PG_KT; }
};

__device__ __forceinline__ int seq_keys(const PagedParams& p, int b) {
    return max(0, min(p.kv_lens[b], p.max_pages << p.page_shift));
}

template <int D, int NW, int KS>
__global__ void __launch_bounds__((NW * KS + 1) * 32, 2)
attn_paged_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PagedParams p) {
    using S = PagedShape<D, NW, KS>;
    constexpr int STAGES = S::STAGES, STAGE = S::STAGE, NBK = S::NBK;
    constexpr int HALF = PG_KT * 128;            // one 64-column half of a tile: 64 rows x 128 bytes
    constexpr int NHALF = D / 64;
    constexpr int KV_BYTES = PG_KT * D * 2;
    constexpr int NCW = NW * KS, ROWS = NW * 16;
    constexpr int KPW = PG_KT / KS;              // keys per warp per tile

    extern __shared__ uint8_t smem_raw[];
    uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float4* xch = reinterpret_cast<float4*>(tiles + STAGES * STAGE);
    float2* xch_ml = reinterpret_cast<float2*>(tiles + STAGES * STAGE + S::XCH);          // [KS][NW * 16]
    PagedBarriers<STAGES>* bars = reinterpret_cast<PagedBarriers<STAGES>*>(tiles + STAGES * STAGE + S::XCH + S::ML);
    volatile uint32_t* abort_flag = &bars->abort_flag;

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == NCW * 32) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], NCW);
        }
        mbar_init(&bars->merge, NCW);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    __syncthreads();
    pdl_wait();

    if (warp == NCW) {
        // ---------------- producer.  This CTA's stretch of the list of tiles: sequence by sequence, in it KV head by KV head
        // (and chunk by chunk of its query rows).
        const int HC = p.Hkv * p.chunks;
        long long total = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const int b = b0 + lane;
            int nt = 0;
            if (b < p.B) {
                const int raw = p.kv_lens[b];
                if (blockIdx.x == 0 && (raw < 0 || raw > (p.max_pages << p.page_shift))) atomicOr(p.dev_status, DEV_LEN_CLAMPED);
                nt = SeqTiles(seq_keys(p, b), p).n_tiles;
            }
            total += __reduce_add_sync(0xffffffffu, nt);      // (32 x 2^24 tiles fit 32 bits)
        }
        total *= HC;
        const long long ctas = total < gridDim.x ? total : gridDim.x;
        const long long begin = blockIdx.x < ctas ? total * blockIdx.x / ctas : 0;
        const long long end = blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : 0;
        if (begin >= end) {
            if (lane == 0) {
                bars->tile[0].flags = TILE_NONE;
                mbar_arrive(&bars->full[0]);
            }
        } else {
            // the sequence of tile `begin`
            int b = 0, lens = 0;                   // (lane i: keys of sequence (b & ~31) + i)
            long long base = 0;                    // first tile of sequence b
            for (int b0 = 0; b0 < p.B; b0 += 32) {
                lens = b0 + lane < p.B ? seq_keys(p, b0 + lane) : 0;
                const int nt = b0 + lane < p.B ? SeqTiles(lens, p).n_tiles : 0;
                int incl = nt;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const int o = __shfl_up_sync(0xffffffffu, incl, off);
                    if (lane >= off) incl += o;
                }
                const long long after = base + static_cast<long long>(incl) * HC;
                const unsigned beyond = __ballot_sync(0xffffffffu, after > begin);
                if (beyond) {
                    const int i = __ffs(beyond) - 1;
                    b = b0 + i;
                    base += static_cast<long long>(__shfl_sync(0xffffffffu, incl - nt, i)) * HC;
                    break;
                }
                base += static_cast<long long>(__shfl_sync(0xffffffffu, incl, 31)) * HC;
            }
            // a cursor over the tiles, PG_AHEAD in front of the copies
            SeqTiles sq(__shfl_sync(0xffffffffu, lens, b & 31), p);
            int u = static_cast<int>((begin - base) / sq.n_tiles), t = static_cast<int>((begin - base) % sq.n_tiles);
            long long at = begin;

            // this lane's piece of a tile: rows [piece * rows_pp, + rows_pp) of one half of K or V
            const int pieces = PG_KT >> min(p.page_shift, 6), rows_pp = PG_KT / pieces;
            const bool active = lane < pieces * NHALF * 2;
            const int piece = lane % pieces, half = lane / pieces % NHALF, is_v = lane / pieces / NHALF;
            const int pool_rows = (p.n_pages * p.Hkv) << p.page_shift;
            const uint32_t dst0 = is_v * KV_BYTES + half * HALF + piece * rows_pp * 128;
            int rows_q[PG_AHEAD + 1];              // pool rows of this lane's pieces of the next tiles
            int kvh = 0, c0 = 0, n_parts = 0, slot0 = 0;
            auto look_up = [&]() -> int {          // the cursor's tile: its descriptor, this lane's pool row; then the next one
                if (at >= end) return 0;
                if (t == 0 || at == begin) {       // tile x lies in the CTA ceil((x + 1) ctas / total) - 1
                    const long long u0 = base + static_cast<long long>(u) * sq.n_tiles, u1 = u0 + sq.n_tiles;
                    c0 = static_cast<int>(((u0 + 1) * ctas + total - 1) / total) - 1;
                    n_parts = static_cast<int>((u1 * ctas + total - 1) / total) - c0;
                    slot0 = total * c0 / ctas >= u0 ? 0 : 1;
                    kvh = u / p.chunks;
                }
                const int key0 = sq.key0(t);
                if (lane == 0) {
                    TileDesc d;
                    d.flags = (t == 0 || at == begin ? TILE_FIRST : 0) | (t == sq.n_tiles - 1 || at == end - 1 ? TILE_LAST : 0) |
                              (at == end - 1 ? TILE_END : 0);
                    if (key0 + PG_KT > sq.n || (p.window > 0 && key0 < sq.n - p.window && key0 + PG_KT > p.sinks)) d.flags |= TILE_MASKED;
                    d.b = b; d.kvh = kvh; d.chunk = u % p.chunks; d.key0 = key0; d.n = sq.n;
                    d.first_cta = c0; d.n_parts = n_parts; d.first_slot = slot0;
                    bars->tile[(at - begin) % PG_INFOS] = d;
                }
                int row = pool_rows;               // behind the pool: zeros
                const int key = key0 + piece * rows_pp;
                if (active && key < sq.n && (key < p.sinks || key + rows_pp > sq.w0)) {
                    const int page = p.table[static_cast<long long>(b) * p.max_pages + (key >> p.page_shift)];
                    if (page >= 0 && page < p.n_pages) row = ((page * p.Hkv + kvh) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
                    else atomicOr(p.dev_status, DEV_INDEX_OUTSIDE);
                }
                ++at;
                if (++t == sq.n_tiles) {
                    t = 0;
                    if (++u == HC) {
                        u = 0;
                        base += static_cast<long long>(sq.n_tiles) * HC;
                        ++b;
                        if ((b & 31) == 0) lens = b + lane < p.B ? seq_keys(p, b + lane) : 0;
                        if (b < p.B) sq = SeqTiles(__shfl_sync(0xffffffffu, lens, b & 31), p);
                    }
                }
                return row;
            };
#pragma unroll
            for (int i = 0; i < PG_AHEAD; ++i) rows_q[i] = look_up();
            int stage = 0;
            uint32_t phase = 0;
            for (long long i = begin; i < end; ++i) {
                rows_q[PG_AHEAD] = look_up();
                if (!__all_sync(0xffffffffu, mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag))) break;
                if (lane == 0) mbar_arrive_expect_tx(&bars->full[stage], 2 * KV_BYTES);
                __syncwarp();
                if (active) tma_load_2d(tiles + stage * STAGE + dst0, is_v ? &tm_v : &tm_k, &bars->full[stage], half * 64, rows_q[0]);
                __syncwarp();
#pragma unroll
                for (int k = 0; k < PG_AHEAD; ++k) rows_q[k] = rows_q[k + 1];
                if (++stage == STAGES) { stage = 0; phase ^= 1; }
            }
        }
    } else {
        // ---------------- consumers
        const int rg = warp % NW, ks = warp / NW;          // row group, key slice
        const int quad = lane >> 2, tq = lane & 3;
        const int mi = lane >> 3, rin = lane & 7;
        const int koff = ks * KPW;
        const float c = p.scale_log2;
        int stage = 0;
        uint32_t phase = 0, merge_phase = 0, n_tile = 0;
        uint32_t qf[D / 16][4];
        float oacc[D / 8][4];
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        int i0 = 0, i1 = 0, h0 = 0, h1 = 0;                // block positions and heads of this lane's two rows
        bool live0 = false, live1 = false;
        // a barrier among the consumer warps, bounded as all waits are
        auto merge_sync = [&]() -> bool {
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->merge);
            const bool ok = mbar_wait(&bars->merge, merge_phase, abort_flag);
            merge_phase ^= 1;
            return __all_sync(0xffffffffu, ok);
        };
        while (true) {
            if (!__all_sync(0xffffffffu, mbar_wait(&bars->full[stage], phase, abort_flag))) break;
            const TileDesc ti = bars->tile[n_tile % PG_INFOS];
            ++n_tile;
            if (ti.flags & TILE_NONE) break;
            uint8_t* kt = tiles + stage * STAGE;
            uint8_t* vt = kt + KV_BYTES;
            const uint32_t kbase = smem_u32(kt), vbase = smem_u32(vt);
            if (ti.flags & TILE_FIRST) {
                const int rho0 = ti.chunk * ROWS + rg * 16 + quad, rho1 = rho0 + 8;
                live0 = rho0 < p.R;
                live1 = rho1 < p.R;
                i0 = live0 ? rho0 / p.g : 0;
                i1 = live1 ? rho1 / p.g : 0;
                h0 = ti.kvh * p.g + (live0 ? rho0 % p.g : 0);
                h1 = ti.kvh * p.g + (live1 ? rho1 % p.g : 0);
                const uint32_t* q0 = reinterpret_cast<const uint32_t*>(p.q + ((static_cast<size_t>(ti.b) * p.L + i0) * p.Hq + h0) * D);
                const uint32_t* q1 = reinterpret_cast<const uint32_t*>(p.q + ((static_cast<size_t>(ti.b) * p.L + i1) * p.Hq + h1) * D);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    qf[kk][0] = live0 ? q0[kk * 8 + tq] : 0u;
                    qf[kk][1] = live1 ? q1[kk * 8 + tq] : 0u;
                    qf[kk][2] = live0 ? q0[kk * 8 + 4 + tq] : 0u;
                    qf[kk][3] = live1 ? q1[kk * 8 + 4 + tq] : 0u;
                }
#pragma unroll
                for (int n = 0; n < D / 8; ++n) oacc[n][0] = oacc[n][1] = oacc[n][2] = oacc[n][3] = 0.f;
                m0 = m1 = -INFINITY;
                l0 = l1 = 0.f;
            }
            const bool masked = ti.flags & TILE_MASKED;
            if (masked) {
                // V rows that no query may see hold whatever lies there: zero this warp's, so that probability 0 times
                // garbage cannot make a NaN
                const int w0 = p.window > 0 ? ti.n - p.L - p.window + 1 : 0;
                bool wrote = false;
                for (int o = lane; o < KPW * 8 * NHALF; o += 32) {
                    const int row = koff + (o >> 3) % KPW, half = (o >> 3) / KPW, key = ti.key0 + row;
                    if (key >= ti.n || (key >= p.sinks && key < w0)) {
                        *reinterpret_cast<uint4*>(vt + half * HALF + row * 128 + (o & 7) * 16) = make_uint4(0, 0, 0, 0);
                        wrote = true;
                    }
                }
                if (wrote) fence_proxy_async_smem();
                __syncwarp();
            }
            // S = Q K^T for this warp's keys
            float sacc[KPW / 8][4];
#pragma unroll
            for (int nb = 0; nb < KPW / 8; ++nb) sacc[nb][0] = sacc[nb][1] = sacc[nb][2] = sacc[nb][3] = 0.f;
#pragma unroll
            for (int kq = 0; kq < D / 32; ++kq) {
                uint32_t kf[KPW / 8][4];
#pragma unroll
                for (int nb = 0; nb < KPW / 8; ++nb) {
                    const int key = koff + nb * 8 + rin, ch = 4 * kq + mi;
                    ldmatrix_x4(kbase + (ch >> 3) * HALF + key * 128 + (((ch & 7) ^ (key & 7)) << 4), kf[nb][0], kf[nb][1], kf[nb][2], kf[nb][3]);
                }
#pragma unroll
                for (int nb = 0; nb < KPW / 8; ++nb) mma_bf16_16816(sacc[nb], qf[2 * kq], kf[nb][0], kf[nb][1]);
#pragma unroll
                for (int nb = 0; nb < KPW / 8; ++nb) mma_bf16_16816(sacc[nb], qf[2 * kq + 1], kf[nb][2], kf[nb][3]);
            }
            if (masked) {
                // keys [sinks, start of the row's window) and from n on do not count
                const int no_window = p.window > 0 ? 0 : ti.n + p.L;
                const int s0 = ti.n - p.L + i0 - p.window + 1 - no_window, s1 = ti.n - p.L + i1 - p.window + 1 - no_window;
#pragma unroll
                for (int nb = 0; nb < KPW / 8; ++nb) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = ti.key0 + koff + nb * 8 + tq * 2 + (e & 1);
                        if (key >= ti.n || (key >= p.sinks && key < (e < 2 ? s0 : s1))) sacc[nb][e] = -INFINITY;
                    }
                }
            }
            float tmax0 = -INFINITY, tmax1 = -INFINITY;
#pragma unroll
            for (int nb = 0; nb < KPW / 8; ++nb) {
                tmax0 = fmaxf(tmax0, fmaxf(sacc[nb][0], sacc[nb][1]));
                tmax1 = fmaxf(tmax1, fmaxf(sacc[nb][2], sacc[nb][3]));
            }
            tmax0 = fmaxf(tmax0, __shfl_xor_sync(0xffffffffu, tmax0, 1));
            tmax0 = fmaxf(tmax0, __shfl_xor_sync(0xffffffffu, tmax0, 2));
            tmax1 = fmaxf(tmax1, __shfl_xor_sync(0xffffffffu, tmax1, 1));
            tmax1 = fmaxf(tmax1, __shfl_xor_sync(0xffffffffu, tmax1, 2));
            // (a row may have seen nothing yet: its reference is then 0, its weights exp2(-inf) = 0)
            const float mn0 = fmaxf(m0, tmax0), mn1 = fmaxf(m1, tmax1);
            const float r0 = mn0 == -INFINITY ? 0.f : mn0 * c, r1 = mn1 == -INFINITY ? 0.f : mn1 * c;
            const bool moved = __any_sync(0xffffffffu, mn0 != m0 || mn1 != m1);
            float ps0 = 0.f, ps1 = 0.f;
            uint32_t pa[KPW / 16][4];
#pragma unroll
            for (int nb = 0; nb < KPW / 8; ++nb) {
                const float e0 = fast_exp2(fmaf(sacc[nb][0], c, -r0)), e1 = fast_exp2(fmaf(sacc[nb][1], c, -r0));
                const float e2 = fast_exp2(fmaf(sacc[nb][2], c, -r1)), e3 = fast_exp2(fmaf(sacc[nb][3], c, -r1));
                ps0 += e0 + e1;
                ps1 += e2 + e3;
                pa[nb >> 1][(nb & 1) * 2 + 0] = pack_bf16(e0, e1);
                pa[nb >> 1][(nb & 1) * 2 + 1] = pack_bf16(e2, e3);
            }
            if (moved) {
                const float a0 = fast_exp2(fmaf(m0, c, -r0)), a1 = fast_exp2(fmaf(m1, c, -r1));
                m0 = mn0;
                m1 = mn1;
                l0 *= a0;
                l1 *= a1;
#pragma unroll
                for (int n = 0; n < D / 8; ++n) {
                    oacc[n][0] *= a0; oacc[n][1] *= a0;
                    oacc[n][2] *= a1; oacc[n][3] *= a1;
                }
            }
            l0 += ps0;
            l1 += ps1;
            // O += P V
#pragma unroll
            for (int kk = 0; kk < KPW / 16; ++kk) {
                const int key = koff + kk * 16 + (mi & 1) * 8 + rin;
#pragma unroll
                for (int nbp = 0; nbp < D / 16; ++nbp) {
                    const int ch = 2 * nbp + (mi >> 1);
                    uint32_t v0, v1, v2, v3;
                    ldmatrix_x4_trans(vbase + (ch >> 3) * HALF + key * 128 + (((ch & 7) ^ (key & 7)) << 4), v0, v1, v2, v3);
                    mma_bf16_16816(oacc[2 * nbp], pa[kk], v0, v1);
                    mma_bf16_16816(oacc[2 * nbp + 1], pa[kk], v2, v3);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->empty[stage]);
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
            if (!(ti.flags & TILE_LAST)) continue;

            // ---------------- the unit's end in this CTA: merge the key slices; each slice's warp finishes its share of the columns
            float tl0 = l0 + __shfl_xor_sync(0xffffffffu, l0, 1), tl1 = l1 + __shfl_xor_sync(0xffffffffu, l1, 1);
            tl0 += __shfl_xor_sync(0xffffffffu, tl0, 2);
            tl1 += __shfl_xor_sync(0xffffffffu, tl1, 2);
            float tm0 = m0 * c, tm1 = m1 * c;              // log2 domain
            float w0[KS], w1[KS];
            if (KS > 1) {
                if (tq == 0) {
                    xch_ml[ks * ROWS + rg * 16 + quad] = make_float2(tm0, tl0);
                    xch_ml[ks * ROWS + rg * 16 + quad + 8] = make_float2(tm1, tl1);
                }
                if (!merge_sync()) break;
                float2 ml0[KS], ml1[KS];
#pragma unroll
                for (int o = 0; o < KS; ++o) {
                    ml0[o] = xch_ml[o * ROWS + rg * 16 + quad];
                    ml1[o] = xch_ml[o * ROWS + rg * 16 + quad + 8];
                    tm0 = fmaxf(tm0, ml0[o].x);
                    tm1 = fmaxf(tm1, ml1[o].x);
                }
                tl0 = tl1 = 0.f;
#pragma unroll
                for (int o = 0; o < KS; ++o) {
                    w0[o] = tm0 == -INFINITY ? 0.f : fast_exp2(ml0[o].x - tm0);
                    w1[o] = tm1 == -INFINITY ? 0.f : fast_exp2(ml1[o].x - tm1);
                    tl0 += ml0[o].y * w0[o];
                    tl1 += ml1[o].y * w1[o];
                }
                constexpr int NBR = NBK / S::ROUNDS;       // column blocks of a round
                bool ok = true;
#pragma unroll
                for (int r = 0; r < S::ROUNDS; ++r) {
#pragma unroll
                    for (int o = 0; o < KS; ++o) {
                        if (o == ks) continue;
#pragma unroll
                        for (int i = 0; i < NBR; ++i) {
                            const float (&v)[4] = oacc[o * NBK + r * NBR + i];
                            xch[(((o * (KS - 1) + (ks < o ? ks : ks - 1)) * NW + rg) * NBR + i) * 32 + lane] = make_float4(v[0], v[1], v[2], v[3]);
                        }
                    }
                    ok = merge_sync();
                    if (!ok) break;
#pragma unroll
                    for (int o = 0; o < KS; ++o) {
                        if (o != ks) continue;
#pragma unroll
                        for (int i = 0; i < NBR; ++i) {
                            float (&v)[4] = oacc[o * NBK + r * NBR + i];
                            v[0] *= w0[o]; v[1] *= w0[o]; v[2] *= w1[o]; v[3] *= w1[o];
#pragma unroll
                            for (int s = 0; s < KS; ++s) {
                                if (s == o) continue;
                                const float4 x = xch[(((o * (KS - 1) + (s < o ? s : s - 1)) * NW + rg) * NBR + i) * 32 + lane];
                                v[0] += x.x * w0[s]; v[1] += x.y * w0[s];
                                v[2] += x.z * w1[s]; v[3] += x.w * w1[s];
                            }
                        }
                    }
                    ok = merge_sync();
                    if (!ok) break;
                }
                if (!ok) break;
            }
            const bool whole = ti.n_parts == 1;
            const float inv0 = whole ? (tl0 > 0.f ? 1.f / tl0 : tl0 == 0.f ? 0.f : tl0) : 1.f;      // (a NaN sum stays one)
            const float inv1 = whole ? (tl1 > 0.f ? 1.f / tl1 : tl1 == 0.f ? 0.f : tl1) : 1.f;
            const size_t orow0 = (static_cast<size_t>(ti.b) * p.L + i0) * p.Hq + h0, orow1 = (static_cast<size_t>(ti.b) * p.L + i1) * p.Hq + h1;
            const int slot = blockIdx.x * 2 + (static_cast<int>(blockIdx.x) == ti.first_cta ? ti.first_slot : 0);
            float* po = p.part_o + static_cast<size_t>(slot) * ROWS * D;
#pragma unroll
            for (int o = 0; o < KS; ++o) {
                if (o != ks) continue;
#pragma unroll
                for (int i = 0; i < NBK; ++i) {
                    const float (&v)[4] = oacc[o * NBK + i];
                    const int col = (o * NBK + i) * 8 + tq * 2;
                    if (whole) {
                        if (live0) *reinterpret_cast<uint32_t*>(p.out + orow0 * D + col) = pack_bf16(v[0] * inv0, v[1] * inv0);
                        if (live1) *reinterpret_cast<uint32_t*>(p.out + orow1 * D + col) = pack_bf16(v[2] * inv1, v[3] * inv1);
                    } else {
                        if (live0) *reinterpret_cast<float2*>(po + (rg * 16 + quad) * D + col) = make_float2(v[0], v[1]);
                        if (live1) *reinterpret_cast<float2*>(po + (rg * 16 + quad + 8) * D + col) = make_float2(v[2], v[3]);
                    }
                }
            }
            if (ks == 0 && tq == 0) {
                if (whole) {
                    if (p.lse != nullptr) {
                        if (live0) p.lse[(static_cast<size_t>(ti.b) * p.Hq + h0) * p.L + i0] = tm0 == -INFINITY ? -INFINITY : (tm0 + log2f(tl0)) * LN2_F;
                        if (live1) p.lse[(static_cast<size_t>(ti.b) * p.Hq + h1) * p.L + i1] = tm1 == -INFINITY ? -INFINITY : (tm1 + log2f(tl1)) * LN2_F;
                    }
                } else {
                    float2* pm = reinterpret_cast<float2*>(p.part_ml) + static_cast<size_t>(slot) * ROWS + rg * 16 + quad;
                    pm[0] = make_float2(tm0, tl0);
                    pm[8] = make_float2(tm1, tl1);
                }
            }
            if (!whole) {
                // ---------------- the last of the unit's CTAs to come joins the parts, in the order of the keys
                __threadfence();
                if (!merge_sync()) break;
                if (threadIdx.x == 0) {
                    const uint32_t before = atomicAdd(&p.counters[ti.first_cta], 1u);
                    bars->arrived = before;
                    if (before == static_cast<uint32_t>(ti.n_parts) - 1) p.counters[ti.first_cta] = 0;      // for the next launch
                    __threadfence();
                }
                if (!merge_sync()) break;
                if (bars->arrived == static_cast<uint32_t>(ti.n_parts) - 1) {
                    const int rows = min(ROWS, p.R - ti.chunk * ROWS);
                    for (int item = threadIdx.x; item < rows * (D / 4); item += NCW * 32) {
                        const int row = item / (D / 4), c4 = item % (D / 4);
                        const float2* pm = reinterpret_cast<const float2*>(p.part_ml) + row;
                        const float* px = p.part_o + row * D + c4 * 4;
                        float m = -INFINITY, l = 0.f;
                        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (int k = 0; k < ti.n_parts; ++k) {
                            const size_t s = static_cast<size_t>(ti.first_cta + k) * 2 + (k == 0 ? ti.first_slot : 0);
                            const float2 ml = __ldcg(pm + s * ROWS);
                            const float4 x = ld_global_cg_f4(px + s * ROWS * D);
                            const float mn = fmaxf(m, ml.x);
                            const float wa = mn == -INFINITY ? 0.f : fast_exp2(m - mn), wb = mn == -INFINITY ? 0.f : fast_exp2(ml.x - mn);
                            m = mn;
                            l = l * wa + ml.y * wb;
                            acc.x = acc.x * wa + x.x * wb; acc.y = acc.y * wa + x.y * wb;
                            acc.z = acc.z * wa + x.z * wb; acc.w = acc.w * wa + x.w * wb;
                        }
                        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
                        const int rho = ti.chunk * ROWS + row, i = rho / p.g, h = ti.kvh * p.g + rho % p.g;
                        const uint2 packed = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                        *reinterpret_cast<uint2*>(p.out + ((static_cast<size_t>(ti.b) * p.L + i) * p.Hq + h) * D + c4 * 4) = packed;
                        if (p.lse != nullptr && c4 == 0)
                            p.lse[(static_cast<size_t>(ti.b) * p.Hq + h) * p.L + i] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * LN2_F;
                    }
                }
            }
            if (ti.flags & TILE_END) break;
        }
    }
    // (the next kernel is let in late: its CTAs would pile up on the few SMs that have room beside this one's)
    pdl_trigger();
    __syncthreads();
    if (*abort_flag) {
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000LL) {}            // copies in flight land
        if (threadIdx.x == 0) atomicOr(p.dev_status, DEV_WAIT_EXPIRED);
        __syncthreads();
    }
}

// Row groups per CTA, by the packed query rows R of a (sequence, KV head): up to 16 rows four key slices share one, up to 32 two
// share two, more take four row groups per chunk of 64 rows.
int paged_row_groups(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : 4; }

template <int D, int NW, int KS>
int launch_paged(const dare_ctx* ctx, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const PagedParams& p, int ctas, cudaStream_t stream) {
    using S = PagedShape<D, NW, KS>;
    static_assert(2 * (S::SMEM + 1024) <= 228 * 1024, "two CTAs per SM");
    static std::atomic<uint64_t> smem_set{0};
    if (ensure_dynamic_smem(smem_set, attn_paged_kernel<D, NW, KS>, S::SMEM) != DARE_OK) return DARE_ERR_CUDA;
    return launch_kernel(attn_paged_kernel<D, NW, KS>, dim3(ctas), (NW * KS + 1) * 32, S::SMEM, stream, 1, tm_k, tm_v, p);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace dare

extern "C" int dare_attn_paged(dare_ctx* ctx, int B, int L, int Hq, int Hkv, int d, float scale, const void* q, const void* k_pages,
                               const void* v_pages, int n_pages, int page_size, const int32_t* block_table, int max_pages,
                               const int32_t* kv_lens, int window, int sinks, void* out, float* lse, void* stream) {
    using namespace dare;
    if (!ctx || !q || !k_pages || !v_pages || !block_table || !kv_lens || !out) return DARE_ERR_NULL;
    if (int rc = check_current_device(ctx)) return rc;
    if (B < 1 || L < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || (d != 64 && d != 128)) return DARE_ERR_SHAPE;
    if (static_cast<long long>(L) * (Hq / Hkv) > (1 << 20)) return DARE_ERR_SHAPE;
    if (int rc = check_pages(B, max_pages, n_pages, page_size, Hkv)) return rc;
    if (!(scale >= 0.f) || isinf(scale) || window < 0 || sinks < 0) return DARE_ERR_RANGE;
    if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out)) return DARE_ERR_ALIGN;
    PagedParams p = {};
    p.B = B; p.L = L; p.Hq = Hq; p.Hkv = Hkv; p.g = Hq / Hkv; p.R = L * p.g;
    const int nw = paged_row_groups(p.R);
    p.chunks = (p.R + nw * 16 - 1) / (nw * 16);
    p.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
    p.n_pages = n_pages; p.max_pages = max_pages;
    // a window that reaches further than any key is none (and keeps the kernel's sums within 32 bits)
    p.window = window >= (max_pages << p.page_shift) ? 0 : window;
    p.sinks = p.window > 0 ? sinks : 0;
    p.scale_log2 = (scale != 0.f ? scale : 1.0f / sqrtf(static_cast<float>(d))) * LOG2E_F;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.table = block_table; p.kv_lens = kv_lens;
    p.out = static_cast<__nv_bfloat16*>(out); p.lse = lse;
    p.counters = ctx->join_counters; p.dev_status = ctx->dev_status;
    // two CTAs per SM, all resident at once; no more than there can be tiles
    const long long tiles = static_cast<long long>(B) * Hkv * p.chunks * ((static_cast<long long>(max_pages) * page_size + PG_KT - 1) / PG_KT);
    long long ctas = 2LL * ctx->sm_count;
    if (ctas > PAGED_MAX_CTAS) ctas = PAGED_MAX_CTAS;
    if (ctas > tiles) ctas = tiles;
    const size_t part_rows = static_cast<size_t>(ctas) * 2 * nw * 16;
    if (part_rows * (d + 2) * sizeof(float) > ctx->workspace_bytes) return DARE_ERR_WORKSPACE;
    p.part_o = static_cast<float*>(ctx->workspace);
    p.part_ml = p.part_o + part_rows * d;
    CUtensorMap tm_k, tm_v;
    const uint64_t pool_rows = static_cast<uint64_t>(n_pages) * Hkv * page_size;
    const uint32_t box_rows = static_cast<uint32_t>(page_size < PG_KT ? page_size : PG_KT);
    int rc = make_tmap_bf16_2d(ctx, &tm_k, k_pages, pool_rows, d, box_rows, 64);
    if (rc == DARE_OK) rc = make_tmap_bf16_2d(ctx, &tm_v, v_pages, pool_rows, d, box_rows, 64);
    if (rc != DARE_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int n = static_cast<int>(ctas);
    if (d == 128)
        return nw == 1 ? launch_paged<128, 1, 4>(ctx, tm_k, tm_v, p, n, s) : nw == 2 ? launch_paged<128, 2, 2>(ctx, tm_k, tm_v, p, n, s)
                                                                                   : launch_paged<128, 4, 1>(ctx, tm_k, tm_v, p, n, s);
    return nw == 1 ? launch_paged<64, 1, 4>(ctx, tm_k, tm_v, p, n, s) : nw == 2 ? launch_paged<64, 2, 2>(ctx, tm_k, tm_v, p, n, s)
                                                                              : launch_paged<64, 4, 1>(ctx, tm_k, tm_v, p, n, s);
}
