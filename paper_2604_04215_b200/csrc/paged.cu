// Attention of one new token, or of a block of L new positions, of each sequence over a paged key-value cache
// (dare_attn_paged): o = softmax(scale q k^T) v over the keys [0, n) of the sequence, the block's own among them, or over those
// of them that lie within a sliding window or among the first `sinks`.
//
// What bounds it is reading K and V once (4 d Hkv bytes per key against 4 d Hq L flops), so the kernel is organised around that
// stream:
//   * the work is cut by keys, not by sequences: the 64-key tiles of all (sequence, KV head) units are one
//     list, and each of the CTAs that the GPU holds at once takes an equal stretch of it.  A single long sequence, a full batch
//     and a ragged one all keep every SM reading until the end.  A unit that lies in several stretches is joined by whichever
//     of its CTAs comes last, in the order of the keys, so that results do not depend on the order of arrival;
//   * the query rows of all Hq / Hkv heads that share a KV head are one tile of up to 8: a key is read once for them.  (More rows
//     go to the tcgen05 kernel of attn.cu, see launch_attn_paged_tc);
//   * a producer warp reads table entries 32 at a time, ahead of their turn, and streams the tiles through a shared-memory ring with TMA (128-byte
//     swizzle; a lane per page piece; pieces that nobody may see are read at a row behind the pool, which TMA fills with zeros);
//   * four consumer warps own 16 keys of each tile: QK^T and PV on warp-level MMAs (m16n8k16) with the keys and channels as rows and
//     the query rows as columns, the online softmax in registers.
// The weights enter the second product as two bf16 values, rounded value and remainder (relative 2^-17 together): with the first alone
// outputs are 1.3 times as far from 64 bits as their own rounding, and the second costs 0.5 % of the time, most of which is spent waiting
// for memory.  Maximum, sum, products and the joined parts are fp32; the output is rounded once.
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace dare {
namespace {

constexpr float LOG2E_F = 1.4426950408889634f;
constexpr float LN2_F = 0.6931471805599453f;

constexpr int PG_KT = 64;          // keys per tile
constexpr int PG_ROWS = 8;         // packed query rows of a unit, at most
constexpr int PG_WARPS = 4;        // consumers, each with 16 of a tile's keys
// Where there is a CTA for each unit, units are taken whole if the longest has no more tiles than PG_SHARES equal shares of all tiles on all
// places and PG_LONGER more: joining costs a CTA 5 to 7.4 k cycles at its end, a tile 0.9 (few CTAs) to 1.5 k (all of them reading).  us cut
// evenly / whole on 296 places, 28 + 4 heads: 256 units of 64 tiles 89.5 / 81.5, 148 of 47 43.8 / 39.9, 148 of 16 19.9 / 17.3, 72 of 11 11.8 / 10.6;
// 72 of 32 19.8 / 23.3, 4 of 8 6.7 / 8.4, 4 of 125 13.7 / 71.7.
constexpr int PG_SHARES = 2, PG_LONGER = 6;
constexpr float PG_LEAST = 0.4f;   // see Stretches
constexpr int PG_UNITS = 8;        // descriptors of units on their way

struct PagedParams {
    int places;                           // CTAs that the GPU holds at once
    int B, L, Hq, Hkv, g, R;              // R = L * g packed query rows per (sequence, KV head)
    int page_shift, n_pages, max_pages;
    int window, sinks;                    // window 0: all keys
    float scale_log2;
    const __nv_bfloat16* q;
    const int32_t *table, *kv_lens;
    __nv_bfloat16* out;
    float* lse;
    float* part_o;                        // [CTAs][2][PG_ROWS][D]: a CTA's first and last unit, where others share them
    float* part_ml;                       // [CTAs][2][PG_ROWS][2]: maximum (log2 domain) and sum
    uint32_t* counters;
    uint32_t* dev_status;
};

enum { TILE_FIRST = 1, TILE_LAST = 2, TILE_END = 4, TILE_MASKED = 8, TILE_NONE = 16 };

// A tile and a unit, as the producer hands them to the consumers.
struct alignas(16) TileDesc { int flags, key0, unit, unused; };      // TILE_*: first / last of its unit in this CTA, last of the CTA, some
                                                                     // row must not see some key; first key; place of the unit's descriptor
struct alignas(16) UnitDesc {
    int b, kvh, n, parts;      // n: keys of the sequence; parts: CTAs that share the unit
    int first_cta, slot, first_slot, unused;      // the first of them, where this CTA's part goes, where first_cta's does
};

template <int STAGES>
struct PagedBarriers {
    uint64_t full[STAGES];
    uint64_t empty[STAGES];
    uint64_t merge;
    TileDesc tile[STAGES];
    UnitDesc unit[PG_UNITS];
    UnitDesc shared_unit[2];           // units that this CTA shares with others: its first one, its last one
    uint32_t abort_flag;
    uint32_t arrived[2];
    // (when a unit's descriptor is written, the tile STAGES + 1 before its first one has been consumed)
    static_assert(PG_UNITS >= STAGES + 1, "descriptors of units");
};

template <int D>
struct PagedShape {
    static constexpr int STAGE = 2 * PG_KT * D * 2;
    static constexpr int STAGES = D == 128 ? 3 : 6;
    static constexpr int ML = 2 * PG_WARPS * PG_ROWS * 8;                             // [unit's parity][slice][row] maximum and sum
    // Query rows arrive with their unit's first tile, where there is room for them in each of the ring's places; rows are 16 bytes
    // apart from a power of two (ldmatrix without bank conflicts).
    static constexpr int Q_ROW = D * 2 + 16;
    static constexpr int Q_STAGE = PG_ROWS * Q_ROW;
    static constexpr int SMEM = STAGES * (STAGE + Q_STAGE) + ML + static_cast<int>(sizeof(PagedBarriers<STAGES>)) + 1024;
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

// The list of all units' tiles cut into stretches of equal length (to one tile), one per CTA (none where there are fewer tiles).  A tile
// after another costs a CTA about as much as eight parts more cost those who join them: the sum of both is least where a stretch
// has PG_LEAST sqrt(tiles of the longest unit) tiles, so it has that many at least, unless units would have to share CTAs for it
// (us for 1 sequence of 777, 4000, 8000 and 40000 keys, 28 + 4 heads, with 0.4: 7.8, 10.4, 13.3, 24.9; with stretches of one tile and more:
// 7.8, 12.4, 22.0, 27.4; with 0.6: 9.5, 12.8, 13.1, 26.9).
// T numbers the list's tiles (see dare_attn_paged).
template <typename T>
struct Stretches {
    int n;                    // CTAs that have one
    T each, more;             // tiles of each; the first `more` have one tile more
    __device__ __forceinline__ Stretches(T tiles, int units, int longest, int ctas) {
        const int least = max(1, static_cast<int>(PG_LEAST * sqrtf(static_cast<float>(longest))));
        n = static_cast<int>(min(static_cast<T>(ctas), max(static_cast<T>(units), tiles / least)));
        each = tiles / n;
        more = tiles - each * n;
    }
    __device__ __forceinline__ T begin(int cta) const { return min(cta, n) * each + min(static_cast<T>(cta), more); }
    __device__ __forceinline__ int cta_of(T tile) const {
        const T longer = more * (each + 1);
        return static_cast<int>(tile < longer ? tile / (each + 1) : more + (tile - longer) / each);
    }
};

__device__ __forceinline__ int seq_keys(const PagedParams& p, int b) {
    return max(0, min(p.kv_lens[b], p.max_pages << p.page_shift));
}

// What a row of a sequence of n keys is divided by, and its lse.  Key n - 1 is visible to every query, and a row's largest score has
// weight 1: a sum of 0 is that of a sequence without keys, or of a row whose visible scores are all -inf, as with an infinity in the
// query that meets keys of the other sign (0 / 0: NaN, as with a NaN in the query).
__device__ __forceinline__ float inverse_sum(float l, int n) { return l > 0.f ? 1.f / l : n > 0 ? NAN : 0.f; }
__device__ __forceinline__ float log_sum(float m, float l, int n) { return l > 0.f ? (m + log2f(l)) * LN2_F : n > 0 ? NAN : -INFINITY; }

// Adds a unit's parts up, in the order of the keys (the order of arrival does not show).  A thread has four channels of a row,
// two rows at once, and asks for JOIN parts at a time: what this costs is trips to L2, one after the other.
constexpr int JOIN = 8;
template <int D>
__device__ __forceinline__ void join_parts(const PagedParams& p, const UnitDesc& unit) {
    constexpr int THREADS = PG_WARPS * 32;
    const UnitDesc u = unit;
    const int items = p.R * (D / 4);
    const float2* part_ml = reinterpret_cast<const float2*>(p.part_ml);
    const float4* part_o = reinterpret_cast<const float4*>(p.part_o);
    for (int item0 = threadIdx.x; item0 < items; item0 += 2 * THREADS) {
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
        for (int k0 = 0; k0 < u.parts; k0 += JOIN) {
            float2 ml[2][JOIN];
            float4 x[2][JOIN];
#pragma unroll
            for (int k = 0; k < JOIN; ++k) {
                const int part = min(k0 + k, u.parts - 1);           // (beyond the last: the last one, counted 0 times)
                const int slot = (u.first_cta + part) * 2 + (part == 0 ? u.first_slot : 0);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int item = min(item0 + e * THREADS, items - 1), at = slot * PG_ROWS + item / (D / 4);
                    ml[e][k] = __ldcg(part_ml + at);
                    x[e][k] = __ldcg(part_o + static_cast<size_t>(at) * (D / 4) + item % (D / 4));
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float mn = m[e];
#pragma unroll
                for (int k = 0; k < JOIN; ++k) mn = fmaxf(mn, ml[e][k].x);
                const float r = mn == -INFINITY ? 0.f : mn, w = fast_exp2(m[e] - r);
                m[e] = mn;
                l[e] *= w;
                acc[e].x *= w; acc[e].y *= w; acc[e].z *= w; acc[e].w *= w;
#pragma unroll
                for (int k = 0; k < JOIN; ++k) {
                    if (k0 + k >= u.parts) continue;
                    const float wk = fast_exp2(ml[e][k].x - r);
                    l[e] += ml[e][k].y * wk;
                    acc[e].x += x[e][k].x * wk; acc[e].y += x[e][k].y * wk;
                    acc[e].z += x[e][k].z * wk; acc[e].w += x[e][k].w * wk;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int item = item0 + e * THREADS;
            if (item >= items) continue;
            const float inv = inverse_sum(l[e], u.n);
            const int rho = item / (D / 4), c4 = item % (D / 4), i = rho / p.g, h = u.kvh * p.g + rho - i * p.g;
            *reinterpret_cast<uint2*>(p.out + ((static_cast<size_t>(u.b) * p.L + i) * p.Hq + h) * D + c4 * 4) =
                make_uint2(pack_bf16(acc[e].x * inv, acc[e].y * inv), pack_bf16(acc[e].z * inv, acc[e].w * inv));
            if (p.lse != nullptr && c4 == 0)
                p.lse[(static_cast<size_t>(u.b) * p.Hq + h) * p.L + i] = log_sum(m[e], l[e], u.n);
        }
    }
}

// Shared memory of a CTA.
template <int D>
struct PagedSmem {
    using S = PagedShape<D>;
    uint8_t *tiles, *q;                    // [STAGES][STAGE], [STAGES][PG_ROWS][Q_ROW]
    float2* ml;
    PagedBarriers<S::STAGES>* bars;
    __device__ __forceinline__ explicit PagedSmem(uint8_t* raw) {
        tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
        q = tiles + S::STAGES * S::STAGE;
        ml = reinterpret_cast<float2*>(q + S::STAGES * S::Q_STAGE);
        bars = reinterpret_cast<PagedBarriers<S::STAGES>*>(q + S::STAGES * S::Q_STAGE + S::ML);
    }
};

// The producer warp: finds this CTA's stretch of the list of tiles (sequence by sequence, in it KV head by KV head) and sends for
// its tiles.
template <int D, typename T>
__device__ __forceinline__ void produce(const CUtensorMap* tm_k, const CUtensorMap* tm_v, const PagedParams& p, const PagedSmem<D>& sm) {
    using S = PagedShape<D>;
    constexpr int STAGES = S::STAGES, KV_BYTES = PG_KT * D * 2;
    PagedBarriers<STAGES>* bars = sm.bars;
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int lane = threadIdx.x & 31;
    T total = 0;
    int longest = 0, lens = 0;                     // (lens, lane i: keys of sequence (b & ~31) + i)
    for (int g0 = 0; g0 < p.B; g0 += 4 * 32) {     // (four loads at a time)
        int raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = g0 + i * 32 + lane < p.B ? p.kv_lens[g0 + i * 32 + lane] : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (g0 + i * 32 >= p.B) break;
            const int keys = max(0, min(raw[i], p.max_pages << p.page_shift));
            if (blockIdx.x == 0 && raw[i] != keys) atomicOr(p.dev_status, DEV_LEN_CLAMPED);
            const int nt = g0 + i * 32 + lane < p.B ? SeqTiles(keys, p).n_tiles : 0;
            total += __reduce_add_sync(0xffffffffu, nt);
            longest = max(longest, __reduce_max_sync(0xffffffffu, nt));
            if (g0 + i == 0) lens = keys;
        }
    }
    const Stretches<T> st(total * p.Hkv, p.B * p.Hkv, longest, gridDim.x);
    T begin = st.begin(blockIdx.x), end = st.begin(blockIdx.x + 1);
    const bool unit_each = p.B * p.Hkv <= static_cast<int>(gridDim.x) && longest - PG_LONGER <= PG_SHARES * total * p.Hkv / p.places;
    if (unit_each) begin = 0, end = static_cast<int>(blockIdx.x) < p.B * p.Hkv;
    if (begin >= end) {
        if (lane == 0) {
            bars->tile[0].flags = TILE_NONE;
            mbar_arrive(&bars->full[0]);
        }
        return;
    }
    int b = 0;                                     // the sequence of tile `begin`; its first tile
    T base = 0;
    if (unit_each) {
        b = static_cast<int>(blockIdx.x) / p.Hkv;
        if (b >= 32) lens = (b & ~31) + lane < p.B ? seq_keys(p, (b & ~31) + lane) : 0;
    } else if (p.B > 1) {
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            if (b0 > 0) lens = b0 + lane < p.B ? seq_keys(p, b0 + lane) : 0;
            const int nt = b0 + lane < p.B ? SeqTiles(lens, p).n_tiles : 0;
            int incl = nt;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, incl, off);
                if (lane >= off) incl += o;
            }
            const unsigned beyond = __ballot_sync(0xffffffffu, base + static_cast<T>(incl) * p.Hkv > begin);
            if (beyond) {
                const int i = __ffs(beyond) - 1;
                b = b0 + i;
                base += static_cast<T>(__shfl_sync(0xffffffffu, incl - nt, i)) * p.Hkv;
                break;
            }
            base += static_cast<T>(__shfl_sync(0xffffffffu, incl, 31)) * p.Hkv;
        }
    }
    // this lane's piece of a tile: rows [piece * rows_pp, + rows_pp) of K or V.  (Both halves of the columns in one copy: a copy takes
    // its lane some 85 cycles to send, and the 16 of a tile of 16-key pages, 2 KB each, were what its CTA waited for.)
    const int pp_shift = min(p.page_shift, 6), pieces_shift = 6 - pp_shift, rows_pp = 1 << pp_shift;      // (64 keys a tile)
    const bool active = lane < 2 << pieces_shift;
    const int piece = lane & ((1 << pieces_shift) - 1), is_v = lane >> pieces_shift;
    const int pool_rows = (p.n_pages * p.Hkv) << p.page_shift;
    const uint32_t dst0 = is_v * KV_BYTES + piece * rows_pp * D * 2;
    const CUtensorMap* tm = is_v ? tm_v : tm_k;
    int n = __shfl_sync(0xffffffffu, lens, b & 31), kvh, t;
    {
        const int nt = SeqTiles(n, p).n_tiles;
        kvh = unit_each ? static_cast<int>(blockIdx.x) - b * p.Hkv : static_cast<int>((begin - base) / nt);
        t = unit_each ? 0 : static_cast<int>(begin - base - static_cast<T>(kvh) * nt);
        if (unit_each) end = nt;
    }
    int stage = 0, unit = 0;
    uint32_t phase = 0;
    for (T at = begin; at < end;) {                // unit by unit
        const SeqTiles sq(n, p);
        const int count = static_cast<int>(min(static_cast<T>(sq.n_tiles - t), end - at));
        // Table entries 32 pieces at a time, a lane each, the next 32 while these are on their way: the pool row that a piece is read from
        // (that behind the pool, zeros, for one that nobody may see and for one without a page).
        const int32_t* table = p.table + static_cast<long long>(b) * p.max_pages;
        auto key_of = [&](int i) { return sq.key0(t + (i >> pieces_shift)) + ((i & ((1 << pieces_shift) - 1)) << pp_shift); };
        auto ask = [&](int i, int& page) -> bool {
            const int key = key_of(i);
            const bool visible = (i >> pieces_shift) < count && key < n && (key < p.sinks || key + rows_pp > sq.w0);
            if (visible) page = table[key >> p.page_shift];
            return visible;
        };
        auto row_of = [&](int i, int page, bool visible) -> int {
            if (!visible) return pool_rows;
            if (page < 0 || page >= p.n_pages) {
                atomicOr(p.dev_status, DEV_INDEX_OUTSIDE);
                return pool_rows;
            }
            return ((page * p.Hkv + kvh) << p.page_shift) + (key_of(i) & ((1 << p.page_shift) - 1));
        };
        int page = 0, page_next = 0;
        bool seen = ask(lane, page), seen_next = ask(lane + 32, page_next);
        const bool whole = t == 0 && count == sq.n_tiles;
        const T unit0 = base + static_cast<T>(kvh) * sq.n_tiles;
        int rows = row_of(lane, page, seen);
        bool ok = true;
        for (int i = 0; i < count; ++i) {
            const int at_piece = i << pieces_shift;
            if (i > 0 && (at_piece & 31) == 0) {
                rows = row_of(at_piece + lane, page_next, seen_next);
                seen_next = ask(at_piece + 32 + lane, page_next);
            }
            const int row = __shfl_sync(0xffffffffu, rows, (at_piece + piece) & 31);
            ok = __all_sync(0xffffffffu, mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag));
            if (!ok) break;
            uint64_t* full = &bars->full[stage];
            // (the bytes may arrive before they are expected: the phase ends with the arrival below)
            if (active) tma_load_3d(sm.tiles + stage * S::STAGE + dst0, tm, full, 0, row, 0);
            if (i == 0) {
                if (lane < p.R) {
                    const int pos = p.L == 1 ? 0 : lane / p.g, h = kvh * p.g + lane - pos * p.g;
                    bulk_load(sm.q + stage * S::Q_STAGE + lane * S::Q_ROW, p.q + ((static_cast<size_t>(b) * p.L + pos) * p.Hq + h) * D, D * 2, full);
                }
                const int c0 = whole ? static_cast<int>(blockIdx.x) : st.cta_of(unit0);
                const int parts = whole ? 1 : st.cta_of(unit0 + sq.n_tiles - 1) - c0 + 1, first_slot = whole || st.begin(c0) == unit0 ? 0 : 1;
                if (lane == 0)
                    bars->unit[unit] = {b, kvh, n, parts, c0, 2 * static_cast<int>(blockIdx.x) + (static_cast<int>(blockIdx.x) == c0 ? first_slot : 0), first_slot, 0};
            }
            if (lane == 0) {
                const int key0 = sq.key0(t + i);
                int flags = (i == 0 ? TILE_FIRST : 0) | (i == count - 1 ? TILE_LAST : 0) | (at + i == end - 1 ? TILE_END : 0);
                if (key0 + PG_KT > n || (p.window > 0 && key0 < n - p.window && key0 + PG_KT > p.sinks)) flags |= TILE_MASKED;
                bars->tile[stage] = {flags, key0, unit, 0};
                mbar_arrive_expect_tx(full, 2 * KV_BYTES + (i == 0 ? p.R * D * 2 : 0));
            }
            __syncwarp();
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        at += count;
        t = 0;
        unit = (unit + 1) % PG_UNITS;
        if (++kvh == p.Hkv) {
            kvh = 0;
            base += static_cast<T>(sq.n_tiles) * p.Hkv;
            ++b;
            if ((b & 31) == 0) lens = b + lane < p.B ? seq_keys(p, b + lane) : 0;
            n = __shfl_sync(0xffffffffu, lens, b & 31);
        }
    }
}

// What a window hides: key j is hidden from query i (at position n - L + i) if sinks <= j < start + i.
__device__ __forceinline__ int window_start(const PagedParams& p, int n) { return p.window > 0 ? n - p.L - p.window + 1 : -p.L; }

// A tile's pieces of pages lie one after the other, in each the halves of its columns.  Where the 16 keys from koff on begin in the first
// half (they are in one piece); the second half is a piece's rows further.
__device__ __forceinline__ int slice_at(const PagedParams& p, int koff, int row_bytes) {
    const int pp = min(p.page_shift, 6);
    return (koff >> pp << pp) * row_bytes + (koff & ((1 << pp) - 1)) * 128;
}
__device__ __forceinline__ int half_stride(const PagedParams& p) { return 128 << min(p.page_shift, 6); }

// V rows that no query may see hold whatever lies there: zeroes those among the 16 keys from key0 on, which `at` holds, so that
// probability 0 times garbage cannot make a NaN.
template <int NHALF>
__device__ __forceinline__ void clear_unseen(const PagedParams& p, int key0, int n, uint8_t* at) {
    const int lane = threadIdx.x & 31, start = window_start(p, n);
    bool wrote = false;
    for (int o = lane; o < 16 * 8 * NHALF; o += 32) {
        const int row = (o >> 3) % 16, half = (o >> 3) / 16, key = key0 + row;
        if (key >= n || (key >= p.sinks && key < start)) {
            *reinterpret_cast<uint4*>(at + half * half_stride(p) + row * 128 + (o & 7) * 16) = make_uint4(0, 0, 0, 0);
            wrote = true;
        }
    }
    if (wrote) fence_proxy_async_smem();
    __syncwarp();
}

// A consumer warp's state for up to 8 query rows: the products are turned round, S^T = K Q^T and O^T = V^T P^T, so that the rows
// are the MMA's 8 columns and half as many MMAs and registers are needed as with rows for its 16.  Lane (quad, tq): keys (and
// channels) quad and quad + 8 of each 16, query rows 2 tq and 2 tq + 1.  A warp owns 16 keys of each tile.
template <int D>
struct FewRows {
    static constexpr int NHALF = D / 64, KV_BYTES = PG_KT * D * 2, KS = PG_WARPS, KPW = PG_KT / KS;
    static_assert(KPW == 16 && PG_ROWS == 8, "a slice is one MMA's keys, the rows are its columns");
    uint32_t qb[D / 16][2];
    float o[D / 16][4];
    float m[2], l[2];
    int row_i[2];              // block positions of this lane's two rows
    int half;                  // bytes from one half of the columns to the other

    __device__ __forceinline__ explicit FewRows(const PagedParams& p) {
        const int tq = threadIdx.x & 3;
        row_i[0] = p.L == 1 ? 0 : 2 * tq / p.g;
        row_i[1] = p.L == 1 ? 0 : (2 * tq + 1) / p.g;
        half = half_stride(p);
    }
    __device__ __forceinline__ void first(const uint8_t* q_rows) {
        const int lane = threadIdx.x & 31;
        const uint32_t qa = smem_u32(q_rows) + (lane & 7) * PagedShape<D>::Q_ROW + (lane >> 3) * 16;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) ldmatrix_x4(qa + j * 64, qb[2 * j][0], qb[2 * j][1], qb[2 * j + 1][0], qb[2 * j + 1][1]);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
    }
    __device__ __forceinline__ void tile(const PagedParams& p, bool masked, int key0, int n, uint8_t* kt, int ks) {
        const int lane = threadIdx.x & 31, quad = lane >> 2, koff = ks * KPW;
        uint8_t* slice = kt + slice_at(p, koff, D * 2);
        const uint32_t kbase = smem_u32(slice), vbase = kbase + KV_BYTES;
        if (masked) clear_unseen<NHALF>(p, key0 + koff, n, slice + KV_BYTES);
        float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};          // (two chains of products)
        {
            const int key = lane & 15;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const int ch = 2 * (kk & 3) + (lane >> 4);
                uint32_t a[4];
                ldmatrix_x4(kbase + (kk >> 2) * half + key * 128 + ((ch ^ (key & 7)) << 4), a[0], a[1], a[2], a[3]);
                if (kk & 1) mma_bf16_16816(s2, a, qb[kk][0], qb[kk][1]);
                else mma_bf16_16816(s, a, qb[kk][0], qb[kk][1]);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += s2[e];
        if (masked) {
            const int start = window_start(p, n);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = key0 + koff + quad + (e >> 1) * 8;
                if (key >= n || (key >= p.sinks && key < start + row_i[e & 1])) s[e] = -INFINITY;
            }
        }
        const float c = p.scale_log2;
        float mn[2], r[2];
        bool same = true;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float t = fmaxf(s[e], s[e + 2]);
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
            mn[e] = fmaxf(m[e], t);
            r[e] = mn[e] == -INFINITY ? 0.f : __fmul_rn(mn[e], c);      // (a row may have seen nothing yet: weights exp2(-inf) = 0)
            same = same && mn[e] == m[e];
        }
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = fast_exp2(fmaf(s[e], c, -r[e & 1]));
        if (__any_sync(0xffffffffu, !same)) {
            // From the old reference, rounded as it was when weights were taken against it, to the new one: exactly 1 for a row that stays.
            // (The unrounded product is up to 2^-24 of itself away from it, each time that another row's maximum moves; a row
            // without a maximum has nothing to carry over.)
            const float f0 = m[0] == -INFINITY ? 0.f : fast_exp2(__fmul_rn(m[0], c) - r[0]);
            const float f1 = m[1] == -INFINITY ? 0.f : fast_exp2(__fmul_rn(m[1], c) - r[1]);
            m[0] = mn[0];
            m[1] = mn[1];
            l[0] *= f0;
            l[1] *= f1;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                o[i][0] *= f0; o[i][1] *= f1;
                o[i][2] *= f0; o[i][3] *= f1;
            }
        }
        l[0] += w[0] + w[2];
        l[1] += w[1] + w[3];
        // weights for the second product: their bf16 values and, in a product of its own, what the rounding left
        const uint32_t h0 = pack_bf16(w[0], w[1]), h1 = pack_bf16(w[2], w[3]);
        const uint32_t p0 = movmatrix_trans(h0), p1 = movmatrix_trans(h1);
        const uint32_t e0 = movmatrix_trans(pack_bf16(w[0] - __uint_as_float(h0 << 16), w[1] - __uint_as_float(h0 & 0xffff0000u)));
        const uint32_t e1 = movmatrix_trans(pack_bf16(w[2] - __uint_as_float(h1 << 16), w[3] - __uint_as_float(h1 & 0xffff0000u)));
        const int key = (lane & 7) + (lane >> 4) * 8;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const int ch = 2 * (i & 3) + ((lane >> 3) & 1);
            uint32_t a[4];
            ldmatrix_x4_trans(vbase + (i >> 2) * half + key * 128 + ((ch ^ (key & 7)) << 4), a[0], a[1], a[2], a[3]);
            mma_bf16_16816(o[i], a, p0, p1);
            mma_bf16_16816(o[i], a, e0, e1);
        }
    }
    // The unit's end in this CTA: every warp lays its part down over its own keys of the tile that it has just read, then the rows are
    // added up four channels at a time.  `kt` is the tile's place, ml [KS][8].
    template <typename Sync>
    __device__ __forceinline__ bool finish(const PagedParams& p, const UnitDesc& u, uint8_t* kt, float2* ml, int ks, Sync&& sync) {
        // place of row q of slice s: pieces of 16 keys of one half of K or V are 2 KB; 8 / (2 NHALF) rows in each
        constexpr int PER = 8 / (2 * NHALF);
        auto at = [&](int s, int q) {
            const int k = q / PER;
            return reinterpret_cast<float*>(kt + slice_at(p, s * KPW, D * 2) + (k / NHALF) * KV_BYTES + (k % NHALF) * half + (q % PER) * (D * 4 + 16) +
                                            k * (PER * 16));
        };
        const int lane = threadIdx.x & 31, quad = lane >> 2, tq = lane & 3;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 4);
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 8);
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 16);
            if (quad == 0) ml[ks * 8 + 2 * tq + e] = make_float2(__fmul_rn(m[e], p.scale_log2), l[e]);
            float* x = at(ks, 2 * tq + e);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                x[i * 16 + quad] = o[i][e];
                x[i * 16 + quad + 8] = o[i][e + 2];
            }
        }
        if (!sync()) return false;
        const bool whole = u.parts == 1;
        for (int item = threadIdx.x; item < p.R * (D / 4); item += KS * 32) {
            const int q = item / (D / 4), c4 = item % (D / 4);
            float2 part[KS];
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                part[s] = ml[s * 8 + q];
                top = fmaxf(top, part[s].x);
            }
            const float ref = top == -INFINITY ? 0.f : top;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const float w = fast_exp2(part[s].x - ref);
                const float4 x = *reinterpret_cast<const float4*>(at(s, q) + c4 * 4);
                sum += part[s].y * w;
                acc.x += x.x * w; acc.y += x.y * w; acc.z += x.z * w; acc.w += x.w * w;
            }
            if (whole) {
                const float inv = inverse_sum(sum, u.n);
                const int i = p.L == 1 ? 0 : q / p.g, h = u.kvh * p.g + q - i * p.g;
                *reinterpret_cast<uint2*>(p.out + ((static_cast<size_t>(u.b) * p.L + i) * p.Hq + h) * D + c4 * 4) =
                    make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                if (p.lse != nullptr && c4 == 0) p.lse[(static_cast<size_t>(u.b) * p.Hq + h) * p.L + i] = log_sum(top, sum, u.n);
            } else {
                *reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(u.slot) * PG_ROWS + q) * D + c4 * 4) = acc;
                if (c4 == 0) reinterpret_cast<float2*>(p.part_ml)[u.slot * PG_ROWS + q] = make_float2(top, sum);
            }
        }
        return true;
    }
};

template <int D, typename T>
__global__ void __launch_bounds__((PG_WARPS + 1) * 32, 2)
attn_paged_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PagedParams p) {
    using S = PagedShape<D>;
    constexpr int STAGES = S::STAGES, NCW = PG_WARPS;
    extern __shared__ uint8_t smem_raw[];
    const PagedSmem<D> sm(smem_raw);
    PagedBarriers<STAGES>* bars = sm.bars;
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
    // rows that are no query's: zero, once
    for (int o = threadIdx.x; o < STAGES * S::Q_STAGE / 16; o += (NCW + 1) * 32) reinterpret_cast<uint4*>(sm.q)[o] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    __syncthreads();
    pdl_wait();

    if (warp == NCW) {
        produce<D, T>(&tm_k, &tm_v, p, sm);
    } else {
        FewRows<D> c(p);
        UnitDesc u = {};
        int stage = 0, n_shared = 0;
        uint32_t phase = 0, merge_phase = 0, parity = 0;
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
            const TileDesc ti = bars->tile[stage];
            if (ti.flags & TILE_NONE) break;
            uint8_t* kt = sm.tiles + stage * S::STAGE;
            if (ti.flags & TILE_FIRST) {
                u = bars->unit[ti.unit];
                c.first(sm.q + stage * S::Q_STAGE);
            }
            c.tile(p, ti.flags & TILE_MASKED, ti.key0, u.n, kt, warp);
            const int this_stage = stage;
            if (++stage == STAGES) { stage = 0; phase ^= 1; }
            if (!(ti.flags & TILE_LAST)) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->empty[this_stage]);
                continue;
            }
            if (!c.finish(p, u, kt, sm.ml + parity * NCW * PG_ROWS, warp, merge_sync)) break;
            parity ^= 1;                                       // (a warp may be a unit ahead of one that still reads its sums)
            fence_proxy_async_smem();                          // (the next copy into this place is the producer's)
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->empty[this_stage]);
            // a shared unit's part has been written; who comes last is found out once, when this CTA has read all its tiles
            if (u.parts > 1) {
                const int k = (ti.flags & TILE_END) ? 1 : 0;   // (in between units are whole)
                if (threadIdx.x == 0) bars->shared_unit[k] = u;
                n_shared |= 1 << k;
            }
            if (!(ti.flags & TILE_END)) continue;
            if (n_shared) {
                if (!merge_sync()) break;
                if (threadIdx.x < 2 && (n_shared >> threadIdx.x & 1)) {
                    const UnitDesc& s = bars->shared_unit[threadIdx.x];
                    const bool last = atomic_inc_acq_rel(&p.counters[s.first_cta]) == static_cast<uint32_t>(s.parts) - 1;
                    bars->arrived[threadIdx.x] = last;
                    if (last) p.counters[s.first_cta] = 0;         // for the next launch
                }
                if (!merge_sync()) break;
                for (int k = 0; k < 2; ++k)
                    if ((n_shared >> k & 1) && bars->arrived[k]) join_parts<D>(p, bars->shared_unit[k]);
            }
            break;
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

template <int D, typename T>
int launch_paged(const dare_ctx* ctx, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const PagedParams& p, int ctas, cudaStream_t stream) {
    using S = PagedShape<D>;
    static_assert(2 * (S::SMEM + 1024) <= 228 * 1024, "two CTAs per SM");
    static std::atomic<uint64_t> smem_set{0};
    if (ensure_dynamic_smem(smem_set, attn_paged_kernel<D, T>, S::SMEM) != DARE_OK) return DARE_ERR_CUDA;
    return launch_kernel(attn_paged_kernel<D, T>, dim3(ctas), (PG_WARPS + 1) * 32, S::SMEM, stream, 1, tm_k, tm_v, p);
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
    if (static_cast<long long>(L) * (Hq / Hkv) > (1 << 20) || Hq / Hkv > 128) return DARE_ERR_SHAPE;
    if (int rc = check_pages(B, max_pages, n_pages, page_size, Hkv)) return rc;
    if (!(scale >= 0.f) || isinf(scale) || window < 0 || sinks < 0) return DARE_ERR_RANGE;
    if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out)) return DARE_ERR_ALIGN;
    PagedAttnArgs a;
    a.B = B; a.L = L; a.Hq = Hq; a.Hkv = Hkv; a.d = d; a.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
    a.n_pages = n_pages; a.max_pages = max_pages;
    // a window that reaches further than any key is none (and keeps the kernels' sums within 32 bits)
    a.window = window >= (max_pages << a.page_shift) ? 0 : window;
    a.sinks = a.window > 0 ? sinks : 0;
    a.scale = scale != 0.f ? scale : 1.0f / sqrtf(static_cast<float>(d));
    a.q = q; a.k_pages = k_pages; a.v_pages = v_pages; a.table = block_table; a.kv_lens = kv_lens; a.out = out; a.lse = lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // Up to PG_ROWS packed query rows take the kernel of this file, more the tcgen05 kernel.  us here / there: 7 rows, 1 sequence of 300 keys
    // 6.8 / 9.2, of 8000 13.3 / 16.6, 18 of 2000 20.0 / 21.2, 64 of 4096 82 / 95, 74 of 250 to 4000 62 / 82.  With the rows as the MMA's 16 rows
    // instead of its 8 columns, 9 to 16 rows took 25.6 / 17.3, 22.4 / 21.3 and 31.4 / 32.7 for 1 of 8000, 18 of 2000 and 74 of 1000, and 32 rows
    // 46 / 17.5, 38 / 21.6 and 39.5 / 33.4.
    if (L * (Hq / Hkv) > PG_ROWS) {
        if (static_cast<long long>(B) * Hkv > 65535) return DARE_ERR_SHAPE;      // (a grid's second dimension)
        return launch_attn_paged_tc(ctx, a, s);
    }

    PagedParams p = {};
    p.B = B; p.L = L; p.Hq = Hq; p.Hkv = Hkv; p.g = Hq / Hkv; p.R = L * p.g;
    p.page_shift = a.page_shift; p.n_pages = n_pages; p.max_pages = max_pages; p.window = a.window; p.sinks = a.sinks;
    p.scale_log2 = a.scale * LOG2E_F;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.table = block_table; p.kv_lens = kv_lens;
    p.out = static_cast<__nv_bfloat16*>(out); p.lse = lse;
    p.counters = ctx->join_counters; p.dev_status = ctx->dev_status;
    // two CTAs per SM, all resident at once; no more than there can be tiles
    const long long tiles = static_cast<long long>(B) * Hkv * ((static_cast<long long>(max_pages) * page_size + PG_KT - 1) / PG_KT);
    // Tiles are numbered in 32 bits, twice their count included, unless sequences that share their pages could have more of them: with 64 bits
    // the divisions in front of a CTA's first tile take 1 sequence of 777 keys from 7.8 to 8.1 us, 64 of up to 4096 from 50.9 to 51.2.
    const bool many = tiles > (1LL << 29);
    long long ctas = 2LL * ctx->sm_count;
    if (ctas > PAGED_MAX_CTAS) ctas = PAGED_MAX_CTAS;
    p.places = static_cast<int>(ctas);
    if (ctas > tiles) ctas = tiles;
    const size_t part_rows = static_cast<size_t>(ctas) * 2 * PG_ROWS;
    if (part_rows * (d + 2) * sizeof(float) > ctx->workspace_bytes) return DARE_ERR_WORKSPACE;
    p.part_o = static_cast<float*>(ctx->workspace);
    p.part_ml = p.part_o + part_rows * d;
    CUtensorMap tm_k, tm_v;
    const uint64_t pool_rows = static_cast<uint64_t>(n_pages) * Hkv * page_size;
    const uint32_t box_rows = static_cast<uint32_t>(page_size < PG_KT ? page_size : PG_KT);
    int rc = make_tmap_bf16_halves(ctx, &tm_k, k_pages, pool_rows, d, box_rows);
    if (rc == DARE_OK) rc = make_tmap_bf16_halves(ctx, &tm_v, v_pages, pool_rows, d, box_rows);
    if (rc != DARE_OK) return rc;
    const int n = static_cast<int>(ctas);
    if (many) return d == 128 ? launch_paged<128, int64_t>(ctx, tm_k, tm_v, p, n, s) : launch_paged<64, int64_t>(ctx, tm_k, tm_v, p, n, s);
    return d == 128 ? launch_paged<128, int>(ctx, tm_k, tm_v, p, n, s) : launch_paged<64, int>(ctx, tm_k, tm_v, p, n, s);
}
