// Norms of queries and keys per head with the position rotation in the same pass, over the rows of a fused projection
// [rows, (Hq + 2 Hkv) d]: into dense q, k, v (dare_qk_norm_rope), with k and v into their pages of a cache
// (dare_paged_kv_append), and the gradient (dare_qk_norm_rope_backward).
//
// For a head x of d values at position p, with weight w:
//     r = 1 / sqrt(mean(x^2) + eps),  y = x r w,  (o_c, o_{c+d/2}) = (y_c cos - y_{c+d/2} sin, y_{c+d/2} cos + y_c sin)
// fp32 inside, rounded to bf16 once, at the end.  Its gradient, with g the output's: z = g turned back by the same angle,
//     dw += z x r,   dx = r (w z - x r mean(w z x r)).
// Everything here is one pass over memory and bound by it, and next to it by the instructions that unpack, add up, rotate and pack.
// The work is cut into items, runs of heads that lie side by side in a row (whole rows, where they fit a stage and there are enough
// of them); a warp takes every so many of them through a ring of its own: bulk copies bring the next item to shared memory while
// the warp works on this one in place, and bulk copies take it away.  So what is in flight does not hang on registers.
// A head is held by d / 16 lanes, 8 channels c.. and their partners c + d/2.. each (two 16-byte pieces), so that a norm is three
// (two) shuffles and a rotation none; the weights are multiplied into the angles once per item.
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace dare {
namespace {

enum { QKN_DENSE = 0, QKN_APPEND = 1, QKN_BACKWARD = 2 };

// One CTA per SM.  Stages of an item's run of heads, in the backward pass of values and of gradients: one that is worked on, the next one,
// one on its way out.  About as fast as a plain copy of the same bytes (4310 rows of 32 + 32 + 32 heads of 128 dense 36.7 us, copied 35.1 to
// 36.7; 19201 of 28 + 4 + 4 57 to 60, copied 61); 12 and 14 warps with larger stages 60 to 66 there.  The backward pass spills with 16 warps'
// 128 registers: 151 us instead of 88.
template <int MODE>
struct QkNormShape {
    static constexpr int WARPS = MODE == QKN_BACKWARD ? 12 : 16;             // at most
    static constexpr int STAGES = 3;
    static constexpr int STAGE_BYTES = MODE == QKN_BACKWARD ? 6144 : 4608;
};

struct QkNormParams {
    const __nv_bfloat16* qkv;                      // [rows, (Hq + 2 Hkv) d]
    int rows, Hq, Hkv;
    const uint4 *wq, *wk;                          // bf16 [d], or NULL: no norm
    float eps;
    const int32_t* positions;                      // [rows]
    const float4* rope;                            // [n_positions, d/2] (cos, sin)
    int n_positions;
    int item_heads, row_items;                     // heads of an item, items of a row
    __nv_bfloat16 *q_out, *k_out, *v_out;          // [rows, Hq, d], [rows, Hkv, d] (append: k_out and v_out are the pages)
    // append
    const int32_t *seq_ids, *table;
    int n_seqs, max_pages, n_pages, page_shift;
    // backward
    const __nv_bfloat16 *gq, *gk, *gv;             // [rows, Hq, d], [rows, Hkv, d] twice
    __nv_bfloat16* dx;                             // [rows, (Hq + 2 Hkv) d]
    float* part;                                   // [CTAs][2][d] sums of the weights' gradients
    uint32_t* dev_status;
};

// An item: heads [h0, h0 + nq + nk + nv) of a row: nq query heads from q0 on, nk key heads from k0 on, nv value heads from v0 on.
struct Item {
    int row, h0, nq, nk, nv, q0, k0, v0;
    __device__ __forceinline__ Item(int row_, int k, int per, int Hq, int Hkv) : row(row_), h0(k * per) {
        const int end = min(h0 + per, Hq + 2 * Hkv);
        q0 = min(h0, Hq);
        nq = min(end, Hq) - q0;
        k0 = min(max(h0 - Hq, 0), Hkv);
        nk = min(max(end - Hq, 0), Hkv) - k0;
        v0 = max(h0 - Hq - Hkv, 0);
        nv = max(end - Hq - Hkv, 0) - v0;
    }
};
// The place of an item in the list of all rows' items, walked in steps of one size.
struct ItemWalk {
    int row, k, n, row_step, k_step;
    __device__ __forceinline__ ItemWalk(int first, int step, int n_)
        : row(first / n_), k(first - row * n_), n(n_), row_step(step / n_), k_step(step - row_step * n_) {}
    __device__ __forceinline__ void next() {
        row += row_step;
        k += k_step;
        if (k >= n) { k -= n; ++row; }
    }
};

// Eight bf16 values as four pairs of fp32, and back.
__device__ __forceinline__ void unpack8(const uint4& v, uint64_t (&f)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pack_b32x2(w[i] << 16, w[i] & 0xffff0000u);
}
__device__ __forceinline__ uint4 pack8(const uint64_t (&f)[4]) {
    return make_uint4(pack_bf16(lo_f32x2(f[0]), hi_f32x2(f[0])), pack_bf16(lo_f32x2(f[1]), hi_f32x2(f[1])),
                      pack_bf16(lo_f32x2(f[2]), hi_f32x2(f[2])), pack_bf16(lo_f32x2(f[3]), hi_f32x2(f[3])));
}
__device__ __forceinline__ uint64_t both(float x) { return pack_f32x2(x, x); }
__device__ __forceinline__ float dot8(const uint64_t (&a)[4], const uint64_t (&b)[4], const uint64_t (&c)[4], const uint64_t (&d)[4]) {
    uint64_t s = mul_f32x2(a[0], b[0]), t = mul_f32x2(c[0], d[0]);
#pragma unroll
    for (int j = 1; j < 4; ++j) {
        s = fma_f32x2(a[j], b[j], s);
        t = fma_f32x2(c[j], d[j], t);
    }
    s = add_f32x2(s, t);
    return lo_f32x2(s) + hi_f32x2(s);
}
template <int LANES>
__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// The forward pass of `heads` heads of one kind, in place: o = r (a (wa cos) - b (wb sin)), r (b (wb cos) + a (wa sin)).
template <int D>
__device__ __forceinline__ void rotate_heads(uint8_t* at, int heads, const uint4* w, float eps, const uint64_t (&cs)[4], const uint64_t (&sn)[4]) {
    constexpr int LANES = D / 16, PER = 32 / LANES;
    const int lane = threadIdx.x & 31, piece = lane % LANES, sub = lane / LANES;
    uint64_t ca[4], sb[4], cb[4], sa[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        ca[j] = cb[j] = cs[j];
        sa[j] = sn[j];
        sb[j] = sn[j] ^ 0x8000000080000000ull;
    }
    if (w != nullptr) {
        uint64_t wa[4], wb[4];
        unpack8(w[piece], wa);
        unpack8(w[LANES + piece], wb);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ca[j] = mul_f32x2(ca[j], wa[j]);
            sa[j] = mul_f32x2(sa[j], wa[j]);
            cb[j] = mul_f32x2(cb[j], wb[j]);
            sb[j] = mul_f32x2(sb[j], wb[j]);
        }
    }
    uint4* x = reinterpret_cast<uint4*>(at + sub * D * 2) + piece;
#pragma unroll 2
    for (int h = 0; h < heads; h += PER, x += PER * D / 8) {
        const bool live = h + sub < heads;         // (beyond the last head lies whatever the stage holds: not written)
        uint64_t a[4], b[4], lo[4], hi[4];
        unpack8(x[0], a);
        unpack8(x[LANES], b);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            lo[j] = fma_f32x2(a[j], ca[j], mul_f32x2(b[j], sb[j]));
            hi[j] = fma_f32x2(b[j], cb[j], mul_f32x2(a[j], sa[j]));
        }
        if (w != nullptr) {
            const uint64_t r = both(rsqrtf(sum_lanes<LANES>(dot8(a, a, b, b)) * (1.f / D) + eps));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lo[j] = mul_f32x2(lo[j], r);
                hi[j] = mul_f32x2(hi[j], r);
            }
        }
        if (live) {
            x[0] = pack8(lo);
            x[LANES] = pack8(hi);
        }
    }
}

// The backward pass of `heads` heads of one kind: gradients g in place, the heads' values x; acc: the weight's gradient so far.
template <int D>
__device__ __forceinline__ void rotate_heads_back(uint8_t* g_at, const uint8_t* x_at, int heads, const uint4* w, float eps, const uint64_t (&cs)[4],
                                                  const uint64_t (&sn)[4], uint64_t (&acc)[8]) {
    constexpr int LANES = D / 16, PER = 32 / LANES;
    const int lane = threadIdx.x & 31, piece = lane % LANES, sub = lane / LANES;
    uint64_t wa[4], wb[4], ns[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) ns[j] = sn[j] ^ 0x8000000080000000ull;
    if (w != nullptr) {
        unpack8(w[piece], wa);
        unpack8(w[LANES + piece], wb);
    }
    uint4* g = reinterpret_cast<uint4*>(g_at + sub * D * 2) + piece;
    const uint4* x = reinterpret_cast<const uint4*>(x_at + sub * D * 2) + piece;
    for (int h = 0; h < heads; h += PER, g += PER * D / 8, x += PER * D / 8) {
        const bool live = h + sub < heads;
        uint64_t ga[4], gb[4], za[4], zb[4];
        unpack8(g[0], ga);
        unpack8(g[LANES], gb);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            za[j] = fma_f32x2(ga[j], cs[j], mul_f32x2(gb[j], sn[j]));
            zb[j] = fma_f32x2(gb[j], cs[j], mul_f32x2(ga[j], ns[j]));
        }
        if (w != nullptr) {
            uint64_t xa[4], xb[4], ya[4], yb[4];
            unpack8(x[0], xa);
            unpack8(x[LANES], xb);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                ya[j] = mul_f32x2(wa[j], za[j]);
                yb[j] = mul_f32x2(wb[j], zb[j]);
            }
            const float r = rsqrtf(sum_lanes<LANES>(dot8(xa, xa, xb, xb)) * (1.f / D) + eps);
            const float m = sum_lanes<LANES>(dot8(ya, xa, yb, xb)) * r * (1.f / D);            // mean(w z x r)
            const uint64_t rr = both(r), mr = both(-m * r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                xa[j] = mul_f32x2(xa[j], rr);                                // x r
                xb[j] = mul_f32x2(xb[j], rr);
                if (live) {
                    acc[j] = fma_f32x2(za[j], xa[j], acc[j]);
                    acc[4 + j] = fma_f32x2(zb[j], xb[j], acc[4 + j]);
                }
                za[j] = fma_f32x2(xa[j], mr, mul_f32x2(ya[j], rr));
                zb[j] = fma_f32x2(xb[j], mr, mul_f32x2(yb[j], rr));
            }
        }
        if (live) {
            g[0] = pack8(za);
            g[LANES] = pack8(zb);
        }
    }
}

template <int D, int MODE>
__global__ void __launch_bounds__(QkNormShape<MODE>::WARPS * 32, 1)
qk_norm_kernel(const QkNormParams p) {
    constexpr int QKN_WARPS = QkNormShape<MODE>::WARPS, QKN_STAGES = QkNormShape<MODE>::STAGES, QKN_STAGE_BYTES = QkNormShape<MODE>::STAGE_BYTES;
    constexpr bool BACK = MODE == QKN_BACKWARD, APPEND = MODE == QKN_APPEND;
    constexpr int LANES = D / 16, HEAD = D * 2;                              // lanes per head, bytes
    constexpr int SECOND = BACK ? QKN_STAGE_BYTES / 2 : 0;                   // the gradients' half of a stage
    extern __shared__ __align__(128) uint8_t qkn_smem[];
    __shared__ uint64_t bars[QKN_WARPS][QKN_STAGES];
    __shared__ uint4 weights[2][D / 8];                                      // (beside the rings there is little L1 left)
    __shared__ uint32_t abort_word;
    volatile uint32_t* abort_flag = &abort_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane % LANES, sub = lane / LANES, warps = blockDim.x >> 5;
    uint8_t* ring = qkn_smem + warp * QKN_STAGES * QKN_STAGE_BYTES;
    if (threadIdx.x == 0) {
        for (int i = 0; i < warps * QKN_STAGES; ++i) mbar_init(&bars[0][0] + i, 1);
        abort_word = 0;
        fence_barrier_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    const int heads_in = p.Hq + 2 * p.Hkv;
    const int step = static_cast<int>(gridDim.x) * warps;
    const int first = warp * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x);      // (few items: spread over the SMs)
    ItemWalk now(first, step, p.row_items), ahead = now;
    const bool normed = p.wq != nullptr;
    if (normed) {
        for (int c = threadIdx.x; c < 2 * (D / 8); c += blockDim.x) weights[c / (D / 8)][c % (D / 8)] = c < D / 8 ? p.wq[c] : p.wk[c - D / 8];
        __syncthreads();
    }
    const uint4 *wq = normed ? weights[0] : nullptr, *wk = normed ? weights[1] : nullptr;

    auto send_for = [&](const ItemWalk& w, int stage, bool wanted) {         // lane 0; an item that is not wanted arrives without bytes
        const Item it(w.row, w.k, p.item_heads, p.Hq, p.Hkv);
        uint8_t* dst = ring + stage * QKN_STAGE_BYTES;
        uint64_t* bar = &bars[warp][stage];
        const uint32_t all = static_cast<uint32_t>(it.nq + it.nk + it.nv) * HEAD;
        // (the backward pass reads the values of queries and keys, where they are normalised)
        const uint32_t values = !wanted ? 0 : !BACK ? all : normed ? static_cast<uint32_t>(it.nq + it.nk) * HEAD : 0;
        mbar_arrive_expect_tx(bar, values + (BACK ? all : 0));
        if (values) bulk_load(dst, p.qkv + (static_cast<int64_t>(it.row) * heads_in + it.h0) * D, values, bar);
        if (BACK) {
            dst += SECOND;
            if (it.nq) bulk_load(dst, p.gq + (static_cast<int64_t>(it.row) * p.Hq + it.q0) * D, it.nq * HEAD, bar);
            if (it.nk) bulk_load(dst + it.nq * HEAD, p.gk + (static_cast<int64_t>(it.row) * p.Hkv + it.k0) * D, it.nk * HEAD, bar);
            if (it.nv) bulk_load(dst + (it.nq + it.nk) * HEAD, p.gv + (static_cast<int64_t>(it.row) * p.Hkv + it.v0) * D, it.nv * HEAD, bar);
        }
    };

    uint64_t acc[2][8];                                                      // the weights' gradients, pairs of channels
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[0][j] = acc[1][j] = 0;
    if (lane == 0 && ahead.row < p.rows) send_for(ahead, 0, true);
    ahead.next();
    // What an item needs besides its heads is asked for ahead of it, so that nothing waits for it: its position (and sequence) two
    // items before, its angles (and page) one item before.  (In the backward pass the angles that wait would spill: 106 us instead of 95 at 19201 rows.)
    struct Place { int pos, seq; };
    auto place_of = [&](const ItemWalk& w) -> Place {
        return w.row < p.rows ? Place{p.positions[w.row], APPEND ? p.seq_ids[w.row] : 0} : Place{-1, -1};
    };
    struct Angles { float4 t[4]; int page; bool inside; };
    auto angles_of = [&](const Place& at) -> Angles {
        Angles a = {};
        a.inside = at.pos >= 0 && at.pos < p.n_positions;
        if (APPEND) {
            a.inside = a.inside && at.seq >= 0 && at.seq < p.n_seqs && (at.pos >> p.page_shift) < p.max_pages;
            if (a.inside) a.page = p.table[static_cast<int64_t>(at.seq) * p.max_pages + (at.pos >> p.page_shift)];
        }
        if (a.inside) {
            const float4* t = p.rope + static_cast<int64_t>(at.pos) * (D / 4) + piece * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) a.t[j] = t[j];
        }
        return a;
    };
    Place place = place_of(now);
    ItemWalk later = now;
    later.next();
    Place place1 = place_of(later);
    Angles angles = {};
    if (!BACK) angles = angles_of(place);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    while (now.row < p.rows) {
        const Item it(now.row, now.k, p.item_heads, p.Hq, p.Hkv);
        const bool reports = now.k == 0 && lane == 0;
        now.next();
        later.next();
        const Place place2 = place_of(later);
        Angles angles1 = {};
        if (BACK) angles = angles_of(place);
        else angles1 = angles_of(place1);
        // the next item takes the place of the last but one, once the copies out of that have read it
        bulk_wait_read<1>();
        __syncwarp();
        // (append: rows of no sequence, as in a padded batch, are not read: 34.1 us instead of 36.5 where 512 of 4310 are)
        if (lane == 0 && ahead.row < p.rows) send_for(ahead, stage == QKN_STAGES - 1 ? 0 : stage + 1, !APPEND || place1.seq >= 0);
        ahead.next();
        uint64_t cs[4], sn[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            cs[j] = pack_f32x2(angles.t[j].x, angles.t[j].z);
            sn[j] = pack_f32x2(angles.t[j].y, angles.t[j].w);
        }
        const int pos = place.pos;
        const int64_t page = angles.page;
        const bool inside = angles.inside && (!APPEND || (page >= 0 && page < p.n_pages));
        if (!inside && reports && !(APPEND && place.seq < 0)) atomicOr(p.dev_status, DEV_INDEX_OUTSIDE);
        ok = __all_sync(0xffffffffu, mbar_wait(&bars[warp][stage], phase, abort_flag));
        if (!ok) break;
        uint8_t* at = ring + stage * QKN_STAGE_BYTES + SECOND;               // what is worked on, in place
        if (!inside) {
            if (!APPEND)                                                     // (append: the row is left out)
                for (int o = lane; o < (it.nq + it.nk + it.nv) * (D / 8); o += 32) reinterpret_cast<uint4*>(at)[o] = make_uint4(0, 0, 0, 0);
        } else if (!BACK) {
            if (it.nq) rotate_heads<D>(at, it.nq, wq, p.eps, cs, sn);
            if (it.nk) rotate_heads<D>(at + it.nq * HEAD, it.nk, wk, p.eps, cs, sn);
        } else {
            if (it.nq) rotate_heads_back<D>(at, at - SECOND, it.nq, wq, p.eps, cs, sn, acc[0]);
            if (it.nk) rotate_heads_back<D>(at + it.nq * HEAD, at - SECOND + it.nq * HEAD, it.nk, wk, p.eps, cs, sn, acc[1]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (BACK) {
            if (lane == 0) bulk_store(p.dx + (static_cast<int64_t>(it.row) * heads_in + it.h0) * D, at, static_cast<uint32_t>(it.nq + it.nk + it.nv) * HEAD);
        } else if (!APPEND || inside) {
            if (lane == 0 && it.nq) bulk_store(p.q_out + (static_cast<int64_t>(it.row) * p.Hq + it.q0) * D, at, it.nq * HEAD);
            at += it.nq * HEAD;
            if (APPEND) {
                // A head's place is a row of its page: short for bulk copies (one each cost 37.8 us instead of 36.8 at 4310 rows of 32 + 32 + 32 heads
                // of 128, 512 of them of no sequence).
                const int64_t in_page = pos & ((1 << p.page_shift) - 1);
                for (int o = lane; o < (it.nk + it.nv) * (D / 8); o += 32) {
                    const int h = o / (D / 8);
                    const int64_t head = h < it.nk ? it.k0 + h : it.v0 + h - it.nk;
                    reinterpret_cast<uint4*>((h < it.nk ? p.k_out : p.v_out) + (((page * p.Hkv + head) << p.page_shift) + in_page) * D)[o % (D / 8)] =
                        reinterpret_cast<const uint4*>(at)[o];
                }
            } else if (lane == 0) {
                if (it.nk) bulk_store(p.k_out + (static_cast<int64_t>(it.row) * p.Hkv + it.k0) * D, at, it.nk * HEAD);
                if (it.nv) bulk_store(p.v_out + (static_cast<int64_t>(it.row) * p.Hkv + it.v0) * D, at + it.nk * HEAD, it.nv * HEAD);
            }
        }
        bulk_commit();
        place = place1;
        place1 = place2;
        if (!BACK) angles = angles1;
        if (++stage == QKN_STAGES) { stage = 0; phase ^= 1; }
    }
    bulk_wait();
    if (BACK && normed) {
        // the CTA's sums, in a fixed order: lanes of the same channels, then the warps
        __syncthreads();                                                     // (the rings are idle)
        float* sums = reinterpret_cast<float*>(qkn_smem);                    // [warp][2][D]
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float x = lo_f32x2(acc[k][j]), y = hi_f32x2(acc[k][j]);
#pragma unroll
                for (int off = LANES; off < 32; off <<= 1) {
                    x += __shfl_xor_sync(0xffffffffu, x, off);
                    y += __shfl_xor_sync(0xffffffffu, y, off);
                }
                if (sub == 0) {
                    float* dst = sums + (warp * 2 + k) * D + (j < 4 ? 0 : D / 2) + piece * 8 + (j & 3) * 2;
                    dst[0] = x;
                    dst[1] = y;
                }
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * D; c += warps * 32) {
            float x = 0.f;
            for (int w = 0; w < warps; ++w) x += sums[w * 2 * D + c];
            p.part[static_cast<int64_t>(blockIdx.x) * 2 * D + c] = x;
        }
    }
    if (!ok) {
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000LL) {}                                // copies in flight land
        if (lane == 0) atomicOr(p.dev_status, DEV_WAIT_EXPIRED);
    }
}

// dw[k][c] = sum over the CTAs' parts, in their order; a warp per 8 channels of one weight's 2 d.
constexpr int DW_COLS = 8, DW_THREADS = 256;
__global__ void __launch_bounds__(DW_THREADS)
qk_norm_weight_sum_kernel(const float* __restrict__ part, int n, int d, float* __restrict__ dwq, float* __restrict__ dwk) {
    __shared__ float s[DW_THREADS / DW_COLS][DW_COLS];
    const int c = blockIdx.x * DW_COLS + threadIdx.x % DW_COLS, slice = threadIdx.x / DW_COLS;
    pdl_wait();
    pdl_trigger();
    float x = 0.f;
#pragma unroll 4
    for (int i = slice; i < n; i += DW_THREADS / DW_COLS) x += part[static_cast<int64_t>(i) * 2 * d + c];
    s[slice][threadIdx.x % DW_COLS] = x;
    __syncthreads();
    if (threadIdx.x < DW_COLS) {
        x = 0.f;
#pragma unroll
        for (int i = 0; i < DW_THREADS / DW_COLS; ++i) x += s[i][threadIdx.x];
        (c < d ? dwq : dwk)[c < d ? c : c - d] = x;
    }
}

template <int D, int MODE>
int launch_qk_norm(const QkNormParams& p, int ctas, int warps, cudaStream_t stream) {
    using S = QkNormShape<MODE>;
    // (a warp's pass may reach 32 / (D / 16) - 1 heads beyond the last of its stage: read, not used)
    constexpr int RING = S::STAGES * S::STAGE_BYTES, SMEM = S::WARPS * RING + 1024;
    static std::atomic<uint64_t> smem_set{0};
    if (ensure_dynamic_smem(smem_set, qk_norm_kernel<D, MODE>, SMEM) != DARE_OK) return DARE_ERR_CUDA;
    return launch_kernel(qk_norm_kernel<D, MODE>, dim3(ctas), warps * 32, warps * RING + 1024, stream, 1, p);
}
// Items as large as a stage holds, equal shares of a row; smaller ones, down to a warp's pass, where there would be none for some
// warps.  One CTA per SM, no more than there are items.
template <int MODE>
int run_qk_norm(const dare_ctx* ctx, QkNormParams& p, int d, int* ctas, cudaStream_t stream) {
    using S = QkNormShape<MODE>;
    const int pass = 32 / (d / 16), most = S::STAGE_BYTES / (d * 2) / (MODE == QKN_BACKWARD ? 2 : 1) / pass * pass, heads = p.Hq + 2 * p.Hkv;
    int n = (heads + most - 1) / most;
    const int64_t warps = static_cast<int64_t>(ctx->sm_count) * S::WARPS;
    while (static_cast<int64_t>(p.rows) * n < warps && n * pass < heads) ++n;
    p.item_heads = ((heads + n - 1) / n + pass - 1) / pass * pass;
    p.row_items = (heads + p.item_heads - 1) / p.item_heads;
    const int64_t items = static_cast<int64_t>(p.rows) * p.row_items;
    *ctas = static_cast<int>(items < ctx->sm_count ? items : ctx->sm_count);
    if (MODE == QKN_BACKWARD && p.wq && static_cast<size_t>(*ctas) * 2 * d * sizeof(float) > ctx->workspace_bytes) return DARE_ERR_WORKSPACE;
    const int64_t share = (items + *ctas - 1) / *ctas;
    const int warps_cta = static_cast<int>(share < S::WARPS ? share : S::WARPS);
    return d == 128 ? launch_qk_norm<128, MODE>(p, *ctas, warps_cta, stream) : launch_qk_norm<64, MODE>(p, *ctas, warps_cta, stream);
}

QkNormParams make_params(const dare_ctx* ctx, const void* qkv, int rows, int Hq, int Hkv, const void* wq, const void* wk, float eps,
                         const int32_t* positions, const float* rope, int n_positions) {
    QkNormParams p = {};
    p.qkv = static_cast<const __nv_bfloat16*>(qkv);
    p.rows = rows; p.Hq = Hq; p.Hkv = Hkv; p.eps = eps; p.positions = positions; p.n_positions = n_positions;
    p.wq = static_cast<const uint4*>(wq); p.wk = static_cast<const uint4*>(wk);
    p.rope = reinterpret_cast<const float4*>(rope);
    p.dev_status = ctx->dev_status;
    return p;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_rows(const dare_ctx* ctx, const void* qkv, int rows, int Hq, int Hkv, int d, const void* wq, const void* wk, float eps,
               const void* positions, const void* rope, int n_positions) {
    if (!ctx || !qkv || !positions || !rope) return DARE_ERR_NULL;
    if ((wq == nullptr) != (wk == nullptr)) return DARE_ERR_NULL;
    if (int rc = check_current_device(ctx)) return rc;
    if (rows < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || (d != 64 && d != 128) || n_positions < 1) return DARE_ERR_SHAPE;
    if (static_cast<int64_t>(Hq) + 2LL * Hkv > (1 << 20) || rows > (1 << 30) / (Hq + 2 * Hkv)) return DARE_ERR_SHAPE;      // (items are 32-bit)
    if (!(eps >= 0.f) || isinf(eps)) return DARE_ERR_RANGE;
    if (!aligned16(qkv) || !aligned16(wq) || !aligned16(wk) || !aligned16(rope)) return DARE_ERR_ALIGN;
    return DARE_OK;
}

}  // namespace
}  // namespace dare

extern "C" {

int dare_rope_table(dare_ctx* ctx, int n_positions, int d, double base, float* table, void* stream) {
    using namespace dare;
    if (!ctx || !table) return DARE_ERR_NULL;
    if (int rc = check_current_device(ctx)) return rc;
    if (n_positions < 1 || (d != 64 && d != 128) || n_positions > (1 << 24)) return DARE_ERR_SHAPE;
    if (!(base > 1.0) || isinf(base)) return DARE_ERR_RANGE;
    if (!aligned16(table)) return DARE_ERR_ALIGN;
    return launch_rope_table(table, nullptr, n_positions, d / 2, base, static_cast<cudaStream_t>(stream));
}

int dare_qk_norm_rope(dare_ctx* ctx, const void* qkv, int n_rows, int Hq, int Hkv, int d, const void* q_weight, const void* k_weight,
                      float eps, const int32_t* positions, const float* rope_table, int n_positions, void* q_out, void* k_out,
                      void* v_out, void* stream) {
    using namespace dare;
    if (!q_out || !k_out || !v_out) return DARE_ERR_NULL;
    if (int rc = check_rows(ctx, qkv, n_rows, Hq, Hkv, d, q_weight, k_weight, eps, positions, rope_table, n_positions)) return rc;
    if (!aligned16(q_out) || !aligned16(k_out) || !aligned16(v_out)) return DARE_ERR_ALIGN;
    QkNormParams p = make_params(ctx, qkv, n_rows, Hq, Hkv, q_weight, k_weight, eps, positions, rope_table, n_positions);
    p.q_out = static_cast<__nv_bfloat16*>(q_out); p.k_out = static_cast<__nv_bfloat16*>(k_out); p.v_out = static_cast<__nv_bfloat16*>(v_out);
    int ctas = 0;
    return run_qk_norm<QKN_DENSE>(ctx, p, d, &ctas, static_cast<cudaStream_t>(stream));
}

int dare_paged_kv_append(dare_ctx* ctx, const void* qkv, int n_rows, int Hq, int Hkv, int d, const void* q_weight,
                         const void* k_weight, float eps, const float* rope_table, int n_positions, const int32_t* seq_ids,
                         const int32_t* positions, const int32_t* block_table, int n_seqs, int max_pages, int n_pages, int page_size,
                         void* k_pages, void* v_pages, void* q_out, void* stream) {
    using namespace dare;
    if (!seq_ids || !block_table || !k_pages || !v_pages || !q_out) return DARE_ERR_NULL;
    if (int rc = check_rows(ctx, qkv, n_rows, Hq, Hkv, d, q_weight, k_weight, eps, positions, rope_table, n_positions)) return rc;
    if (int rc = check_pages(n_seqs, max_pages, n_pages, page_size, Hkv)) return rc;
    if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(q_out)) return DARE_ERR_ALIGN;
    QkNormParams p = make_params(ctx, qkv, n_rows, Hq, Hkv, q_weight, k_weight, eps, positions, rope_table, n_positions);
    p.q_out = static_cast<__nv_bfloat16*>(q_out); p.k_out = static_cast<__nv_bfloat16*>(k_pages); p.v_out = static_cast<__nv_bfloat16*>(v_pages);
    p.seq_ids = seq_ids; p.table = block_table; p.n_seqs = n_seqs; p.max_pages = max_pages; p.n_pages = n_pages;
    p.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
    int ctas = 0;
    return run_qk_norm<QKN_APPEND>(ctx, p, d, &ctas, static_cast<cudaStream_t>(stream));
}

int dare_qk_norm_rope_backward(dare_ctx* ctx, const void* qkv, int n_rows, int Hq, int Hkv, int d, const void* q_weight,
                               const void* k_weight, float eps, const int32_t* positions, const float* rope_table, int n_positions,
                               const void* d_q, const void* d_k, const void* d_v, void* d_qkv, float* d_q_weight,
                               float* d_k_weight, void* stream) {
    using namespace dare;
    if (!d_q || !d_k || !d_v || !d_qkv) return DARE_ERR_NULL;
    if (q_weight && (!d_q_weight || !d_k_weight)) return DARE_ERR_NULL;
    if (int rc = check_rows(ctx, qkv, n_rows, Hq, Hkv, d, q_weight, k_weight, eps, positions, rope_table, n_positions)) return rc;
    if (!aligned16(d_q) || !aligned16(d_k) || !aligned16(d_v) || !aligned16(d_qkv)) return DARE_ERR_ALIGN;
    QkNormParams p = make_params(ctx, qkv, n_rows, Hq, Hkv, q_weight, k_weight, eps, positions, rope_table, n_positions);
    p.gq = static_cast<const __nv_bfloat16*>(d_q); p.gk = static_cast<const __nv_bfloat16*>(d_k); p.gv = static_cast<const __nv_bfloat16*>(d_v);
    p.dx = static_cast<__nv_bfloat16*>(d_qkv);
    p.part = static_cast<float*>(ctx->workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int ctas = 0, rc = run_qk_norm<QKN_BACKWARD>(ctx, p, d, &ctas, s);
    if (rc != DARE_OK || !q_weight) return rc;
    return launch_kernel(qk_norm_weight_sum_kernel, dim3(2 * d / DW_COLS), DW_THREADS, 0, s, 1, static_cast<const float*>(p.part), ctas, d,
                         d_q_weight, d_k_weight);
}

}  // extern "C"
