// Norms of queries and keys per head with the position rotation in the same pass, over the rows of a fused projection
// [rows, (Hq + 2 Hkv) d]: into dense q, k, v (dare_qk_norm_rope), with k and v into their pages of a cache
// (dare_paged_kv_append), and the gradient (dare_qk_norm_rope_backward).
//
// For a head x of d values at position p, with weight w:
//     r = 1 / sqrt(mean(x^2) + eps),  y = x r w,  (o_c, o_{c+d/2}) = (y_c cos - y_{c+d/2} sin, y_{c+d/2} cos + y_c sin)
// fp32 inside, rounded to bf16 once, at the end.  Its gradient, with g the output's: z = g turned back by the same angle,
//     dw += z x r,   dx = r (w z - x r mean(w z x r)).
// Everything here is one pass over memory.  A head is held by d / 16 lanes, 8 channels c.. and their partners c + d/2.. each
// (two 16-byte pieces), so that a norm is three (two) shuffles and a rotation none; a warp takes a row, or a part of its
// heads where rows are few, keeps the row's 8 angles and the weights in registers and walks the heads.
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace dare {
namespace {

constexpr int QKN_WARPS = 8;        // warps per CTA

struct QkNormParams {
    const uint4* qkv;               // [rows, (Hq + 2 Hkv) d]
    int rows, Hq, Hkv;
    const uint4 *wq, *wk;           // bf16 [d], or NULL: no norm
    float eps;
    const int32_t* positions;       // [rows]
    const float4* rope;             // [n_positions, d/2] (cos, sin)
    int n_positions;
    int warps_per_row;
    uint4 *q_out, *k_out, *v_out;   // [rows, Hq, d], [rows, Hkv, d] (append: k_out and v_out are the pages)
    // append
    const int32_t *seq_ids, *table;
    int n_seqs, max_pages, n_pages, page_shift;
    uint32_t* dev_status;
};

struct QkNormGradParams {
    const uint4* qkv;
    int rows, Hq, Hkv;
    const uint4 *wq, *wk;
    float eps;
    const int32_t* positions;
    const float4* rope;
    int n_positions;
    int warps_per_row;
    const uint4 *gq, *gk, *gv;      // [rows, Hq, d], [rows, Hkv, d] twice
    uint4* dx;                      // [rows, (Hq + 2 Hkv) d]
    float* part;                    // [CTAs][2][d] sums of the weights' gradients
    uint32_t* dev_status;
};

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
template <int LANES>
__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// The 8 angles of a lane's channels at position pos (two to a 16-byte load).
template <int D>
__device__ __forceinline__ void load_angles(const float4* rope, int64_t pos, int piece, bool inside, float (&cs)[8], float (&sn)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 t = inside ? rope[pos * (D / 4) + piece * 4 + j] : make_float4(0.f, 0.f, 0.f, 0.f);
        cs[2 * j] = t.x;
        sn[2 * j] = t.y;
        cs[2 * j + 1] = t.z;
        sn[2 * j + 1] = t.w;
    }
}

// A row's heads in groups of 32 / LANES, queries, keys and values each starting a group of its own (so that a group's kind is
// the same in all lanes).
struct HeadGroups {
    int nq, nk, n;       // groups of queries, of keys (and as many of values), of all
    __device__ __forceinline__ HeadGroups(int Hq, int Hkv, int per) : nq((Hq + per - 1) / per), nk((Hkv + per - 1) / per), n(nq + 2 * nk) {}
};

// Where a lane's head of group `grp` is: kind 0 q, 1 k, 2 v; h the head within its kind; live: there is such a head.
struct HeadPlace {
    int kind, h, count;
    bool live;
    __device__ __forceinline__ HeadPlace(const HeadGroups& hg, int grp, int sub, int per, int Hq, int Hkv) {
        kind = grp < hg.nq ? 0 : grp < hg.nq + hg.nk ? 1 : 2;
        h = (grp - (kind == 0 ? 0 : kind == 1 ? hg.nq : hg.nq + hg.nk)) * per + sub;
        count = kind == 0 ? Hq : Hkv;
        live = h < count;
    }
};

template <int D, bool APPEND>
__global__ void __launch_bounds__(QKN_WARPS * 32)
qk_norm_rope_kernel(const QkNormParams p) {
    constexpr int LANES = D / 16, PER = 32 / LANES, V8 = D / 8;      // lanes per head, heads per warp, 16-byte pieces per head
    const int lane = threadIdx.x & 31, piece = lane % LANES, sub = lane / LANES;
    const int item = blockIdx.x * QKN_WARPS + (threadIdx.x >> 5);
    const int row = item / p.warps_per_row, part = item % p.warps_per_row;
    pdl_wait();
    pdl_trigger();
    if (row >= p.rows) return;
    const int pos = p.positions[row];
    bool inside = pos >= 0 && pos < p.n_positions;
    int64_t page = 0;
    if (APPEND) {
        const int seq = p.seq_ids[row];
        if (seq < 0) return;                                         // the row belongs to no sequence
        inside = inside && seq < p.n_seqs && (pos >> p.page_shift) < p.max_pages;
        if (inside) {
            page = p.table[static_cast<int64_t>(seq) * p.max_pages + (pos >> p.page_shift)];
            inside = page >= 0 && page < p.n_pages;
        }
    }
    if (!inside) {
        if (lane == 0 && part == 0) atomicOr(p.dev_status, DEV_INDEX_OUTSIDE);
        if (APPEND) return;
    }
    float cs[8], sn[8];
    load_angles<D>(p.rope, pos, piece, inside, cs, sn);
    const HeadGroups hg(p.Hq, p.Hkv, PER);
    const uint4* src = p.qkv + static_cast<int64_t>(row) * (p.Hq + 2 * p.Hkv) * V8;
    for (int grp = part; grp < hg.n; grp += p.warps_per_row) {
        const HeadPlace at(hg, grp, sub, PER, p.Hq, p.Hkv);
        const int h_in = at.h + (at.kind == 0 ? 0 : at.kind == 1 ? p.Hq : p.Hq + p.Hkv);
        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
        if (at.live) {
            lo = src[h_in * V8 + piece];
            hi = src[h_in * V8 + LANES + piece];
        }
        if (at.kind < 2) {
            float a[8], b[8];
            unpack8(lo, a);
            unpack8(hi, b);
            const uint4* w = at.kind == 0 ? p.wq : p.wk;
            if (w != nullptr) {
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss += a[j] * a[j] + b[j] * b[j];
                const float r = rsqrtf(sum_lanes<LANES>(ss) * (1.f / D) + p.eps);
                float wa[8], wb[8];
                unpack8(w[piece], wa);
                unpack8(w[LANES + piece], wb);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    a[j] *= r * wa[j];
                    b[j] *= r * wb[j];
                }
            }
            float x[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = a[j] * cs[j] - b[j] * sn[j];
                y[j] = b[j] * cs[j] + a[j] * sn[j];
            }
            lo = pack8(x);
            hi = pack8(y);
        }
        if (!at.live) continue;
        if (!APPEND && !inside) lo = hi = make_uint4(0, 0, 0, 0);
        uint4* dst;
        if (at.kind == 0) dst = p.q_out + (static_cast<int64_t>(row) * p.Hq + at.h) * V8;
        else if (APPEND) dst = (at.kind == 1 ? p.k_out : p.v_out) + (((page * p.Hkv + at.h) << p.page_shift) + (pos & ((1 << p.page_shift) - 1))) * V8;
        else dst = (at.kind == 1 ? p.k_out : p.v_out) + (static_cast<int64_t>(row) * p.Hkv + at.h) * V8;
        dst[piece] = lo;
        dst[LANES + piece] = hi;
    }
}

template <int D>
__global__ void __launch_bounds__(QKN_WARPS * 32)
qk_norm_rope_backward_kernel(const QkNormGradParams p) {
    constexpr int LANES = D / 16, PER = 32 / LANES, V8 = D / 8;
    __shared__ float s_dw[QKN_WARPS][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane % LANES, sub = lane / LANES;
    float acc[2][16];
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[0][j] = acc[1][j] = 0.f;
    const HeadGroups hg(p.Hq, p.Hkv, PER);
    pdl_wait();
    pdl_trigger();
    const int64_t items = static_cast<int64_t>(p.rows) * p.warps_per_row;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * QKN_WARPS + warp; item < items; item += static_cast<int64_t>(gridDim.x) * QKN_WARPS) {
        const int row = static_cast<int>(item / p.warps_per_row), part = static_cast<int>(item % p.warps_per_row);
        const int pos = p.positions[row];
        const bool inside = pos >= 0 && pos < p.n_positions;
        if (!inside && lane == 0 && part == 0) atomicOr(p.dev_status, DEV_INDEX_OUTSIDE);
        float cs[8], sn[8];
        load_angles<D>(p.rope, pos, piece, inside, cs, sn);
        const int64_t row_at = static_cast<int64_t>(row) * (p.Hq + 2 * p.Hkv);
        for (int grp = part; grp < hg.n; grp += p.warps_per_row) {
            const HeadPlace at(hg, grp, sub, PER, p.Hq, p.Hkv);
            const int h_in = at.h + (at.kind == 0 ? 0 : at.kind == 1 ? p.Hq : p.Hq + p.Hkv);
            const uint4* g = (at.kind == 0 ? p.gq : at.kind == 1 ? p.gk : p.gv) + (static_cast<int64_t>(row) * at.count + at.h) * V8;
            uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
            const bool on = at.live && inside;
            if (on) {
                lo = g[piece];
                hi = g[LANES + piece];
            }
            if (at.kind < 2) {
                float ga[8], gb[8], za[8], zb[8];
                unpack8(lo, ga);
                unpack8(hi, gb);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    za[j] = ga[j] * cs[j] + gb[j] * sn[j];
                    zb[j] = gb[j] * cs[j] - ga[j] * sn[j];
                }
                const uint4* w = at.kind == 0 ? p.wq : p.wk;
                if (w != nullptr) {
                    uint4 xlo = make_uint4(0, 0, 0, 0), xhi = xlo;
                    if (on) {
                        xlo = p.qkv[(row_at + h_in) * V8 + piece];
                        xhi = p.qkv[(row_at + h_in) * V8 + LANES + piece];
                    }
                    float xa[8], xb[8], wa[8], wb[8];
                    unpack8(xlo, xa);
                    unpack8(xhi, xb);
                    unpack8(w[piece], wa);
                    unpack8(w[LANES + piece], wb);
                    float ss = 0.f, dot = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        ss += xa[j] * xa[j] + xb[j] * xb[j];
                        dot += wa[j] * za[j] * xa[j] + wb[j] * zb[j] * xb[j];
                    }
                    const float r = rsqrtf(sum_lanes<LANES>(ss) * (1.f / D) + p.eps);
                    const float m = sum_lanes<LANES>(dot) * r * (1.f / D);          // mean(w z x r)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float ua = xa[j] * r, ub = xb[j] * r;
                        const float ta = za[j] * ua, tb = zb[j] * ub;
                        if (at.kind == 0) { acc[0][j] += ta; acc[0][8 + j] += tb; }
                        else { acc[1][j] += ta; acc[1][8 + j] += tb; }
                        za[j] = r * (wa[j] * za[j] - ua * m);
                        zb[j] = r * (wb[j] * zb[j] - ub * m);
                    }
                }
                lo = pack8(za);
                hi = pack8(zb);
            }
            if (!at.live) continue;
            uint4* dst = p.dx + (row_at + h_in) * V8;
            dst[piece] = lo;
            dst[LANES + piece] = hi;
        }
    }
    if (p.wq == nullptr) return;
    // the CTA's sums, in a fixed order: lanes of the same channels, then warps
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float x = acc[k][j];
#pragma unroll
            for (int off = LANES; off < 32; off <<= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
            if (sub == 0) s_dw[warp][(j < 8 ? 0 : D / 2) + piece * 8 + (j & 7)] = x;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += QKN_WARPS * 32) {
            float x = 0.f;
#pragma unroll
            for (int w = 0; w < QKN_WARPS; ++w) x += s_dw[w][c];
            p.part[(static_cast<int64_t>(blockIdx.x) * 2 + k) * D + c] = x;
        }
        __syncthreads();
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

// Warps per row: one where the rows fill the GPU (32 warps on each SM), else up to one for each group of heads.
int pick_warps_per_row(int rows, int Hq, int Hkv, int d, int sm_count) {
    const int per = 32 / (d / 16), groups = (Hq + per - 1) / per + 2 * ((Hkv + per - 1) / per);
    int w = 1;
    while (w * 2 <= groups && static_cast<int64_t>(rows) * w < 32LL * sm_count) w *= 2;
    return w;
}

int backward_ctas(int rows, int warps_per_row, int sm_count) {
    const int64_t need = (static_cast<int64_t>(rows) * warps_per_row + QKN_WARPS - 1) / QKN_WARPS;
    return static_cast<int>(need < 2LL * sm_count ? need : 2LL * sm_count);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_rows(const dare_ctx* ctx, const void* qkv, int rows, int Hq, int Hkv, int d, const void* wq, const void* wk, float eps,
               const void* positions, const void* rope, int n_positions) {
    if (!ctx || !qkv || !positions || !rope) return DARE_ERR_NULL;
    if ((wq == nullptr) != (wk == nullptr)) return DARE_ERR_NULL;
    if (int rc = check_current_device(ctx)) return rc;
    if (rows < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || (d != 64 && d != 128) || n_positions < 1) return DARE_ERR_SHAPE;
    if (static_cast<int64_t>(Hq) + 2LL * Hkv > (1 << 20) || rows > (1 << 26)) return DARE_ERR_SHAPE;
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
    QkNormParams p = {};
    p.qkv = static_cast<const uint4*>(qkv);
    p.rows = n_rows; p.Hq = Hq; p.Hkv = Hkv; p.eps = eps; p.positions = positions; p.n_positions = n_positions;
    p.wq = static_cast<const uint4*>(q_weight); p.wk = static_cast<const uint4*>(k_weight);
    p.rope = reinterpret_cast<const float4*>(rope_table);
    p.q_out = static_cast<uint4*>(q_out); p.k_out = static_cast<uint4*>(k_out); p.v_out = static_cast<uint4*>(v_out);
    p.dev_status = ctx->dev_status;
    p.warps_per_row = pick_warps_per_row(n_rows, Hq, Hkv, d, ctx->sm_count);
    const int64_t items = static_cast<int64_t>(n_rows) * p.warps_per_row;
    return launch_kernel(d == 128 ? qk_norm_rope_kernel<128, false> : qk_norm_rope_kernel<64, false>,
                         dim3(static_cast<unsigned>((items + QKN_WARPS - 1) / QKN_WARPS)), QKN_WARPS * 32, 0,
                         static_cast<cudaStream_t>(stream), 1, p);
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
    QkNormParams p = {};
    p.qkv = static_cast<const uint4*>(qkv);
    p.rows = n_rows; p.Hq = Hq; p.Hkv = Hkv; p.eps = eps; p.positions = positions; p.n_positions = n_positions;
    p.wq = static_cast<const uint4*>(q_weight); p.wk = static_cast<const uint4*>(k_weight);
    p.rope = reinterpret_cast<const float4*>(rope_table);
    p.q_out = static_cast<uint4*>(q_out); p.k_out = static_cast<uint4*>(k_pages); p.v_out = static_cast<uint4*>(v_pages);
    p.seq_ids = seq_ids; p.table = block_table; p.n_seqs = n_seqs; p.max_pages = max_pages; p.n_pages = n_pages;
    p.page_shift = __builtin_ctz(static_cast<unsigned>(page_size));
    p.dev_status = ctx->dev_status;
    p.warps_per_row = pick_warps_per_row(n_rows, Hq, Hkv, d, ctx->sm_count);
    const int64_t items = static_cast<int64_t>(n_rows) * p.warps_per_row;
    return launch_kernel(d == 128 ? qk_norm_rope_kernel<128, true> : qk_norm_rope_kernel<64, true>,
                         dim3(static_cast<unsigned>((items + QKN_WARPS - 1) / QKN_WARPS)), QKN_WARPS * 32, 0,
                         static_cast<cudaStream_t>(stream), 1, p);
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
    QkNormGradParams p = {};
    p.qkv = static_cast<const uint4*>(qkv);
    p.rows = n_rows; p.Hq = Hq; p.Hkv = Hkv; p.eps = eps; p.positions = positions; p.n_positions = n_positions;
    p.wq = static_cast<const uint4*>(q_weight); p.wk = static_cast<const uint4*>(k_weight);
    p.rope = reinterpret_cast<const float4*>(rope_table);
    p.gq = static_cast<const uint4*>(d_q); p.gk = static_cast<const uint4*>(d_k); p.gv = static_cast<const uint4*>(d_v);
    p.dx = static_cast<uint4*>(d_qkv);
    p.part = static_cast<float*>(ctx->workspace);
    p.dev_status = ctx->dev_status;
    p.warps_per_row = pick_warps_per_row(n_rows, Hq, Hkv, d, ctx->sm_count);
    const int ctas = backward_ctas(n_rows, p.warps_per_row, ctx->sm_count);
    if (q_weight && static_cast<size_t>(ctas) * 2 * d * sizeof(float) > ctx->workspace_bytes) return DARE_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc = launch_kernel(d == 128 ? qk_norm_rope_backward_kernel<128> : qk_norm_rope_backward_kernel<64>, dim3(ctas), QKN_WARPS * 32,
                           0, s, 1, p);
    if (rc != DARE_OK || !q_weight) return rc;
    return launch_kernel(qk_norm_weight_sum_kernel, dim3(2 * d / DW_COLS), DW_THREADS, 0, s, 1, static_cast<const float*>(p.part), ctas, d,
                         d_q_weight, d_k_weight);
}

}  // extern "C"
