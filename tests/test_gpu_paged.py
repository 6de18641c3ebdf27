"""GPU parity of the operators around a paged key-value cache against the fp64 oracle.

Bars, from the arithmetic (bf16 inputs taken as they are; half a bf16 step is 2^-8 relative):
  * norms and rotation: one rounding at the end, 2^-8 |ref|.  In front of it: the sum of d <= 128 squares, its root, the products and the
    angles' rounding cost less than 2^-20 relative of each of the two terms of a rotation.
  * attention: the weights are rounded to bf16 in front of the second product, 2^-8 sum_j p_j |v_j| (up to 8 query rows per KV head: as two
    bf16 values, 2^-16); the output, 2^-8 |o|; scores
    are fp32 sums of d products, off by at most d 2^-24 max_j scale sum_c |q_c k_jc| (= s), and so are logarithms of weights and
    lse; e^(2s) - 1 <= 3 s of sum_j p_j |v_j|.  The exponential (2^-22), sums over keys and joins: 2^-16 (they are fp32 sums of at most 2^7 parts
    of a tile's 64 keys in turn).
  * gradients: of the rows as the forward; of the weights, an fp32 sum whose longest chain is below 2^9: 2^-15 sum |terms|, and 2^-20
    of each term.
"""
import numpy as np
import pytest
import torch

from oracle import dare_paged_oracle as P
from paper_2604_04215_b200 import binding as dare
from paper_2604_04215_b200 import inputs as I

from _util import f64

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    c = dare.Context(0)
    yield c
    c.close()


def _np(t):
    return t.float().cpu().double().numpy()


def _weights(d, seed, on=True):
    if not on:
        return None, None
    return tuple((1 + 0.25 * I.normal_bf16(seed, I.TID_W + i, (d,)).float()).to(torch.bfloat16) for i in range(2))


def _c(t):
    return None if t is None else t.cuda()


# ---------------------------------------------------------------------------------------------- norms and rotation

def _near_rotated(got, ref):
    """`ref` [..., d]: half a step of the value, 2^-20 of the two terms (bounded by the pair's length times sqrt 2)."""
    d = ref.shape[-1]
    pair = np.hypot(ref[..., :d // 2], ref[..., d // 2:])
    bound = HALF * np.abs(ref) + 2.0 ** -19 * np.concatenate([pair, pair], axis=-1) + 1e-30
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound).all(), f"excess {(np.abs(got - ref) - bound).max()}"


def test_rope_table(ctx):
    for n, d, base in ((1, 64, 10000.0), (1001, 128, 1e6), (70001, 64, 10000.0)):
        t = dare.dare_rope_table(ctx, n, d, base).cpu().double().numpy()
        rows = np.unique(np.array([0, 1, n // 2, n - 1]).clip(0, n - 1))
        ang = rows[:, None] * base ** (-2.0 * np.arange(d // 2) / d)
        # fp32 rounding of cos and sin, and what 2^-52 of the angle in radians costs
        bar = 2.0 ** -24 + ang.max() * 2.0 ** -50
        assert np.abs(t[rows, :, 0] - np.cos(ang)).max() <= bar and np.abs(t[rows, :, 1] - np.sin(ang)).max() <= bar


@pytest.mark.parametrize("rows,hq,hkv,d,weights", [
    (1, 1, 1, 64, True), (1, 28, 4, 128, True), (7, 14, 2, 64, True), (33, 32, 32, 128, False), (131, 4, 4, 64, True),
    (5, 3, 3, 128, True), (5, 6, 1, 64, False), (1100, 9, 3, 64, True), (9001, 2, 1, 128, True), (2, 71, 1, 128, True)])
def test_norm_rope_and_its_gradient(ctx, rows, hq, hkv, d, weights):
    seed, n_pos = rows + hq, 4099
    qkv = (I.normal_bf16(seed, 1, (rows, (hq + 2 * hkv) * d)).float() * (1 + 20 * (torch.arange(rows) % 3 == 1))[:, None]).to(torch.bfloat16)
    if rows > 4:
        qkv[3] = 0                                            # a row of zeros: eps alone
    pos = I.uniform_int(seed, 2, (rows,), 0, n_pos - 1)
    pos[0] = n_pos - 1
    outside = rows > 4
    if outside:
        pos[1], pos[2] = -1, n_pos
    wq, wk = _weights(d, seed, weights)
    g = [I.normal_bf16(seed, 3 + i, (rows, h, d)) for i, h in enumerate((hq, hkv, hkv))]
    table = dare.dare_rope_table(ctx, n_pos, d)
    q, k, v = dare.dare_qk_norm_rope(ctx, qkv.cuda(), pos.cuda(), table, hkv, _c(wq), _c(wk), EPS)
    dx, dwq, dwk = dare.dare_qk_norm_rope_backward(ctx, qkv.cuda(), pos.cuda(), table, *[t.cuda() for t in g], _c(wq), _c(wk), EPS)
    assert ctx.device_status() == (dare.DEV_INDEX_OUTSIDE if outside else 0)
    some = np.unique(np.concatenate([np.arange(min(rows, 40)), np.arange(max(0, rows - 9), rows)]))
    x64, p64 = f64(qkv)[some], pos.numpy()[some]
    rq, rk, rv = P.qk_norm_rope(x64, p64, hkv, d, f64(wq), f64(wk), EPS, n_positions=n_pos)
    _near_rotated(_np(q)[some], rq)
    _near_rotated(_np(k)[some], rk)
    assert (_np(v)[some] == rv).all()

    rdx, _, _ = P.qk_norm_rope_backward(x64, p64, hkv, d, *[f64(t)[some] for t in g], f64(wq), f64(wk), EPS, n_positions=n_pos)
    got, ref = _np(dx)[some].reshape(len(some), -1, d), rdx.reshape(len(some), -1, d)
    if not weights:
        _near_rotated(got[:, :hq + hkv], ref[:, :hq + hkv])
    else:
        # dx = r (w z - u mean(w z u)): 2^-19 of the terms r |w z| and r |u| mean |w z u|
        xs = x64.reshape(len(some), -1, d)[:, :hq + hkv]
        r = 1 / np.sqrt((xs ** 2).mean(axis=-1, keepdims=True) + EPS)
        gg = np.concatenate([f64(g[0])[some], f64(g[1])[some]], axis=1)
        pair = np.hypot(gg[..., :d // 2], gg[..., d // 2:])
        wz = np.concatenate([pair, pair], axis=-1) * np.concatenate([np.broadcast_to(np.abs(f64(wq)), (hq, d)), np.broadcast_to(np.abs(f64(wk)), (hkv, d))])
        u = np.abs(xs) * r
        bound = HALF * np.abs(ref[:, :hq + hkv]) + 2.0 ** -18 * r * (wz + u * (wz * u).mean(axis=-1, keepdims=True)) + 1e-30
        assert (np.abs(got[:, :hq + hkv] - ref[:, :hq + hkv]) <= bound).all()
    assert (got[:, hq + hkv:] == ref[:, hq + hkv:]).all()
    if not weights:
        assert dwq is None and dwk is None
        return
    # the weights' gradients over all rows, vectorised (the oracle's formula; the loops above are the definition)
    inside = (pos.numpy() >= 0) & (pos.numpy() < n_pos)
    x = f64(qkv).reshape(rows, -1, d)[inside]
    ang = pos.numpy()[inside][:, None] * 10000.0 ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    for got_w, lo, hi, gi in ((dwq, 0, hq, g[0]), (dwk, hq, hq + hkv, g[1])):
        gi = f64(gi)[inside]
        a, b = gi[..., :d // 2], gi[..., d // 2:]
        z = np.concatenate([a * c + b * s, b * c - a * s], axis=-1)
        t = z * x[:, lo:hi] / np.sqrt((x[:, lo:hi] ** 2).mean(axis=-1, keepdims=True) + EPS)
        pair = np.hypot(a, b)
        size = np.concatenate([pair, pair], axis=-1) * np.abs(x[:, lo:hi]) / np.sqrt((x[:, lo:hi] ** 2).mean(axis=-1, keepdims=True) + EPS)
        bound = (2.0 ** -15 + 2.0 ** -19) * size.sum(axis=(0, 1)) + 1e-30
        assert (np.abs(got_w.cpu().double().numpy() - t.sum(axis=(0, 1))) <= bound).all()


def test_norm_rope_gradient_against_differences_of_the_forward(ctx):
    """sum(g . forward(x + h e)) - sum(g . forward(x - h e)) over 2 h for weights: the forward is linear in them, so that its only
    error is the rounding of its outputs, 2^-8 of each term and side."""
    rows, hq, hkv, d, h = 40, 4, 2, 64, 0.5
    qkv = I.normal_bf16(1, 1, (rows, (hq + 2 * hkv) * d)).cuda()
    pos = torch.arange(rows, dtype=torch.int32).cuda()
    table = dare.dare_rope_table(ctx, rows, d)
    wq, wk = torch.ones(d, dtype=torch.bfloat16).cuda(), torch.ones(d, dtype=torch.bfloat16).cuda()
    g = [I.normal_bf16(1, 3 + i, (rows, n, d)).cuda() for i, n in enumerate((hq, hkv, hkv))]
    _, dwq, _ = dare.dare_qk_norm_rope_backward(ctx, qkv, pos, table, *g, wq, wk, EPS)
    for c in (0, 17, 32, 63):
        up, down = wq.clone(), wq.clone()
        up[c] += h
        down[c] -= h
        qu, qd = (dare.dare_qk_norm_rope(ctx, qkv, pos, table, hkv, w, wk, EPS)[0].double() for w in (up, down))
        diff = ((qu - qd) * g[0].double()).sum() / (2 * h)
        cols = [c % 32, c % 32 + 32]
        bar = HALF * ((qu.abs() + qd.abs()) * g[0].double().abs())[..., cols].sum() / (2 * h)
        assert abs(diff - dwq[c].double()) <= bar


# ---------------------------------------------------------------------------------------------- append

def _tables(seed, lens, page, spare=3):
    """Scattered pages for sequences of the given lengths; entries behind a sequence's last page are no pages at all."""
    per = max(1, max(-(-n // page) for n in lens))
    used = [-(-n // page) for n in lens]
    n_pages = sum(used) + spare
    order = np.random.default_rng(seed).permutation(n_pages)
    table = np.full((len(lens), per), -12345, dtype=np.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    return table, n_pages


@pytest.mark.parametrize("hq,hkv,d,page,weights", [(28, 4, 128, 16, True), (4, 4, 64, 64, False), (14, 2, 64, 32, True), (32, 8, 128, 1024, True)])
def test_append(ctx, hq, hkv, d, page, weights):
    seed, lens = 5, [1, page, page + 1, 0, 37, 2 * page + 5]
    table, n_pages = _tables(seed, lens, page)
    seq, pos = [], []
    for b, n in enumerate(lens):
        for p in range(max(0, n - 33), n):
            seq.append(b)
            pos.append(p)
    order = np.random.default_rng(1).permutation(len(seq))
    seq, pos = list(np.array(seq)[order]), list(np.array(pos)[order])
    n_pos = 2 * page + 5
    # rows of no sequence, a sequence that there is not, positions behind the angles, before 0, on an entry that is no page
    seq += [-1, -7, len(lens), 0, 0, 3]
    pos += [0, 10 ** 9, 0, n_pos, -1, 0]
    rows = len(seq)
    qkv = I.normal_bf16(seed, 1, (rows, (hq + 2 * hkv) * d))
    wq, wk = _weights(d, seed, weights)
    rope = dare.dare_rope_table(ctx, n_pos, d)
    kp, vp = (I.normal_bf16(seed, 6 + i, (n_pages, hkv, page, d)) for i in range(2))
    q0 = I.normal_bf16(seed, 8, (rows, hq, d))
    kd, vd, qd = kp.cuda(), vp.cuda(), q0.cuda()
    dare.dare_paged_kv_append(ctx, qkv.cuda(), torch.tensor(np.array(seq, dtype=np.int32)).cuda(), torch.tensor(np.array(pos, dtype=np.int32)).cuda(),
                              torch.from_numpy(table).cuda(), kd, vd, rope, _c(wq), _c(wk), EPS, q_out=qd)
    assert ctx.device_status() == dare.DEV_INDEX_OUTSIDE
    q, k, v = P.qk_norm_rope(f64(qkv), np.clip(pos, 0, n_pos - 1), hkv, d, f64(wq), f64(wk), EPS)
    rk, rv, rq = f64(kp).copy(), f64(vp).copy(), f64(q0).copy()
    assert P.paged_append(rk, rv, rq, q, k, v, seq, pos, table, n_pos)
    assert (_np(vd) == rv).all()
    _near_rotated(_np(kd), rk)
    _near_rotated(_np(qd), rq)
    # whatever was not written is as it was, bit for bit
    same_k, same_q = (rk == f64(kp)), (rq == f64(q0))
    assert (_np(kd)[same_k] == f64(kp)[same_k]).all() and (_np(qd)[same_q] == f64(q0)[same_q]).all()


# ---------------------------------------------------------------------------------------------- attention

def _attend_case(seed, B, L, hq, hkv, d, page, lens, window, sinks, plant=True):
    table, n_pages = _tables(seed, lens, page)
    q = I.normal_bf16(seed, 1, (B, L, hq, d), 1.5)
    kp, vp = (I.normal_bf16(seed, 6 + i, (n_pages, hkv, page, d)) for i in range(2))
    if plant:
        # NaN and infinities wherever no query may look: other pages, ends of last pages, between sinks and window
        seen = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            first = max(0, n - L - window + 1) if window else 0
            for j in list(range(min(sinks if window else 0, n))) + list(range(first, n)):
                seen[table[b, j // page], j % page] = True
        for t, bad in ((kp, float("nan")), (vp, float("inf"))):
            t.masked_fill_(~seen[:, None, :, None], bad)
        if window:
            for b, n in enumerate(lens):
                first = max(0, n - L - window + 1)
                for i in range(table.shape[1]):
                    if i * page >= sinks and (i + 1) * page <= first:
                        table[b, i] = 10 ** 6 if i % 2 else -1
    return q, kp, vp, table


def _check_attend(out, lse, q, kp, vp, table, lens, window, sinks, scale=0.0):
    ro, rl, pv, sabs = P.attn_paged(f64(q), f64(kp), f64(vp), table, lens, window, sinks, scale)
    d = q.shape[-1]
    s = d * 2.0 ** -24 * sabs                                            # [B, Hq, L]
    few = q.shape[1] * q.shape[2] // kp.shape[1] <= 8
    cost = np.swapaxes(3 * s, 1, 2)[..., None] + (2.0 ** -16 if few else HALF) + 2.0 ** -16
    bound = HALF * np.abs(ro) * (1 + HALF) + cost * pv + 1e-30
    got = _np(out)
    assert np.isfinite(got).all()
    assert (np.abs(got - ro) <= bound).all(), f"excess {(np.abs(got - ro) - bound).max()}"
    if lse is not None:
        gl = lse.cpu().double().numpy()
        assert (np.isneginf(gl) == np.isneginf(rl)).all()
        fin = np.isfinite(rl)
        assert (np.abs(gl[fin] - rl[fin]) <= (s + 2.0 ** -16 * (1 + np.abs(rl) + sabs))[fin]).all()


def _attend(ctx, q, kp, vp, table, lens, window, sinks, lse=True, **kw):
    B, L, hq, _ = q.shape
    lse_t = torch.full((B, hq, L), 7.0, device="cuda") if lse else None
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    dare.dare_attn_paged(ctx, q.cuda(), kp.cuda(), vp.cuda(), torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                         window=window, sinks=sinks, out=out, lse=lse_t, **kw)
    torch.cuda.synchronize()
    return out, lse_t


@pytest.mark.parametrize("L,hq,hkv,d,page,lens,window,sinks", [
    (1, 4, 4, 64, 16, [1], 0, 0),
    (1, 28, 4, 128, 16, [777], 0, 0),
    (1, 28, 4, 128, 64, [64, 65, 0, 63, 1, 128, 300], 0, 0),
    (1, 32, 8, 128, 32, [5, 1000, 31, 32, 33, 0], 0, 0),
    (1, 14, 2, 64, 128, [129, 2, 511], 0, 0),
    (1, 1, 1, 128, 1024, [2049, 1024], 0, 0),
    (1, 71, 1, 64, 16, [100, 17], 0, 0),                     # two chunks of rows, the second nearly empty
    (4, 32, 32, 128, 32, [4, 500, 0, 63], 0, 0),
    (4, 8, 2, 64, 16, [70, 4, 16], 0, 0),                    # 16 rows
    (5, 8, 2, 128, 16, [70, 5, 17], 0, 0),                   # 20 rows
    (8, 16, 4, 64, 64, [200, 8], 0, 0),                      # 32 rows
    (32, 28, 4, 128, 64, [640, 0, 33], 0, 0),                # 224 rows
    (33, 3, 1, 64, 16, [99, 33], 0, 0),                      # 99 rows
    (32, 4, 4, 64, 32, [96], 0, 0),
    (130, 2, 1, 128, 128, [300, 130], 0, 0),
    (1, 32, 8, 128, 16, [900, 64, 65, 1, 0, 70], 64, 4),
    (1, 28, 4, 128, 64, [900, 63, 200], 1, 0),
    (1, 4, 4, 64, 16, [500, 130], 100, 70),
    (1, 4, 4, 64, 128, [500, 130], 17, 0),
    (4, 8, 2, 128, 32, [400, 4, 70, 0, 129], 33, 5),
    (4, 8, 8, 64, 16, [400, 65], 1, 1),
    (32, 28, 4, 128, 16, [512, 40], 48, 4),
    (40, 4, 2, 64, 64, [512, 40], 7, 130),
    (1, 128, 1, 64, 16, [100, 3], 0, 0),                     # as many heads on one as a tile has rows, and a few less
    (3, 100, 1, 128, 32, [77, 3], 20, 2),
    (4, 4, 2, 64, 16, [2, 1, 3, 4], 0, 0),                   # fewer keys than queries
    (4, 4, 2, 64, 16, [2, 1, 3, 70], 2, 1),
    (40, 4, 2, 64, 16, [39, 1, 90], 3, 1),
    (2, 4, 4, 64, 16, [90], 90, 3),
    (2, 4, 4, 64, 16, [90], 2 ** 31 - 1, 2 ** 31 - 1),
])
def test_attend(ctx, L, hq, hkv, d, page, lens, window, sinks):
    q, kp, vp, table = _attend_case(L + hq, len(lens), L, hq, hkv, d, page, lens, window, sinks)
    for b, n in enumerate(lens):
        if n == 0:
            q[b] = float("nan")                              # an empty place of the batch: its queries are anything
    out, lse = _attend(ctx, q, kp, vp, table, lens, window, sinks)
    assert ctx.device_status() == 0
    for b, n in enumerate(lens):
        if n == 0:
            assert (out[b] == 0).all() and torch.isneginf(lse[b]).all()
            q[b] = 0
    _check_attend(out, lse, q, kp, vp, table, lens, window, sinks)
    again, lse2 = _attend(ctx, q, kp, vp, table, lens, window, sinks)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("L,hq,hkv,d,page,n_seqs,longest,window,sinks", [
    (32, 28, 4, 128, 64, 7, 300, 0, 0),                      # 224 rows in two tiles, one of them half full
    (32, 28, 4, 128, 16, 29, 150, 0, 0),                     # both tiles of a pair
    (32, 28, 4, 128, 32, 29, 260, 50, 3),
    (32, 28, 4, 64, 16, 29, 700, 0, 0),                      # the long ones of them taken one tile at a time
    (32, 28, 4, 64, 32, 29, 900, 400, 4),
    (19, 14, 2, 64, 16, 60, 600, 0, 0),                      # 133 rows: a full tile and one of 7
    (32, 28, 4, 128, 16, 7, 700, 64, 70),
    (97, 4, 4, 64, 16, 10, 300, 0, 0),                       # one tile per sequence, 31 rows of it empty
    (130, 16, 4, 64, 128, 13, 260, 0, 0),                    # five tiles
    (130, 16, 4, 64, 32, 13, 330, 33, 4),
    (200, 2, 2, 128, 16, 10, 420, 1, 0),
    (40, 3, 1, 128, 1024, 40, 130, 0, 0),                    # 120 rows: 42 positions of 3 heads
])
def test_attend_many_rows(ctx, L, hq, hkv, d, page, n_seqs, longest, window, sinks):
    """Enough units of 96 rows and more for the tcgen05 kernel."""
    rng = np.random.default_rng(L + n_seqs)
    lens = [0 if i % 11 == 5 else int(n) for i, n in enumerate(rng.integers(L, longest, n_seqs))]
    lens[0], lens[1], lens[-1] = longest, L, -(-L // 64) * 64
    q, kp, vp, table = _attend_case(L, n_seqs, L, hq, hkv, d, page, lens, window, sinks)
    out, lse = _attend(ctx, q, kp, vp, table, lens, window, sinks)
    assert ctx.device_status() == 0
    _check_attend(out, lse, q, kp, vp, table, lens, window, sinks)
    again, lse2 = _attend(ctx, q, kp, vp, table, lens, window, sinks)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_attend_many_rows_reports_lengths_and_pages_outside(ctx):
    lens = [100, 128, 40, 60, 70, 80, 90, 100, 110, 120]
    q, kp, vp, table = _attend_case(3, 10, 32, 28, 4, 64, 16, lens, 0, 0, plant=False)
    given = [table.shape[1] * 16 + 5, -3] + lens[2:]
    table[0, 7] = table[1, 7]
    out, lse = _attend(ctx, q, kp, vp, table, given, 0, 0)
    assert ctx.device_status() == dare.DEV_LEN_CLAMPED
    _check_attend(out, lse, q, kp, vp, table, [table.shape[1] * 16, 0] + lens[2:], 0, 0)
    table[3, 1], table[4, 0] = -1, kp.shape[0]
    out, lse = _attend(ctx, q, kp, vp, table, lens, 0, 0)
    assert ctx.device_status() == dare.DEV_INDEX_OUTSIDE
    _check_attend(out, lse, q, kp, vp, table, lens, 0, 0)


@pytest.mark.parametrize("L", [1, 3, 40])
def test_attend_many_sequences(ctx, L):
    """More sequences than the GPU has CTAs, of a few keys each; then few of them with all the work in one."""
    rng = np.random.default_rng(L)
    lens = [0 if i % 9 == 8 else int(n) for i, n in enumerate(rng.integers(L, 3 * L + 40, 700 if L < 40 else 90))]
    q, kp, vp, table = _attend_case(L, len(lens), L, 4, 2, 64, 16, lens, 0, 0)
    out, lse = _attend(ctx, q, kp, vp, table, lens, 0, 0)
    assert ctx.device_status() == 0
    _check_attend(out, lse, q, kp, vp, table, lens, 0, 0)
    lens = [L, 9000, L + 1, 0]
    q, kp, vp, table = _attend_case(L + 1, len(lens), L, 4, 2, 64, 32, lens, 0, 0)
    out, lse = _attend(ctx, q, kp, vp, table, lens, 0, 0)
    assert ctx.device_status() == 0
    _check_attend(out, lse, q, kp, vp, table, lens, 0, 0)


@pytest.mark.parametrize("B,hkv,lo,hi,window,sinks", [(70, 4, 600, 700, 0, 0), (35, 8, 100, 5000, 200, 4), (140, 2, 64, 300, 0, 0), (9, 1, 1, 20, 0, 0)])
def test_attend_units_of_like_length(ctx, B, hkv, lo, hi, window, sinks):
    """Units that each get a CTA of their own, in the first 32 sequences and behind them, empty places among them."""
    rng = np.random.default_rng(B)
    lens = [0 if i % 13 == 6 else int(n) for i, n in enumerate(rng.integers(lo, hi, B))]
    q, kp, vp, table = _attend_case(B, B, 1, 2 * hkv, hkv, 64, 16, lens, window, sinks)
    out, lse = _attend(ctx, q, kp, vp, table, lens, window, sinks)
    assert ctx.device_status() == 0
    _check_attend(out, lse, q, kp, vp, table, lens, window, sinks)


def test_attend_scale_shared_pages_and_no_lse(ctx):
    lens = [200, 150, 200]
    q, kp, vp, table = _attend_case(1, 3, 1, 8, 2, 128, 16, lens, 0, 0, plant=False)
    table[1, :9] = table[0, :9]                              # a prompt that two rollouts share
    table[2] = table[0]
    out, _ = _attend(ctx, q, kp, vp, table, lens, 0, 0, lse=False, scale=0.3)
    _check_attend(out, None, q, kp, vp, table, lens, 0, 0, scale=0.3)


def test_attend_large_scores(ctx):
    """Scores of some hundreds: the running maximum moves, weights underflow."""
    lens = [700, 65]
    q, kp, vp, table = _attend_case(2, 2, 2, 8, 2, 128, 16, lens, 0, 0)
    q = (q.float() * 20).to(torch.bfloat16)
    out, lse = _attend(ctx, q, kp, vp, table, lens, 0, 0)
    _check_attend(out, lse, q, kp, vp, table, lens, 0, 0)


@pytest.mark.parametrize("B,L,hq,hkv,n", [(2, 1, 14, 2, 300), (1, 1, 28, 4, 8000), (2, 32, 28, 4, 500), (1, 16, 14, 2, 4000), (9, 200, 28, 4, 600)])
def test_attend_query_that_is_not_finite(ctx, B, L, hq, hkv, n):
    """NaN in that query's own output and log-sum, nothing elsewhere: units whole and in parts, both kernels."""
    d, page, per = 128, 64, -(-n // 64)
    k, v = (I.normal_bf16(B + n, t, (B * per, hkv, page, d)).cuda() for t in (1, 2))
    q = I.normal_bf16(B + n, 3, (B, L, hq, d)).cuda()
    table = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    lse, lse0 = (torch.empty(B, hq, L, device="cuda") for _ in range(2))
    out0 = dare.dare_attn_paged(ctx, q, k, v, table, lens, lse=lse0)
    for value in (float("nan"), float("inf")):
        bad = q.clone()
        bad[0, L // 2, 1, 3] = value
        out = dare.dare_attn_paged(ctx, bad, k, v, table, lens, lse=lse)
        assert out[0, L // 2, 1].isnan().all() and lse[0, 1, L // 2].isnan()
        out[0, L // 2, 1], lse[0, 1, L // 2] = out0[0, L // 2, 1], lse0[0, 1, L // 2]
        assert torch.equal(out, out0) and torch.equal(lse, lse0)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("B,L,hq,hkv,n,window", [
    (2, 1, 14, 2, 1, 0), (3, 4, 4, 2, 2, 0), (2, 1, 14, 2, 300, 0), (1, 1, 28, 4, 8000, 0), (1, 1, 28, 4, 8000, 3000),      # up to 8 rows
    (2, 32, 28, 4, 1, 0), (9, 200, 28, 4, 600, 0), (2, 32, 28, 4, 500, 0), (1, 16, 14, 2, 4000, 0), (1, 16, 14, 2, 4000, 1500)])
def test_attend_query_whose_scores_are_all_minus_infinity(ctx, B, L, hq, hkv, n, window):
    """An infinite channel whose product with every visible key has the same sign: NaN for either sign, in units whole and in parts; a batch place
    without keys stays zero and -inf whatever its queries are."""
    d, page, per = 128, 64, -(-n // 64)
    k, v = (I.normal_bf16(B + n, t, (B * per, hkv, page, d)).cuda() for t in (1, 2))
    k[..., 3] = k[..., 3].abs() + 0.5
    q = I.normal_bf16(B + n, 3, (B, L, hq, d)).cuda()
    table = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    if B > 1:
        lens[B - 1] = 0
    lse, lse0 = (torch.empty(B, hq, L, device="cuda") for _ in range(2))
    out0 = dare.dare_attn_paged(ctx, q, k, v, table, lens, window=window, lse=lse0)
    assert out0.isfinite().all()
    for value in (float("inf"), -float("inf")):
        bad = q.clone()
        bad[0, L // 2, 1, 3] = value
        if B > 1:
            bad[B - 1, 0, :, 3] = value
        out = dare.dare_attn_paged(ctx, bad, k, v, table, lens, window=window, lse=lse)
        assert out[0, L // 2, 1].isnan().all() and lse[0, 1, L // 2].isnan()
        out[0, L // 2, 1], lse[0, 1, L // 2] = out0[0, L // 2, 1], lse0[0, 1, L // 2]
        if window:                                           # (a row may move its warp's reference a tile later: other roundings)
            assert out.isfinite().all() and lse.isfinite().all()
        else:
            assert torch.equal(out, out0) and torch.equal(lse, lse0)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("n,per_sm", [(64 * 600, 2), (64 * 40, 2), (64 * 3000, 1)])
def test_attend_a_rows_sum_does_not_move_with_its_neighbours_maximum(ctx, n, per_sm):
    """Two heads on the same keys, a unit per CTA.  All scores of the first are equal, 4126.5 scale, which has no 24-bit logarithm to the base 2; those of the second
    rise with every tile, so that its maximum moves each time.  With values 1 over the first half of the keys and 0 over the second
    the first head's output is 1/2, and what the second one does must not show in it."""
    d, page, tiles = 64, 64, n // 64
    B = per_sm * torch.cuda.get_device_properties(0).multi_processor_count
    t = torch.arange(tiles, dtype=torch.float32)
    k, v = (torch.zeros(tiles, 1, page, d) for _ in range(2))
    k[..., 0] = 63.0
    k[..., 1], k[..., 2], k[..., 3] = ((t // 256).view(-1, 1, 1), (t // 16 % 16).view(-1, 1, 1), (t % 16).view(-1, 1, 1))
    v[:tiles // 2, ..., 0] = 1.0
    k, v = (x.to(torch.bfloat16).cuda() for x in (k, v))
    table = torch.arange(tiles, dtype=torch.int32, device="cuda").repeat(B, 1)      # (all sequences share their pages)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    q = torch.zeros(B, 1, 2, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0, 0] = 65.5
    lse, found = torch.empty(B, 2, 1, device="cuda"), []
    for rise in (0.0, 1.0):
        q[..., 1, 1], q[..., 1, 2], q[..., 1, 3] = 256 * rise, 16 * rise, rise
        out = dare.dare_attn_paged(ctx, q, k, v, table, lens, lse=lse)
        assert (out[:, 0, 0, 0] == 0.5).all()
        found.append(lse[:, 0].clone())
    assert torch.equal(*found)
    # an fp32 sum of n / 4 equal weights a warp at most, pairs of them at a time; the logarithms' and the product's rounding
    want = 65.5 * 63.0 * 0.125 + np.log(n)
    assert np.abs(found[0].double().cpu().numpy() - want).max() <= 2.0 ** -21 * (want + 1) + n / 32 * 2.0 ** -24
    assert ctx.device_status() == 0


def test_attend_reports_lengths_and_pages_outside(ctx):
    lens = [200, 100]
    q, kp, vp, table = _attend_case(3, 2, 1, 4, 2, 64, 16, lens, 0, 0, plant=False)
    cap = table.shape[1] * 16
    table[1, 7:] = table[0, 7:13]
    for given, taken in (([cap + 1, 100], [cap, 100]), ([-5, 2 ** 31 - 1], [0, cap])):
        out, lse = _attend(ctx, q, kp, vp, table, given, 0, 0)
        assert ctx.device_status() == dare.DEV_LEN_CLAMPED
        _check_attend(out, lse, q, kp, vp, table, taken, 0, 0)
    table[0, 2], table[1, 6] = kp.shape[0], -1               # one of them a page that a length of 100 reaches into
    out, lse = _attend(ctx, q, kp, vp, table, lens, 0, 0)
    assert ctx.device_status() == dare.DEV_INDEX_OUTSIDE
    _check_attend(out, lse, q, kp, vp, table, lens, 0, 0)    # (zeros: the oracle's sequence() reads them so too)


def test_attend_pool_beyond_32_bit_offsets(ctx):
    hq, hkv, d, page, n_pages = 8, 8, 128, 64, 34000          # 2.2 G elements, 4.5 GB each
    kp, vp = (torch.zeros(n_pages, hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rope = dare.dare_rope_table(ctx, 4096, d)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    rows = 150
    qkv = I.normal_bf16(9, 1, (rows, 3 * hq * d))
    pos = torch.arange(rows, dtype=torch.int32)
    qd = dare.dare_paged_kv_append(ctx, qkv.cuda(), torch.zeros(rows, dtype=torch.int32, device="cuda"), pos.cuda(), table, kp, vp, rope)
    q, k, v = P.qk_norm_rope(f64(qkv), pos.numpy(), hkv, d)
    _near_rotated(_np(kp[n_pages - 2, :, :22]), k[128:].transpose(1, 0, 2))
    assert (_np(vp[n_pages - 1]) == v[:64].transpose(1, 0, 2)).all()
    out, _ = _attend_on(ctx, qd[-1:].view(1, 1, hq, d), kp, vp, table, [rows])
    small = [0, n_pages - 2, n_pages - 1]
    ks, vs = kp[small].cpu(), vp[small].cpu()
    _check_attend(out, None, qd[-1:].view(1, 1, hq, d).cpu(), ks, vs, np.array([[2, 0, 1]]), [rows], 0, 0)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("L,hq,hkv", [(1, 32, 32), (2, 128, 32), (3, 96, 32)])
def test_attend_table_as_wide_as_allowed(ctx, L, hq, hkv):
    """Two sequences, short, under a table of 2^30 positions: 2^34 of them and more over all KV heads."""
    lens, page, d = [700, 3], 1024, 64
    q, kp, vp, table = _attend_case(5, 2, L, hq, hkv, d, page, lens, 0, 0, plant=False)
    wide = torch.full((2, 2 ** 30 // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = torch.from_numpy(table)
    lse = torch.empty(2, hq, L, device="cuda")
    out = dare.dare_attn_paged(ctx, q.cuda(), kp.cuda(), vp.cuda(), wide, torch.tensor(lens, dtype=torch.int32, device="cuda"), lse=lse)
    assert ctx.device_status() == 0
    _check_attend(out, lse, q, kp, vp, table, lens, 0, 0)


def test_attend_many_sequences_under_a_wide_table(ctx):
    """65536 sequences under 513 pages of 1024 positions: 2^29 + 2^20 tiles, if all were filled; the same as under 3."""
    q = I.normal_bf16(6, 1, (65536, 1, 1, 64)).cuda()
    kp, vp = (I.normal_bf16(6, 6 + i, (3, 1, 1024, 64)).cuda() for i in range(2))
    lens = torch.from_numpy(np.random.default_rng(6).integers(0, 50, 65536).astype(np.int32))
    lens[::5000] = 2 * 1024 + 77
    table = torch.zeros(65536, 513, dtype=torch.int32, device="cuda")
    table[:, :3] = torch.tensor([2, 0, 1], dtype=torch.int32)
    lens = lens.cuda()
    out = dare.dare_attn_paged(ctx, q, kp, vp, table, lens)
    assert torch.equal(out, dare.dare_attn_paged(ctx, q, kp, vp, table[:, :3].contiguous(), lens)) and ctx.device_status() == 0
    some = list(range(0, 65536, 5000)) + [65535]
    _check_attend(out[some], None, q[some].cpu(), kp.cpu(), vp.cpu(), table[some, :3].cpu().numpy(), lens[some].tolist(), 0, 0)


def _attend_on(ctx, q, kp, vp, table, lens, window=0, sinks=0):
    out = dare.dare_attn_paged(ctx, q, kp, vp, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), window=window, sinks=sinks)
    torch.cuda.synchronize()
    return out, None


# ---------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_prompt_blocks_and_tokens_over_one_cache(ctx, window, sinks):
    """Three rollouts: ragged prompts in one append, then blocks of 4, then single tokens with one rollout finished; each step's
    attention against the oracle on the cache as the GPU has it, the cache against the oracle's own append."""
    hq, hkv, d, page, prompts = 8, 2, 64, 16, [37, 5, 16]
    B, cap = 3, 5
    table = np.random.default_rng(0).permutation(B * cap).reshape(B, cap).astype(np.int32)
    wq, wk = _weights(d, 4)
    n_pos = cap * page
    rope = dare.dare_rope_table(ctx, n_pos, d)
    kp, vp = (torch.full((B * cap, hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rk, rv = _np(kp), _np(vp)
    td = torch.from_numpy(table).cuda()
    lens = [0] * B

    def step(new, step_no):
        L = max(new)
        seq = np.array([b if i < n else -1 for b, n in enumerate(new) for i in range(L)], dtype=np.int32)
        pos = np.array([lens[b] + i if i < n else 0 for b, n in enumerate(new) for i in range(L)], dtype=np.int32)
        qkv = I.normal_bf16(step_no, 1, (B * L, (hq + 2 * hkv) * d))
        q = torch.zeros(B * L, hq, d, dtype=torch.bfloat16, device="cuda")
        dare.dare_paged_kv_append(ctx, qkv.cuda(), torch.from_numpy(seq).cuda(), torch.from_numpy(pos).cuda(), td, kp, vp, rope, wq.cuda(),
                                  wk.cuda(), EPS, q_out=q)
        oq, ok, ov = P.qk_norm_rope(f64(qkv), pos, hkv, d, f64(wq), f64(wk), EPS)
        P.paged_append(rk, rv, np.zeros_like(oq), oq, ok, ov, seq, pos, table, n_pos)
        for b in range(B):
            lens[b] += new[b]
        got_k, got_v = _np(kp), _np(vp)
        assert (np.isnan(got_k) == np.isnan(rk)).all() and ((got_v == rv) | np.isnan(rv)).all()
        _near_rotated(np.nan_to_num(got_k), np.nan_to_num(rk))
        return q.view(B, L, hq, d)

    step(prompts, 1)                                         # (the prompt's own attention is not what is looked at here)
    for n, new in enumerate([[4, 4, 4], [4, 4, 4], [1, 1, 1], [1, 0, 1], [1, 0, 1]]):
        q = step(new, 2 + n)
        out, _ = _attend_on(ctx, q, kp, vp, td, [m if k else 0 for m, k in zip(lens, new)], window, sinks)
        _check_attend(out, None, q.cpu(), kp.cpu(), vp.cpu(), table, [m if k else 0 for m, k in zip(lens, new)], window, sinks)
    assert ctx.device_status() == 0


def test_norms_in_front_of_packed_attention(ctx):
    """The training side: norms and rotation of packed tokens, dare_attn_varlen on what they give, against both oracles."""
    from oracle import dare_oracle as O
    hq, hkv, d, cu = 8, 2, 64, [0, 5, 70, 71]
    qkv = I.normal_bf16(3, 1, (71, (hq + 2 * hkv) * d))
    pos = torch.cat([torch.arange(b - a, dtype=torch.int32) for a, b in zip(cu, cu[1:])])
    wq, wk = _weights(d, 3)
    rope = dare.dare_rope_table(ctx, 65, d)
    q, k, v = dare.dare_qk_norm_rope(ctx, qkv.cuda(), pos.cuda(), rope, hkv, wq.cuda(), wk.cuda(), EPS)
    out = dare.dare_attn_varlen(ctx, q, k, v, torch.tensor(cu, dtype=torch.int32).cuda(), 65)
    ref = O.attn_varlen(_np(q), _np(k), _np(v), np.array(cu))
    ref = ref[0] if isinstance(ref, tuple) else ref
    assert np.abs(_np(out) - ref).max() <= 2e-2
    _near_rotated(_np(q), P.qk_norm_rope(f64(qkv), pos.numpy(), hkv, d, f64(wq), f64(wk), EPS)[0])


def test_paged_attention_is_the_dense_one(ctx):
    """The same keys in pages and in a dense cache: dare_attn_paged against dare_attn_block, both within their roundings."""
    B, L, hq, hkv, d, n, page = 2, 4, 8, 2, 128, 384, 64
    q = I.normal_bf16(7, 1, (B, L, hq, d)).cuda()
    k, v = (I.normal_bf16(7, 2 + i, (B, hkv, n, d)) for i in range(2))
    dense = dare.dare_attn_block(ctx, q, k.cuda(), v.cuda())
    kp, vp = (t.view(B, hkv, n // page, page, d).transpose(1, 2).reshape(-1, hkv, page, d).contiguous() for t in (k, v))
    table = np.arange(B * n // page, dtype=np.int32).reshape(B, -1)
    out, _ = _attend(ctx, q.cpu(), kp, vp, table, [n, n], 0, 0)
    _, _, pv, _ = P.attn_paged(f64(q.cpu()), f64(kp), f64(vp), table, [n, n])
    assert (np.abs(_np(out) - _np(dense)) <= 2 * HALF * (np.abs(_np(out)) + 1.1 * pv)).all()


def test_graph_replay_and_another_stream(ctx):
    """Append and attention captured once and replayed on new contents of the same buffers, then run on a side stream."""
    hq, hkv, d, page, lens = 8, 2, 64, 16, [40, 300]
    table, n_pages = _tables(2, lens, page)
    td = torch.from_numpy(table).cuda()
    rope = dare.dare_rope_table(ctx, 512, d)
    kp, vp = (I.normal_bf16(2, 6 + i, (n_pages, hkv, page, d)).cuda() for i in range(2))
    qkv = I.normal_bf16(2, 1, (2, (hq + 2 * hkv) * d)).cuda()
    seq, pos = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, 1], [n - 1 for n in lens]))
    nd = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q, out = torch.zeros(2, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 1, hq, d, dtype=torch.bfloat16, device="cuda")

    def both(stream=None):
        dare.dare_paged_kv_append(ctx, qkv, seq, pos, td, kp, vp, rope, q_out=q, stream=stream)
        dare.dare_attn_paged(ctx, q.view(2, 1, hq, d), kp, vp, td, nd, out=out, stream=stream)
    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for seed in (11, 12, 13):
        qkv.copy_(I.normal_bf16(seed, 1, tuple(qkv.shape)))
        pos.copy_(torch.tensor([lens[0] - 1, lens[1] - 1], dtype=torch.int32))
        nd.copy_(torch.tensor([lens[0], lens[1] - seed % 2], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        _check_attend(out, None, q.view(2, 1, hq, d).cpu(), kp.cpu(), vp.cpu(), table, nd.tolist(), 0, 0)
    want = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert torch.equal(out, want) and ctx.device_status() == 0


def test_backward_captured_and_replayed(ctx):
    rows, hq, hkv, d = 300, 8, 2, 64
    qkv = I.normal_bf16(1, 1, (rows, (hq + 2 * hkv) * d)).cuda()
    pos = torch.arange(rows, dtype=torch.int32).cuda()
    rope = dare.dare_rope_table(ctx, rows, d)
    wq, wk = (t.cuda() for t in _weights(d, 1))
    g = [I.normal_bf16(1, 3 + i, (rows, h, d)).cuda() for i, h in enumerate((hq, hkv, hkv))]
    outs = [torch.empty_like(qkv), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")]
    call = lambda: dare.dare_qk_norm_rope_backward(ctx, qkv, pos, rope, *g, wq, wk, EPS, *outs)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in outs:
        t.fill_(7)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))       # the sums are added in a fixed order


# ---------------------------------------------------------------------------------------------- refusals

def test_refusals(ctx):
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    before = dare.dare_kernel_launches()

    def attend(q=(2, 1, 4, 64), pool=(5, 2, 16, 64), table=(2, 3), **kw):
        return dare.dare_attn_paged(ctx, bf(*q), bf(*pool), bf(*pool), i32(*table), i32(q[0]), check=False, **kw)
    assert attend(pool=(5, 2, 24, 64)) == -2 and attend(pool=(5, 2, 8, 64)) == -2 and attend(pool=(5, 2, 2048, 64)) == -2
    assert attend(q=(2, 1, 4, 32), pool=(5, 2, 16, 32)) == -2 and attend(q=(2, 1, 5, 64)) == -2
    for empty in (dict(q=(0, 1, 4, 64), table=(0, 3)), dict(q=(2, 0, 4, 64)), dict(table=(2, 0)), dict(pool=(0, 2, 16, 64))):
        assert attend(**empty) == -1                         # (an empty tensor has no address)
    assert attend(q=(2, 1, 258, 64)) == -2                   # 129 query heads per KV head
    assert attend(q=(40000, 9, 2, 64), table=(40000, 1)) == -2      # more (sequence, KV head) pairs of more than 8 rows than a grid has
    assert attend(window=-1) == -4 and attend(sinks=-1) == -4 and attend(scale=-1.0) == -4 and attend(scale=float("nan")) == -4
    assert attend(scale=float("inf")) == -4
    rope = torch.zeros(10, 32, 2, device="cuda")

    def append(pool=(5, 2, 16, 64), rows=3, **kw):
        return dare.dare_paged_kv_append(ctx, bf(rows, 8 * 64), i32(rows), i32(rows), i32(2, 3), bf(*pool), bf(*pool), rope, check=False, **kw)
    assert append(pool=(5, 2, 24, 64)) == -2 and append(rows=0) == -1 and append(eps=-1.0) == -4 and append(eps=float("nan")) == -4
    assert append(q_weight=bf(64)) == -1                     # one weight without the other
    assert dare.dare_qk_norm_rope(ctx, bf(3, 8 * 64), i32(3), rope, 3, check=False) == -2          # 2 query heads on 3
    assert dare.dare_qk_norm_rope(ctx, bf(3, 8 * 64), i32(3), rope[:0], 2, check=False) == -1
    x = torch.zeros(8 * 64 * 3 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(3, 8 * 64)
    assert dare.dare_qk_norm_rope(ctx, x, i32(3), rope, 2, check=False) == -3
    assert dare.dare_qk_norm_rope_backward(ctx, bf(3, 8 * 64), i32(3), rope, bf(3, 4, 64), bf(3, 2, 64), bf(3, 2, 64), bf(64), None,
                                           check=False) == -1
    assert dare.dare_rope_table(ctx, 4, 32, check=False) == -2 and dare.dare_rope_table(ctx, 4, 64, base=1.0, check=False) == -4
    assert dare.dare_kernel_launches() == before and ctx.device_status() == 0
    with pytest.raises(ValueError, match="contiguous"):
        dare.dare_attn_paged(ctx, bf(2, 1, 4, 64), bf(5, 2, 64, 16).transpose(2, 3), bf(5, 2, 64, 16).transpose(2, 3), i32(2, 3), i32(2))
    with pytest.raises(ValueError, match="expected shape"):
        dare.dare_attn_paged(ctx, bf(2, 1, 4, 64), bf(5, 2, 16, 64), bf(5, 2, 32, 64), i32(2, 3), i32(2))
    with pytest.raises(ValueError, match="dtype"):
        dare.dare_attn_paged(ctx, bf(2, 1, 4, 64), bf(5, 2, 16, 64), bf(5, 2, 16, 64), i32(2, 3), i32(2).long())


@pytest.mark.parametrize("native", [True, False])
def test_window_and_sinks_beyond_32_bits_are_refused(ctx, monkeypatch, native):
    """Not taken modulo 2^32, by either way through the binding."""
    if not native:
        monkeypatch.setattr(dare, "_marshal", dare._NoNative)
    q, pages = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.full((1,), 20, dtype=torch.int32, device="cuda")
    before = dare.dare_kernel_launches()
    for kw in (dict(window=2 ** 32 + 5), dict(window=2 ** 31), dict(window=2 ** 70), dict(window=-2 ** 32 + 5), dict(window=5, sinks=2 ** 32),
               dict(window=5, sinks=-2 ** 40)):
        assert dare.dare_attn_paged(ctx, q, pages, pages, table, lens, check=False, **kw) == -4
    assert dare.dare_kernel_launches() == before
    dare.dare_attn_paged(ctx, q, pages, pages, table, lens, window=2 ** 31 - 1, sinks=2 ** 31 - 1)
    assert dare.dare_kernel_launches() == before + 1 and ctx.device_status() == 0


def test_refusals_of_counts_beyond_the_limits(ctx):
    """Given to the library as numbers: there is no memory for such tensors.  All are refused on the host."""
    lib, hq, hkv, d = dare.load(), 4, 2, 64
    x, pages = torch.zeros(4, 8 * d, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, hkv, 16, d, dtype=torch.bfloat16, device="cuda")
    ints, rope = torch.zeros(16, dtype=torch.int32, device="cuda"), torch.zeros(10, d // 2, 2, device="cuda")
    a, i, r, pg = x.data_ptr(), ints.data_ptr(), rope.data_ptr(), pages.data_ptr()
    before = dare.dare_kernel_launches()
    rows = 2 ** 30 // (hq + 2 * hkv) + 1
    assert lib.dare_qk_norm_rope(ctx.handle, a, rows, hq, hkv, d, None, None, EPS, i, r, 10, a, a, a, None) == -2
    assert lib.dare_qk_norm_rope_backward(ctx.handle, a, rows, hq, hkv, d, None, None, EPS, i, r, 10, a, a, a, a, None, None, None) == -2
    assert lib.dare_paged_kv_append(ctx.handle, a, rows, hq, hkv, d, None, None, EPS, r, 10, i, i, i, 1, 1, 1, 16, pg, pg, a, None) == -2
    assert lib.dare_rope_table(ctx.handle, 2 ** 24 + 1, d, 10000.0, r, None) == -2
    for base in (1.0, 0.5, 0.0, -2.0, float("inf"), float("nan")):
        assert lib.dare_rope_table(ctx.handle, 10, d, base, r, None) == -4
    for pool in ((2 ** 27, 16), (2 ** 21, 1024)):            # 2^31 rows of 2 KV heads and more: positions of the pool are 32-bit
        n_pages, page = pool
        assert lib.dare_attn_paged(ctx.handle, 1, 1, 4, 2, d, 0.0, a, pg, pg, n_pages, page, i, 1, i, 0, 0, a, None, None) == -2
        assert lib.dare_paged_kv_append(ctx.handle, a, 1, hq, hkv, d, None, None, EPS, r, 10, i, i, i, 1, 1, n_pages, page, pg, pg, a, None) == -2
    assert lib.dare_attn_paged(ctx.handle, 1, 1, 4, 2, d, 0.0, a, pg, pg, 1, 16, i, 2 ** 26 + 1, i, 0, 0, a, None, None) == -2
    assert lib.dare_attn_paged(ctx.handle, 1, 2 ** 19 + 1, 4, 2, d, 0.0, a, pg, pg, 1, 16, i, 1, i, 0, 0, a, None, None) == -2
    assert dare.dare_kernel_launches() == before and ctx.device_status() == 0


def test_workspace_too_small_is_refused():
    small = dare.Context(0, workspace_bytes=1 << 16)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    n = torch.ones(64, dtype=torch.int32, device="cuda")
    table = torch.zeros(64, 64, dtype=torch.int32, device="cuda")
    assert dare.dare_attn_paged(small, bf(64, 1, 4, 64), bf(5, 2, 16, 64), bf(5, 2, 16, 64), table, n, check=False) == -5
    assert small.device_status() == 0
    small.close()
