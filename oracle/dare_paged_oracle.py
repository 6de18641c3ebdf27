"""fp64 definitions of the operators around a paged key-value cache: norms of queries and keys per head with the position
rotation, their gradient, the append to the pages and the attention over them.  Plain loops over sequences, positions and
heads; nothing is tiled, split or fused."""
import numpy as np


def _angles(position, d, base):
    return position * base ** (-2.0 * np.arange(d // 2) / d)


def rotate(x, position, base=10000.0):
    """x [..., d] at `position`: channel c turns together with channel c + d/2."""
    d = x.shape[-1]
    a, b = x[..., :d // 2], x[..., d // 2:]
    c, s = np.cos(_angles(position, d, base)), np.sin(_angles(position, d, base))
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def norm(x, weight, eps):
    return x if weight is None else x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * weight


def qk_norm_rope(qkv, positions, n_kv_heads, d, wq=None, wk=None, eps=1e-6, base=10000.0, n_positions=None):
    """qkv [rows, (Hq + 2 Hkv) d] -> q [rows, Hq, d], k, v [rows, Hkv, d]; zeros for positions outside [0, n_positions)."""
    rows = qkv.shape[0]
    x = qkv.reshape(rows, -1, d)
    hq = x.shape[1] - 2 * n_kv_heads
    q, k, v = np.zeros((rows, hq, d)), np.zeros((rows, n_kv_heads, d)), np.zeros((rows, n_kv_heads, d))
    for m in range(rows):
        p = int(positions[m])
        if p < 0 or (n_positions is not None and p >= n_positions):
            continue
        q[m] = rotate(norm(x[m, :hq], wq, eps), p, base)
        k[m] = rotate(norm(x[m, hq:hq + n_kv_heads], wk, eps), p, base)
        v[m] = x[m, hq + n_kv_heads:]
    return q, k, v


def qk_norm_rope_backward(qkv, positions, n_kv_heads, d, dq, dk, dv, wq=None, wk=None, eps=1e-6, base=10000.0, n_positions=None):
    """Gradients with respect to qkv, wq, wk (the last two None without weights) by the chain rule, one head at a time: the
    rotation's transpose, the weight, and the derivative of x / n with n = sqrt(mean x^2 + eps) as a full d x d matrix."""
    rows = qkv.shape[0]
    x = qkv.reshape(rows, -1, d)
    hq = x.shape[1] - 2 * n_kv_heads
    dx = np.zeros_like(x)
    dws = [None if w is None else np.zeros(d) for w in (wq, wk)]
    for m in range(rows):
        p = int(positions[m])
        if p < 0 or (n_positions is not None and p >= n_positions):
            continue
        for h in range(hq + n_kv_heads):
            which = 0 if h < hq else 1
            w, g = (wq, wk)[which], (dq[m, h] if h < hq else dk[m, h - hq])
            z = rotate(g, -p, base)
            if w is None:
                dx[m, h] = z
                continue
            n = np.sqrt((x[m, h] ** 2).mean() + eps)
            dws[which] += z * x[m, h] / n
            jac = np.eye(d) / n - np.outer(x[m, h], x[m, h]) / (d * n ** 3)
            dx[m, h] = jac.T @ (z * w)
        dx[m, hq + n_kv_heads:] = dv[m]
    return dx.reshape(rows, -1), dws[0], dws[1]


def paged_append(k_pages, v_pages, q_out, q, k, v, seq_ids, positions, table, n_positions):
    """In place on the pages [n_pages, Hkv, page, d] and q_out; returns whether some row had to be left out."""
    n_pages, page = k_pages.shape[0], k_pages.shape[2]
    outside = False
    for m in range(len(seq_ids)):
        s, p = int(seq_ids[m]), int(positions[m])
        if s < 0:
            continue
        at = int(table[s, p // page]) if s < table.shape[0] and 0 <= p < min(n_positions, table.shape[1] * page) else -1
        if at < 0 or at >= n_pages:
            outside = True
            continue
        k_pages[at, :, p % page], v_pages[at, :, p % page], q_out[m] = k[m], v[m], q[m]
    return outside


def sequence(pages, table_row, n):
    """The first n positions of a sequence, [Hkv, n, d]; pages outside the pool are zeros."""
    n_pages, hkv, page, d = pages.shape
    out = np.zeros((hkv, n, d))
    for j0 in range(0, n, page):
        at, m = int(table_row[j0 // page]), min(page, n - j0)
        if 0 <= at < n_pages:
            out[:, j0:j0 + m] = pages[at, :, :m]
    return out


def attn_paged(q, k_pages, v_pages, table, kv_lens, window=0, sinks=0, scale=0.0):
    """q [B, L, Hq, d] -> o [B, L, Hq, d], lse [B, Hq, L], and the sums of p_j |v_j| and the largest sum_c |q_c k_jc| * scale (what
    roundings of the weights and of the scores can cost).  Only visible keys are touched."""
    B, L, hq, d = q.shape
    hkv, cap = k_pages.shape[1], table.shape[1] * k_pages.shape[2]
    scale = scale or 1.0 / np.sqrt(d)
    o, lse = np.zeros(q.shape), np.full((B, hq, L), -np.inf)
    pv, sabs = np.zeros(q.shape), np.zeros((B, hq, L))
    for b in range(B):
        n = min(max(int(kv_lens[b]), 0), cap)
        if n == 0:
            continue
        j = np.arange(n)
        first = max(0, n - L - window + 1) if window else 0
        some = (j >= first) | (j < sinks) if window else np.ones(n, bool)
        k, v = np.zeros((hkv, n, d)), np.zeros((hkv, n, d))
        for key in j[some]:
            at, r = int(table[b, key // k_pages.shape[2]]), key % k_pages.shape[2]
            if 0 <= at < k_pages.shape[0]:
                k[:, key], v[:, key] = k_pages[at, :, r], v_pages[at, :, r]
        for i in range(L):
            seen = np.ones(n, bool) if not window else (j < sinks) | (j > n - L + i - window)
            for h in range(hq):
                kh, vh = k[h * hkv // hq][seen], v[h * hkv // hq][seen]
                if not len(kh):
                    continue
                z = scale * kh @ q[b, i, h]
                e = np.exp(z - z.max())
                o[b, i, h] = e @ vh / e.sum()
                lse[b, h, i] = z.max() + np.log(e.sum())
                pv[b, i, h] = e @ np.abs(vh) / e.sum()
                sabs[b, h, i] = scale * (np.abs(kh) @ np.abs(q[b, i, h])).max()
    return o, lse, pv, sabs
