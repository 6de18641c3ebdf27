"""The measured work of the operators around a paged key-value cache: norms of queries and keys with the position rotation
(and their backward pass), the append to the cache, and the attention that reads it.

`run` computes them through the public calls of paper_2604_04215_b200.binding (own = True) or in plain elementary torch
operations in 32 bits (own = False); `exact` computes them in 64 bits.  Head layouts are those of
paper_2604_04215_b200.inputs (LLaDA-, Dream- and SDAR-shaped: 32 + 32 and 28 + 4 heads of 128, 4 + 4 of 64) and generic
ones.  A case is one of

    append    rows of a fused projection: q and k normalised per head and rotated to their sequence's position, k and v
              written to their pages
    attend    `new` positions of each sequence over its pages, all earlier positions and each other visible, optionally
              within a sliding window and beside a few first positions
    norm      the same norms and rotation for packed sequences, without a cache (scoring and update passes)
    norm_back its gradient with respect to the projection's rows and to the two weights
"""
import math
import random

import torch

own = False

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
EPS, BASE = 1e-6, 10000.0
HEADS = [(28, 4, 128), (32, 32, 128), (32, 8, 128), (4, 4, 64), (14, 2, 64)]


def listed():
    return [
        # A token each of 64 sequences of very different lengths, three places of the batch empty.
        dict(name="append_tokens", kind="append", q_heads=32, kv_heads=8, dim=128, seqs=64, new=1, ragged=True, longest=9001,
             page=16, norm=True),
        # The prompts of 16 rollouts, up to 512 tokens each, no norms: a prefill's append.
        dict(name="append_prompts", kind="append", q_heads=32, kv_heads=32, dim=128, seqs=16, new=512, ragged=True,
             longest=512, page=32, norm=False),
        # One token of one sequence of 777: what a single user waits for.
        dict(name="attend_token", kind="attend", q_heads=28, kv_heads=4, dim=128, seqs=1, new=1, ragged=False, longest=777,
             page=16, window=0, sinks=0),
        # A token each of 64 sequences of up to 4096: a decoding batch.
        dict(name="attend_tokens", kind="attend", q_heads=28, kv_heads=4, dim=128, seqs=64, new=1, ragged=True, longest=4096,
             page=64, window=0, sinks=0),
        # One token over a long context: all of it has to be cut into pieces and joined.
        dict(name="attend_token_long", kind="attend", q_heads=32, kv_heads=8, dim=128, seqs=1, new=1, ragged=False,
             longest=131071, page=64, window=0, sinks=0),
        # Blocks of 4 over caches of up to 5120, every head with its own keys: the largest read.
        dict(name="attend_blocks_4", kind="attend", q_heads=32, kv_heads=32, dim=128, seqs=64, new=4, ragged=True,
             longest=5120, page=32, window=0, sinks=0),
        # Blocks of 32 with grouped heads: 224 query rows share each key, the tensor pipe is as near as the memory.
        dict(name="attend_blocks_32", kind="attend", q_heads=28, kv_heads=4, dim=128, seqs=32, new=32, ragged=True,
             longest=1280, page=64, window=0, sinks=0),
        # Sliding window of 1024 and four first tokens over contexts of up to 16 thousand.
        dict(name="attend_window", kind="attend", q_heads=32, kv_heads=8, dim=128, seqs=32, new=1, ragged=True, longest=16000,
             page=16, window=1024, sinks=4),
        # The prompts of 7 rollouts behind a shared instruction: long blocks, bound by the products.
        dict(name="attend_prompts", kind="attend", q_heads=28, kv_heads=4, dim=128, seqs=7, new=500, ragged=True, longest=1500,
             page=128, window=0, sinks=0),
        # Packed sequences of an update, 19 thousand tokens, forward.
        dict(name="norm_packed", kind="norm", q_heads=28, kv_heads=4, dim=128, rows=19201, norm=True),
        # The same, backward.
        dict(name="norm_back_packed", kind="norm_back", q_heads=28, kv_heads=4, dim=128, rows=19201, norm=True),
        # A small model's short batch, backward: launches count.
        dict(name="norm_back_small", kind="norm_back", q_heads=4, kv_heads=4, dim=64, rows=131, norm=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "norm", "norm_back"])
    hq, hkv, d = rng.choice(HEADS)
    case = dict(kind=kind, q_heads=hq, kv_heads=hkv, dim=d)
    if kind in ("norm", "norm_back"):
        return dict(case, rows=_log_int(rng, 1, 19201 * 4608 // ((hq + 2 * hkv) * d)), norm=rng.random() < 0.8)
    case.update(page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.6)
    if kind == "append":
        new = rng.choice([1, 1, 4, 32, _log_int(rng, 2, 512)])
        seqs = _log_int(rng, 1, min(64, 8192 // new))
        return dict(case, seqs=seqs, new=new, longest=max(new, _log_int(rng, 16, 8192)), norm=rng.random() < 0.7)
    new = rng.choice([1, 1, 1, 2, 4, 8, 32, _log_int(rng, 2, 512)])
    seqs = _log_int(rng, 1, 64)
    # no more keys to read than the largest listed case has, and no more products
    most = min(131071, 64 * 5120 * 32 * 128 // (seqs * hkv * d), 32 * 32 * 28 * 128 * 9000 // (seqs * new * hq * d))
    longest = max(new, _log_int(rng, 17, max(18, most)))
    window = rng.choice([0, 0, 0, _log_int(rng, 16, 4096)])
    return dict(case, seqs=seqs, new=new, longest=longest, window=window, sinks=rng.choice([0, 4, 64]) if window else 0)


# ---------------------------------------------------------------------------------------------- inputs

_CTX = []


def _context():
    """One context per program, as a rollout worker keeps it."""
    if not _CTX:
        from paper_2604_04215_b200 import binding as dare
        _CTX.append(dare.Context(torch.cuda.current_device()))
    return _CTX[0]


def _lengths(case):
    """Keys of each sequence, its new positions among them (0: an empty place of the batch).  A function of the case."""
    n, new, longest = case["seqs"], case["new"], case["longest"]
    if not case["ragged"]:
        return [longest] * n
    rng = random.Random("lengths %d %d %d" % (n, new, longest))
    low = max(1, longest // 16) if case["kind"] == "append" and new == longest else max(new, longest // 16)
    lengths = [rng.randint(low, longest) for _ in range(n)]
    for i in range(7, n, 20):
        lengths[i] = 0
    lengths[0] = longest
    return lengths


def _visible(case):
    """Keys that a case has to read, over all sequences."""
    total = 0
    for n in _lengths(case):
        first = max(0, n - case["new"] - case["window"] + 1) if case["window"] else 0
        total += n - first + min(first, case["sinks"])
    return total


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=BF16)


def _rope_table(n_positions, d):
    c = torch.arange(d // 2, device="cuda", dtype=F64)
    angle = torch.arange(n_positions, device="cuda", dtype=F64)[:, None] * BASE ** (-2.0 * c / d)
    return torch.stack([torch.cos(angle), torch.sin(angle)], dim=2).to(F32)


def _pages(case, gen, s):
    """A pool a little larger than its sequences need, their pages scattered over it."""
    page, lengths = case["page"], _lengths(case)
    per_seq = -(-max(lengths) // page)
    used = sum(-(-n // page) for n in lengths)
    n_pages = used + 5
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(I32).cpu()
    table = torch.zeros(case["seqs"], per_seq, dtype=I32)
    at = 0
    for b, n in enumerate(lengths):
        k = -(-n // page)
        table[b, :k] = order[at:at + k]
        at += k
    shape = (n_pages, case["kv_heads"], page, case["dim"])
    s.update(table=table.cuda(), k_pages=_normal(gen, *shape), v_pages=_normal(gen, *shape))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1009 + 17)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    s = dict(kind=case["kind"], hq=hq, hkv=hkv, d=d)
    if case["kind"] != "attend":
        if case["norm"]:
            # trained weights are near one; a row of a projection has entries of order one with a few heads much larger
            s["wq"] = (1 + 0.25 * torch.randn(d, generator=gen, device="cuda")).to(BF16)
            s["wk"] = (1 + 0.25 * torch.randn(d, generator=gen, device="cuda")).to(BF16)
        else:
            s["wq"] = s["wk"] = None
    if case["kind"] in ("norm", "norm_back"):
        rows = case["rows"]
        s["qkv"] = _normal(gen, rows, (hq + 2 * hkv) * d)
        # packed sequences of 16 to 1024 tokens: positions start again at 0
        rng, positions = random.Random(int(seed)), []
        while len(positions) < rows:
            positions += range(min(rng.randint(16, 1024), rows - len(positions)))
        s["positions"] = torch.tensor(positions, dtype=I32, device="cuda")
        s["rope"] = _rope_table(1024, d)
        if case["kind"] == "norm":
            s["out"] = [torch.empty(rows, h, d, dtype=BF16, device="cuda") for h in (hq, hkv, hkv)]
        else:
            s["grads"] = [_normal(gen, rows, h, d) for h in (hq, hkv, hkv)]
            s["out"] = [torch.empty_like(s["qkv"])] + [torch.empty(d, dtype=F32, device="cuda") if case["norm"] else None for _ in range(2)]
        return s
    lengths, new = _lengths(case), case["new"]
    _pages(case, gen, s)
    if case["kind"] == "append":
        # the last `new` positions of each sequence, all of a shorter one; the rows of empty places belong to no sequence
        seq, pos = [], []
        for b, n in enumerate(lengths):
            k = min(new, n) if n else new
            seq += [b if n else -1] * k
            pos += range(n - k, n) if n else [0] * k
        s["seq_ids"] = torch.tensor(seq, dtype=I32, device="cuda")
        s["positions"] = torch.tensor(pos, dtype=I32, device="cuda")
        s["qkv"] = _normal(gen, len(seq), (hq + 2 * hkv) * d)
        s["rope"] = _rope_table(max(lengths), d)
        s["q_out"] = torch.zeros(len(seq), hq, d, dtype=BF16, device="cuda")
    else:
        s.update(window=case["window"], sinks=case["sinks"], kv_lens=torch.tensor(lengths, dtype=I32, device="cuda"),
                 q=_normal(gen, len(lengths), new, hq, d))
        s["out"] = torch.empty_like(s["q"])
    return s


# ---------------------------------------------------------------------------------------------- one pass

def _angles(positions, d):
    c = torch.arange(d // 2, device=positions.device, dtype=F64)
    angle = positions.to(F64)[:, None, None] * BASE ** (-2.0 * c / d)
    return torch.cos(angle).to(F32), torch.sin(angle).to(F32)


def _norm_rope(x, weight, cos, sin):
    """x fp32 [rows, heads, d]."""
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(dim=2, keepdim=True) + EPS) * weight.float()
    a, b = x[..., :x.shape[2] // 2], x[..., x.shape[2] // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2).to(BF16)


def _norm_rope_back(x, weight, cos, sin, g):
    """Gradients with respect to x [rows, heads, d] and weight."""
    half = x.shape[2] // 2
    z = torch.cat([g[..., :half] * cos + g[..., half:] * sin, g[..., half:] * cos - g[..., :half] * sin], dim=2)
    if weight is None:
        return z, None
    r = 1 / torch.sqrt((x * x).mean(dim=2, keepdim=True) + EPS)
    xr, wz = x * r, weight.float() * z
    return r * (wz - xr * (wz * xr).mean(dim=2, keepdim=True)), (z * xr).sum(dim=(0, 1))


def _split(s):
    rows, hq, hkv, d = s["qkv"].shape[0], s["hq"], s["hkv"], s["d"]
    x = s["qkv"].view(rows, hq + 2 * hkv, d)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _plain_norm(s):
    q, k, v = _split(s)
    cos, sin = _angles(s["positions"], s["d"])
    return [_norm_rope(q.float(), s["wq"], cos, sin), _norm_rope(k.float(), s["wk"], cos, sin), v.contiguous()]


def _plain_norm_back(s):
    q, k, _ = _split(s)
    cos, sin = _angles(s["positions"], s["d"])
    gq, gk, gv = s["grads"]
    dq, dwq = _norm_rope_back(q.float(), s["wq"], cos, sin, gq.float())
    dk, dwk = _norm_rope_back(k.float(), s["wk"], cos, sin, gk.float())
    d_qkv = torch.cat([dq.to(BF16), dk.to(BF16), gv], dim=1).view_as(s["qkv"])
    return [t for t in (d_qkv, dwq, dwk) if t is not None]


def _plain_append(s):
    q, k, v = _plain_norm(s)
    rows = torch.nonzero(s["seq_ids"] >= 0)[:, 0]
    seq, pos, page = s["seq_ids"][rows].long(), s["positions"][rows].long(), s["k_pages"].shape[2]
    at = s["table"][seq, pos // page].long()
    s["k_pages"][at, :, pos % page] = k[rows]
    s["v_pages"][at, :, pos % page] = v[rows]
    s["q_out"][rows] = q[rows]
    return [s["q_out"], s["k_pages"], s["v_pages"]]


def _plain_attend(s):
    q, lens = s["q"], s["kv_lens"].long()
    B, L, hq, d = q.shape
    hkv = s["hkv"]
    # [B, pages, Hkv, page, d] -> [B, Hkv, keys, d]
    k, v = (p[s["table"].long()].transpose(1, 2).reshape(B, hkv, -1, d) for p in (s["k_pages"], s["v_pages"]))
    j = torch.arange(k.shape[2], device=q.device)
    at = (lens - L)[:, None] + torch.arange(L, device=q.device)                  # [B, L] positions of the queries
    seen = (j < lens[:, None])[:, None, :].expand(B, L, -1)                      # [B, L, keys]
    if s["window"]:
        seen = seen & ((j < s["sinks"]) | (j > at[:, :, None] - s["window"]))
    x = q.float().view(B, L, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, d)
    z = torch.matmul(x, k.float().transpose(2, 3)) / math.sqrt(d)
    z = z.view(B, hkv, hq // hkv, L, -1).masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(dim=4, keepdim=True).clamp_min(-3e38)
    e = torch.exp(z - top).view(B, hkv, -1, z.shape[4])
    total = e.sum(dim=3, keepdim=True)
    v = v.float().masked_fill(~(j < lens[:, None])[:, None, :, None], 0.0)
    o = torch.matmul(e, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.view(B, hkv, hq // hkv, L, d).permute(0, 3, 1, 2, 4).reshape(B, L, hq, d).to(BF16)


def _own(s):
    from paper_2604_04215_b200 import binding as dare
    ctx, kind = _context(), s["kind"]
    if kind == "attend":
        return dare.dare_attn_paged(ctx, s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_lens"], window=s["window"],
                                    sinks=s["sinks"], out=s["out"])
    if kind == "append":
        dare.dare_paged_kv_append(ctx, s["qkv"], s["seq_ids"], s["positions"], s["table"], s["k_pages"], s["v_pages"],
                                  s["rope"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS, q_out=s["q_out"])
        return [s["q_out"], s["k_pages"], s["v_pages"]]
    if kind == "norm":
        q, k, v = s["out"]
        dare.dare_qk_norm_rope(ctx, s["qkv"], s["positions"], s["rope"], s["hkv"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS,
                               q_out=q, k_out=k, v_out=v)
        return [q, k, v]
    d_qkv, dwq, dwk = s["out"]
    dare.dare_qk_norm_rope_backward(ctx, s["qkv"], s["positions"], s["rope"], *s["grads"], q_weight=s["wq"], k_weight=s["wk"],
                                    eps=EPS, d_qkv=d_qkv, d_q_weight=dwq, d_k_weight=dwk)
    return [t for t in (d_qkv, dwq, dwk) if t is not None]


def run(s):
    if own:
        return _own(s)
    return {"attend": _plain_attend, "append": _plain_append, "norm": _plain_norm, "norm_back": _plain_norm_back}[s["kind"]](s)


# ---------------------------------------------------------------------------------------------- what it has to do

def work(case):
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "attend":
        lengths, seen = _lengths(case), _visible(case)
        rows = sum(case["new"] for n in lengths if n) * hq
        return {"bytes": 2 * d * rows + 2 * d * len(lengths) * case["new"] * hq + 4 * d * hkv * seen + 4 * len(lengths) + 4 * (seen // case["page"]),
                "flops": 4 * d * hq * case["new"] * seen}
    if case["kind"] == "append":
        lengths = _lengths(case)
        rows = sum(min(case["new"], n) for n in lengths)
        index = 12
    else:
        rows, index = case["rows"], 4
    values = rows * (hq + 2 * hkv) * d
    passes = 3 if case["kind"] == "norm_back" else 2
    return {"bytes": 2 * passes * values + index * rows, "flops": (20 if passes == 3 else 10) * values}


# ---------------------------------------------------------------------------------------------- in 64 bits

def _exact_rotate(x, positions, sign):
    """x [rows, heads, d] in 64 bits: channels c and c + d/2 as one complex number, turned by sign * angle."""
    d = x.shape[2]
    angle = positions.to(F64)[:, None] * torch.exp(torch.arange(0, d, 2, device=x.device, dtype=F64) * (-math.log(BASE) / d))
    turn = torch.polar(torch.ones_like(angle), sign * angle)[:, None, :]
    y = torch.complex(x[:, :, :d // 2], x[:, :, d // 2:]) * turn
    return torch.cat([y.real, y.imag], dim=2)


def _exact_rows(s):
    rows, hq, hkv, d = s["qkv"].shape[0], s["hq"], s["hkv"], s["d"]
    x = s["qkv"].double().view(rows, hq + 2 * hkv, d)
    found = []
    for head, heads, weight in ((0, hq, s["wq"]), (hq, hkv, s["wk"])):
        y = x[:, head:head + heads]
        if weight is not None:
            y = weight.double() * y * (y.pow(2).sum(dim=2, keepdim=True) / d + EPS).rsqrt()
        found.append(_exact_rotate(y, s["positions"], 1.0))
    return found + [x[:, hq + hkv:]]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_rows(s)
    if case["kind"] == "norm_back":
        rows, hq, hkv, d = s["qkv"].shape[0], s["hq"], s["hkv"], s["d"]
        x = s["qkv"].double().view(rows, hq + 2 * hkv, d)
        parts, weights = [], []
        for head, heads, weight, g in ((0, hq, s["wq"], s["grads"][0]), (hq, hkv, s["wk"], s["grads"][1])):
            z = _exact_rotate(g.double(), s["positions"], -1.0)
            if weight is not None:
                # y = w u, u = x / n with n = sqrt(|x|^2 / d + eps):  du = (1 - u u^T / d) / n
                n = (x[:, head:head + heads].pow(2).mean(dim=2, keepdim=True) + EPS).sqrt()
                u = x[:, head:head + heads] / n
                weights.append(torch.einsum("rhd,rhd->d", z, u))
                z = z * weight.double()
                z = (z - u * torch.einsum("rhd,rhd->rh", z, u)[:, :, None] / d) / n
            parts.append(z)
        return [torch.cat(parts + [s["grads"][2].double()], dim=1).view(rows, -1)] + weights
    if case["kind"] == "append":
        q, k, v = _exact_rows(s)
        k_pages, v_pages, q_out, page = s["k_pages"].double(), s["v_pages"].double(), s["q_out"].double(), case["page"]
        # every row's place in the pool, as one number
        for b in range(case["seqs"]):
            mine = s["seq_ids"] == b
            if not bool(mine.any()):
                continue
            at = s["positions"][mine].long()
            pages = s["table"][b].long()[torch.div(at, page, rounding_mode="floor")]
            k_pages[pages, :, at % page], v_pages[pages, :, at % page] = k[mine], v[mine]
            q_out[mine] = q[mine]
        return [q_out, k_pages, v_pages]
    out = torch.zeros(s["q"].shape, dtype=F64, device="cuda")
    group = case["q_heads"] // case["kv_heads"]
    for b, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        pages = s["table"][b, :-(-n // case["page"])].long()
        for h in range(case["kv_heads"]):
            k = s["k_pages"][pages, h].double().view(-1, case["dim"])[:n]
            v = s["v_pages"][pages, h].double().view(-1, case["dim"])[:n]
            heads = slice(h * group, (h + 1) * group)
            z = torch.einsum("lgd,nd->lgn", s["q"][b, :, heads].double(), k) * case["dim"] ** -0.5
            if case["window"]:
                # query i stands at n - new + i and looks back over `window` positions, itself among them
                for i in range(case["new"]):
                    z[i, :, min(case["sinks"], n):max(0, min(n, n - case["new"] + i - case["window"] + 1))] = -math.inf
            out[b, :, heads] = torch.einsum("lgn,nd->lgd", torch.softmax(z, dim=2), v)
    return out
