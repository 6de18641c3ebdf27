"""Pins of the paged-cache oracle, and what the entry points refuse; CPU only."""
import numpy as np
import pytest
import torch

from oracle import dare_model_oracle as MO
from oracle import dare_paged_oracle as P
from paper_2604_04215_b200 import binding


def _rng(seed):
    return np.random.default_rng(seed)


def test_rotation_is_the_stack_oracles_and_keeps_norms():
    x = _rng(0).standard_normal((3, 64))
    y = np.stack([P.rotate(x, p) for p in (0, 1, 977)])
    assert np.allclose(y[0], x) and np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
    z = x[:, :32] + 1j * x[:, 32:]
    turned = z * np.exp(1j * 977 * 10000.0 ** (-np.arange(32) / 32))
    assert np.allclose(y[2], np.concatenate([turned.real, turned.imag], axis=-1))
    # positions enter scores by their difference
    assert np.isclose(P.rotate(x[0], 40) @ P.rotate(x[1], 33), P.rotate(x[0], 7) @ P.rotate(x[1], 0))


def test_norm_has_unit_rms_and_the_weight_scales_channels():
    x = 3 * _rng(1).standard_normal((5, 128))
    assert np.allclose((P.norm(x, np.ones(128), 0.0) ** 2).mean(axis=-1), 1.0)
    w = _rng(2).standard_normal(128)
    assert np.allclose(P.norm(x, w, 0.0), P.norm(x, np.ones(128), 0.0) * w)
    assert np.array_equal(P.norm(x, None, 1e-6), x)


@pytest.mark.parametrize("weights", [True, False])
def test_backward_is_the_derivative_of_the_forward(weights):
    rng = _rng(3)
    rows, hq, hkv, d, pos = 3, 4, 2, 8, np.array([0, 5, 1001])
    x = rng.standard_normal((rows, (hq + 2 * hkv) * d))
    wq, wk = (rng.standard_normal(d), rng.standard_normal(d)) if weights else (None, None)
    g = [rng.standard_normal((rows, h, d)) for h in (hq, hkv, hkv)]

    def value(x, wq, wk):
        return sum((a * b).sum() for a, b in zip(P.qk_norm_rope(x, pos, hkv, d, wq, wk, 1e-3), g))

    def differences(f, at, eps=1e-6):
        out = np.zeros(at.size)
        for i in range(at.size):
            e = np.zeros(at.size)
            e[i] = eps
            out[i] = (f(at + e.reshape(at.shape)) - f(at - e.reshape(at.shape))) / (2 * eps)
        return out.reshape(at.shape)
    dx, dwq, dwk = P.qk_norm_rope_backward(x, pos, hkv, d, *g, wq, wk, 1e-3)
    assert np.allclose(dx, differences(lambda t: value(t, wq, wk), x), atol=1e-7)
    if weights:
        assert np.allclose(dwq, differences(lambda t: value(x, t, wk), wq), atol=1e-7)
        assert np.allclose(dwk, differences(lambda t: value(x, wq, t), wk), atol=1e-7)
    else:
        assert dwq is None and dwk is None


def test_rows_outside_the_table_are_zero_and_without_gradient():
    x = _rng(4).standard_normal((3, 4 * 8))
    q, k, v = P.qk_norm_rope(x, [-1, 2, 9], 1, 8, np.ones(8), np.ones(8), n_positions=9)
    assert not q[0].any() and not v[2].any() and q[1].any()
    dx, _, _ = P.qk_norm_rope_backward(x, [-1, 2, 9], 1, 8, q + 1, k + 1, v + 1, np.ones(8), np.ones(8), n_positions=9)
    assert not dx[0].any() and not dx[2].any() and dx[1].any()


@pytest.mark.parametrize("L,window,sinks", [(1, 0, 0), (3, 0, 0), (1, 7, 0), (3, 7, 2), (4, 1, 0), (4, 1, 3), (2, 100, 5)])
def test_attention_over_pages_is_masked_library_attention(L, window, sinks):
    rng = _rng(5)
    hq, hkv, d, page, lens = 4, 2, 16, 4, [L, 9, 22, 0]
    B = len(lens)
    table = rng.permutation(B * 6).reshape(B, 6)
    kp, vp = rng.standard_normal((2, B * 6, hkv, page, d))
    q = rng.standard_normal((B, L, hq, d))
    o, lse, pv, _ = P.attn_paged(q, kp, vp, table, lens, window, sinks)
    assert not o[3].any() and np.isneginf(lse[3]).all()
    for b in range(3):
        n = lens[b]
        k, v = (torch.from_numpy(np.repeat(P.sequence(t, table[b], n), hq // hkv, axis=0)) for t in (kp, vp))
        p = torch.arange(n - L, n)[:, None]
        j = torch.arange(n)[None, :]
        seen = torch.ones(L, n, dtype=torch.bool) if not window else (j < sinks) | (j > p - window)
        qq = torch.from_numpy(q[b]).transpose(0, 1)
        ref = torch.nn.functional.scaled_dot_product_attention(qq, k, v, attn_mask=seen[None].expand(hq, -1, -1))
        assert np.allclose(o[b], ref.transpose(0, 1).numpy(), atol=1e-12)
        z = (qq @ k.transpose(1, 2) / 4.0).masked_fill(~seen, -np.inf)
        assert np.allclose(lse[b], torch.logsumexp(z, dim=-1).numpy())
    assert (pv + 1e-12 >= np.abs(o)).all()


def test_append_then_sequence_gives_the_rows_back():
    rng = _rng(6)
    hkv, d, page = 2, 4, 4
    kp, vp = np.zeros((7, hkv, page, d)), np.zeros((7, hkv, page, d))
    table = np.array([[6, 0, 3], [2, 5, 1]])
    q, k, v = rng.standard_normal((6, 3, d)), rng.standard_normal((6, hkv, d)), rng.standard_normal((6, hkv, d))
    q_out = np.full((6, 3, d), 7.0)
    assert P.paged_append(kp, vp, q_out, q, k, v, [0, 0, 1, -1, 1, 2], [3, 4, 11, 0, 12, 0], table, 100)
    assert np.array_equal(P.sequence(kp, table[0], 5)[:, 3:], k[:2].transpose(1, 0, 2))
    assert np.array_equal(P.sequence(vp, table[1], 12)[:, 11], v[2])
    assert np.count_nonzero(kp.any(axis=(1, 3))) == 3 and (q_out[3:] == 7).all() and np.array_equal(q_out[:3], q[:3])


def test_stack_oracle_agrees_without_norms():
    """The rotation is the one of the layer stack (same pairing of channels, same base)."""
    x = _rng(7).standard_normal((4, 64))
    for p in (0, 3, 100):
        assert np.allclose(MO.rope(x[None], np.array([p]), 10000.0)[0], P.rotate(x, p))


# ---------------------------------------------------------------------------------------------- refusals without a GPU

NAMES = ["dare_rope_table", "dare_qk_norm_rope", "dare_qk_norm_rope_backward", "dare_paged_kv_append", "dare_attn_paged"]


@pytest.mark.parametrize("name", NAMES)
def test_null_context_is_refused(name):
    import ctypes
    f = getattr(binding.load(), name)
    args = [0 if t in (ctypes.c_int, ctypes.c_float, ctypes.c_double) else None for t in f.argtypes]
    assert f(*args) == -1


class _Ctx:
    import ctypes
    handle = ctypes.c_void_p(0)


@pytest.fixture
def no_gpu(monkeypatch):
    """The binding's own checks come before anything touches a device: run them on host tensors."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_marshal", binding._NoNative)
    monkeypatch.setattr(binding, "_raw", lambda stream, device: 0)


def _bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def _i(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def test_binding_refuses_shapes_that_do_not_belong_together(no_gpu):
    q, pages, table, lens = _bf(2, 1, 4, 64), _bf(5, 2, 16, 64), _i(2, 3), _i(2)
    for bad in (dict(v_pages=_bf(5, 2, 32, 64)), dict(kv_lens=_i(3)), dict(block_table=_i(1, 3)), dict(out=_bf(2, 1, 4, 128)),
                dict(lse=torch.zeros(2, 1, 4)), dict(k_pages=_bf(5, 2, 16, 128), v_pages=_bf(5, 2, 16, 128))):
        kw = dict(k_pages=pages, v_pages=pages, block_table=table, kv_lens=lens)
        kw.update(bad)
        with pytest.raises(ValueError, match="expected shape"):
            binding.dare_attn_paged(_Ctx, q, **kw)
    qkv, rope = _bf(6, 8 * 64), torch.zeros(10, 32, 2)
    for bad in (dict(seq_ids=_i(5)), dict(positions=_i(7)), dict(q_weight=_bf(128)), dict(k_weight=_bf(32)), dict(q_out=_bf(6, 3, 64)),
                dict(v_pages=_bf(4, 2, 16, 64)), dict(rope_table=torch.zeros(10, 64, 2))):
        kw = dict(seq_ids=_i(6), positions=_i(6), block_table=table, k_pages=pages, v_pages=pages, rope_table=rope)
        kw.update(bad)
        with pytest.raises(ValueError, match="expected shape"):
            binding.dare_paged_kv_append(_Ctx, qkv, **kw)
    with pytest.raises(ValueError, match="do not hold"):
        binding.dare_paged_kv_append(_Ctx, _bf(6, 4 * 64), _i(6), _i(6), table, pages, pages, rope)
    with pytest.raises(ValueError, match="do not hold"):
        binding.dare_qk_norm_rope(_Ctx, _bf(6, 8 * 64 + 8), _i(6), rope, 2)
    with pytest.raises(ValueError, match="expected shape"):
        binding.dare_qk_norm_rope(_Ctx, qkv, _i(5), rope, 2)
    with pytest.raises(ValueError, match="expected shape"):
        binding.dare_qk_norm_rope_backward(_Ctx, qkv, _i(6), rope, _bf(6, 4, 64), _bf(6, 2, 64), _bf(6, 1, 64))


def test_binding_refuses_host_tensors_and_other_types(no_gpu):
    q, pages = _bf(2, 1, 4, 64), _bf(5, 2, 16, 64)
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.dare_attn_paged(_Ctx, q, pages, pages, _i(2, 3), _i(2))
