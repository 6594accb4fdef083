"""CPU-side checks of the layers with 4-bit weights: the packed layout, and what the entry points refuse."""
import ctypes as ct

import numpy as np
import pytest
import torch

from packed_reference import code_at
from paper_2002_10711_b200 import binding, layer

BF16, FP16, FLOAT, INT8 = binding.BF16, binding.FP16, binding.FLOAT, binding.INT8


@pytest.mark.parametrize("K,C,group", [(1, 1, 32), (16, 128, 128), (17, 129, 64), (40, 300, 32), (33, 257, 384)])
def test_layout_and_round_trip(K, C, group):
    rng = np.random.default_rng(K * 1000 + C)
    q = torch.from_numpy(rng.integers(0, 16, (K, C), dtype=np.uint8))
    groups = -(-C // group)
    s = torch.rand(K, groups).to(torch.bfloat16)
    z = torch.from_numpy(rng.integers(0, 16, (K, groups), dtype=np.uint8))
    w = layer.pack_w4(q, s, z, group)
    assert w.codes.numel() == binding.packed_code_bytes(K, C)
    assert w.scales.numel() == w.zeros.numel() == binding.packed_scale_count(K, C, group)
    codes = w.codes.numpy()
    for k in {0, K - 1, K // 2}:
        for c in range(C):
            assert code_at(codes, k, c) == q[k, c]
    assert w.scales[K // 16 if K % 16 else K // 16 - 1, groups - 1, (K - 1) % 16] == s[K - 1, groups - 1]
    q2, s2, z2 = layer.unpack_w4(w)
    assert torch.equal(q, q2) and torch.equal(s, s2) and torch.equal(z, z2)


def test_pack_a_batch():
    q = torch.randint(0, 16, (3, 20, 70))
    s = torch.rand(3, 20, 3).half()
    w = layer.pack_w4(q, s, None, 32)
    assert w.codes.shape == (3, 2, 1, 16, 4, 16) and w.scales.shape == (3, 2, 3, 16) and w.zeros is None
    one = layer.pack_w4(q[1], s[1], None, 32)
    assert torch.equal(w.codes[1], one.codes) and torch.equal(w.scales[1], one.scales)


def test_pack_refuses():
    q, s = torch.zeros(4, 40, dtype=torch.uint8), torch.ones(4, 2).half()
    layer.pack_w4(q, s, None, 32)
    for bad in ((q, s[:, :1], None, 32), (q, s.float(), None, 32), (q + 16, s, None, 32),
                (q, s, torch.full((4, 2), 16), 32), (q, s, torch.zeros(4, 1), 32)):
        with pytest.raises(ValueError):
            layer.pack_w4(*bad)


def test_sizes():
    assert binding.packed_code_bytes(10, 512) == 1024 * 4
    assert binding.packed_scale_count(10, 512, 32) == 16 * 16
    assert binding.packed_scale_count(17, 513, 512) == 2 * 2 * 16
    for K, C, group in ((0, 8, 32), (8, 0, 32), (8, 8, 16), (8, 8, 96), (8, 8, 0), (8, 8, 192), (-1, 8, 32),
                        (1 << 25, 8, 32)):
        assert binding.packed_scale_count(K, C, group) == 0
    assert binding.packed_code_bytes(1 << 24, 1 << 24) == (1 << 20) * (1 << 17) * 1024   # no 32-bit product


def _packed(K=32, C=256, group=128, scale=BF16, codes=16, scales=32, zeros=None):
    return binding.packed(K, C, group, scale, codes, scales, zeros)


def _code(fn, *a, **kw):
    with pytest.raises(binding.WinoError) as e:
        fn(*a, stream=0, **kw)
    return e.value.code


def test_quantize_refuses():
    go = lambda w, x=64, t=FLOAT, stride=256, v=None: _code(binding.quantize_weights, w, x, t, stride, v)  # noqa: E731
    for bad in (_packed(K=0), _packed(C=0), _packed(group=48), _packed(scale=FLOAT), _packed(scale=INT8),
                _packed(codes=None), _packed(scales=None), _packed(K=(1 << 24) + 1)):
        assert go(bad) == binding.ERR_INVALID
    for bad in (_packed(codes=17), _packed(scales=24), _packed(zeros=8)):
        assert go(bad) == binding.ERR_ALIGNMENT
    assert go(_packed(), None) == binding.ERR_INVALID
    assert go(_packed(), t=INT8) == binding.ERR_INVALID
    assert go(_packed(), stride=255) == binding.ERR_INVALID
    assert go(_packed(), 66) == binding.ERR_ALIGNMENT
    assert go(_packed(), v=66) == binding.ERR_ALIGNMENT
    assert binding._lib.wino_quantize_weights(None, 64, FLOAT, 256, None, None) == binding.ERR_INVALID


def test_linear_refuses():
    def go(M=2, xt=BF16, yt=BF16, xs=256, ys=32, w=None, x=64, b=None, y=96, **kw):
        return _code(binding.linear_forward, M, xt, yt, xs, ys, w or _packed(), x, b, y, **kw)
    assert go(M=-1) == binding.ERR_INVALID
    assert go(xt=4) == go(yt=-1) == binding.ERR_INVALID
    assert go(xs=255) == go(ys=31) == go(xs=-256) == binding.ERR_INVALID
    assert go(x=None) == go(y=None) == binding.ERR_INVALID
    assert go(w=_packed(group=31)) == binding.ERR_INVALID
    assert go(w=_packed(codes=8)) == binding.ERR_ALIGNMENT
    assert go(x=65) == go(y=97) == go(b=66) == binding.ERR_ALIGNMENT
    assert go(xt=INT8, q_x=dict(scale=0.0)) == go(xt=INT8, q_x=dict(scale=float("nan"))) == binding.ERR_INVALID
    assert go(xt=INT8, q_x=dict(scale=1.0, zero_point=128)) == binding.ERR_INVALID
    assert go(yt=INT8, q_Y=dict(scale=1.0, qmin=-129)) == binding.ERR_INVALID
    assert binding._lib.wino_linear_forward(None, 64, None, 96, None) == binding.ERR_INVALID
    # no rows: nothing to do, nothing looked at
    binding.linear_forward(0, BF16, BF16, 256, 32, _packed(), None, None, None, stream=0)


def _desc(T=2, D=256, I=64, E=8, k=2, dtype=BF16, xs=256, ys=256, gate=None, up=None, down=None, normalize=True):
    g = dict(K=I, C=D)
    return binding.experts_desc(T, D, I, E, k, dtype, xs, ys, gate or _packed(**g), up or _packed(**g),
                                down or _packed(K=D, C=I), normalize)


def test_experts_refuses():
    def go(d, x=64, r=64, rb=None, y=64, ids=64, w=64, ws=64):
        return _code(binding.experts_forward, d, x, r, rb, y, ids, w, ws)
    for bad in (_desc(T=-1), _desc(D=0), _desc(I=0), _desc(E=0), _desc(k=0), _desc(k=9), _desc(dtype=INT8),
                _desc(xs=255), _desc(ys=255), _desc(gate=_packed(K=65, C=256)), _desc(up=_packed(K=64, C=255)),
                _desc(down=_packed(K=256, C=65)), _desc(up=_packed(K=64, C=256, group=64)),
                _desc(up=_packed(K=64, C=256, zeros=64)), _desc(up=_packed(K=64, C=256, scale=FP16))):
        assert go(bad) == binding.ERR_INVALID
    assert go(_desc(E=513)) == go(_desc(E=64, k=17)) == binding.ERR_UNSUPPORTED
    for kw in (dict(x=None), dict(r=None), dict(y=None), dict(ids=None), dict(w=None)):
        assert go(_desc(), **kw) == binding.ERR_INVALID
    assert go(_desc(), ws=None) == binding.ERR_WORKSPACE
    for kw in (dict(x=65), dict(r=65), dict(y=65), dict(ids=66), dict(w=66), dict(rb=66), dict(ws=72)):
        assert go(_desc(), **kw) == binding.ERR_ALIGNMENT
    assert binding._lib.wino_experts_workspace_bytes(None) == 0
    assert binding.experts_workspace_bytes(_desc(E=513)) == 0
    assert binding.experts_workspace_bytes(_desc(T=3, I=60, k=2)) == 3 * 2 * 64 * 2 * 2
    # more tokens than go through at once need no more
    assert binding.experts_workspace_bytes(_desc(T=64)) == binding.experts_workspace_bytes(_desc(T=100000))
    binding.experts_forward(_desc(T=0), None, None, None, None, None, None, None, stream=0)


def test_tensor_functions_refuse_without_a_gpu():
    w = layer.pack_w4(torch.zeros(4, 40, dtype=torch.uint8), torch.ones(4, 2).half(), None, 32)
    with pytest.raises(TypeError):
        layer.linear_w4([1.0], w)
    with pytest.raises(TypeError):
        layer.linear_w4(torch.zeros(1, 40), w.codes)
    with pytest.raises(ValueError):       # not on a GPU
        layer.linear_w4(torch.zeros(1, 40), w)
    with pytest.raises(ValueError):
        layer.quantize_w4(torch.zeros(4, 40), 32)
    with pytest.raises(TypeError):
        layer.quantize_w4(None)
    with pytest.raises(ValueError):
        layer.experts_w4(torch.zeros(1, 40), torch.zeros(2, 40), w, w, w, 1)


def test_tangents_are_refused():
    """Dual tensors of forward-mode derivatives: the result would have no tangent."""
    w = layer.pack_w4(torch.zeros(4, 40, dtype=torch.uint8), torch.ones(4, 2).half(), None, 32)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(w.scales, torch.ones_like(w.scales))
        with pytest.raises(ValueError, match="tangent"):
            layer.linear_w4(torch.zeros(1, 40), w._replace(scales=dual))
        router = torch.autograd.forward_ad.make_dual(torch.zeros(2, 40), torch.ones(2, 40))
        with pytest.raises(ValueError, match="tangent"):
            layer.experts_w4(torch.zeros(1, 40), router, w, w, w, 1)
        with torch.no_grad(), pytest.raises(ValueError, match="tangent"):      # which does not end forward mode
            layer.linear_w4(torch.zeros(1, 40), w._replace(scales=dual))


def test_pending_negations_are_refused():
    """Views whose elements torch negates when they are read (imaginary parts of conjugates)."""
    q, s, z = torch.zeros(4, 40, dtype=torch.uint8), torch.ones(4, 2).half(), torch.zeros(4, 2, dtype=torch.uint8)
    w = layer.pack_w4(q, s, z, 32)
    x, neg = torch.zeros(1, 40), torch._neg_view
    for bad in (w._replace(scales=neg(w.scales)), w._replace(zeros=neg(w.zeros)), w._replace(codes=neg(w.codes))):
        with pytest.raises(ValueError, match="resolve_neg"):
            layer.linear_w4(x, bad)
    with pytest.raises(ValueError, match="resolve_neg"):
        layer.experts_w4(x, neg(torch.zeros(2, 40)), w, w, w, 1)


def test_pack_takes_whole_numbers_only():
    q, s = torch.full((4, 40), 3), torch.ones(4, 2).half()
    want = layer.pack_w4(q, s, torch.full((4, 2), 7), 32)
    got = layer.pack_w4(q.float(), s, torch.full((4, 2), 7.0), 32)
    assert all(torch.equal(u, v) for u, v in zip(want[:3], got[:3]))
    nan = torch.full((4, 2), float("nan"))
    for bad in ((q + 0.5, s, None), (q.float().index_fill(1, torch.tensor([7]), float("nan")), s, None), (q, s, torch.full((4, 2), 6.75)),
                (q, s, nan), (q - 4, s, None), (q + 253, s, None), (q * float("inf"), s, None)):
        with pytest.raises(ValueError):
            layer.pack_w4(*bad, 32)
