"""Layers with 4-bit weights on the GPU, against plain references in 64 bits."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from paper_2002_10711_b200 import binding, layer

pytestmark = pytest.mark.gpu
F32, BF, HF, I8 = torch.float32, torch.bfloat16, torch.float16, torch.int8


def _on_gpu(w):
    return layer.W4(*(v.cuda() if isinstance(v, torch.Tensor) else v for v in w))


def _weights(rng, K, C, group, scale_dtype=BF, zeros=False, batch=()):
    q, s, z = ref.random_packed(rng, K, C, group, scale_dtype, zeros, batch)
    return _on_gpu(layer.pack_w4(q, s, z, group)), ref.matrix(q, s, z, group)


def _inputs(rng, shape, dtype):
    if dtype == I8:
        return torch.from_numpy(rng.integers(-128, 128, shape, dtype=np.int8))
    return torch.from_numpy(rng.normal(0, 1, shape)).to(dtype)


def _check(y, want, bound, dtype):
    got = y.double().cpu()
    tol = bound + ref.half_step(dtype) * (want.abs() + bound)
    assert torch.isfinite(got).all()
    worst = ((got - want).abs() / tol.clamp_min(1e-300)).max() if want.numel() else 0.0
    assert worst <= 1.0, f"{float(worst)} times the bound"


def _linear_case(M, C, K, group, dtype, zeros=False, bias=False, scale_dtype=BF, seed=0):
    rng = np.random.default_rng(seed + M * 7 + C * 3 + K)
    w, W = _weights(rng, K, C, group, scale_dtype, zeros)
    x = _inputs(rng, (M, C), dtype)
    b = torch.from_numpy(rng.normal(0, 1, K)).float() if bias else None
    q_x = dict(scale=0.03125, zero_point=int(rng.integers(-128, 128))) if dtype == I8 else None
    y = layer.linear_w4(x.cuda(), w, None if b is None else b.cuda(), q_x)
    xd = x.double() if q_x is None else (x.double() - q_x["zero_point"]) * q_x["scale"]
    want, bound = ref.linear(xd, W, b, group, 3 if dtype == F32 else 1)
    out = F32 if dtype == I8 else dtype
    assert y.dtype == out and y.shape == (M, K)
    _check(y, want, bound, out)


@pytest.mark.parametrize("dtype", [BF, HF, F32, I8])
@pytest.mark.parametrize("M,C,K,group,zeros,bias", [
    (1, 1, 1, 32, False, False),
    (1, 128, 16, 128, False, True),
    (1, 512, 10, 32, False, True),
    (1, 1000, 33, 64, True, False),
    (2, 127, 17, 32, True, True),
    (3, 136, 130, 64, False, False),
    (5, 2000, 101, 32, True, True),
    (8, 1024, 64, 128, True, False),
    (9, 1160, 48, 128, False, True),
    (16, 384, 256, 256, True, False),
    (17, 500, 40, 64, False, False),
    (33, 700, 129, 384, True, True),
    (64, 256, 96, 128, False, False),
    (70, 300, 272, 1024, True, True),
    (129, 640, 128, 128, True, False),
    (300, 72, 50, 32, False, True),
])
def test_linear(M, C, K, group, zeros, bias, dtype):
    _linear_case(M, C, K, group, dtype, zeros, bias, HF if K % 2 else BF)


@pytest.mark.parametrize("dtype", [BF, I8])
@pytest.mark.parametrize("M,C,K", [(1, 8192, 4096), (1, 16384, 256), (4, 4096, 2048), (24, 4096, 1040), (64, 2048, 2064)])
def test_linear_large(M, C, K, dtype):
    _linear_case(M, C, K, 128, dtype, True)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("M,C,K,group,zeros,bias", [
    (13, 8200, 6200, 128, True, True),          # one pass of 16 rows, sizes that fill no tile
    (16, 6184, 8201, 64, False, False),
    (9, 16384, 3200, 16384, True, False),       # a scale for each output
    (20, 3336, 3100, 32, True, True),
    (32, 4096, 2561, 128, False, True),
    (40, 2568, 2700, 256, True, False),
    (64, 2048, 2600, 128, False, False),
    (64, 1032, 5000, 32, True, True),
    (65, 1160, 3500, 384, True, True),
    (130, 904, 2500, 64, False, True),
    (300, 128, 8300, 128, True, False),         # a single chunk of inputs
    (1000, 72, 4500, 128, False, True),
])
def test_linear_many_rows(M, C, K, group, zeros, bias, dtype):
    assert -(-M // 16) * K * C >= (50e6 if M <= 16 else 20e6)      # sizes that the tcgen05 kernel takes
    _linear_case(M, C, K, group, dtype, zeros, bias, HF if K % 2 else BF)
    assert binding.direct_last_status() == 0


def test_linear_many_rows_strided_and_infinite():
    rng = np.random.default_rng(31)
    M, C, K, group = 70, 1160, 3600, 128
    w, W = _weights(rng, K, C, group, BF, True)
    base = _inputs(rng, (M + 1, C + 24), BF).cuda()
    x = base[1:, 8:8 + C]                                 # rows on 16-byte boundaries inside a larger buffer
    room = torch.full((M, K + 9), 7.0, dtype=BF, device="cuda")
    layer.linear_w4(x, w, out=room[:, 5:5 + K])
    assert (room[:, :5] == 7).all() and (room[:, 5 + K:] == 7).all()
    want, bound = ref.linear(x.double().cpu(), W, None, group)
    _check(room[:, 5:5 + K], want, bound, BF)
    clean = room[:, 5:5 + K].cpu()
    bad = x.clone()
    bad[3, 7], bad[69, 1159], bad[64, 0] = float("nan"), float("inf"), float("-inf")
    y = layer.linear_w4(bad, w).cpu()
    rest = [m for m in range(M) if m not in (3, 64, 69)]
    assert torch.equal(y[rest], clean[rest])
    want = bad.double().cpu() @ W.T
    for m in (3, 64, 69):
        assert torch.equal(torch.isnan(y[m]), torch.isnan(want[m]))
        fine = ~torch.isnan(want[m])
        assert (torch.sign(y[m].double())[fine] == torch.sign(want[m])[fine]).all()
    # unaligned rows of the same values go another way to the same place
    odd = base.flatten()[1:1 + M * C].view(M, C).clone()
    shifted = torch.empty(M * C + 1, dtype=BF, device="cuda")[1:].view(M, C)
    shifted.copy_(odd)
    want, bound = ref.linear(odd.double().cpu(), W, None, group)
    _check(layer.linear_w4(shifted, w), want, bound, BF)
    _check(layer.linear_w4(odd, w), want, bound, BF)


@pytest.mark.parametrize("M", [1, 3, 20, 150])
@pytest.mark.parametrize("dtype", [BF, HF, F32, I8])
def test_linear_strides_and_alignment(M, dtype):
    # rows of x that start anywhere, rows of y inside a larger buffer whose other elements stay
    rng = np.random.default_rng(M)
    C, K, group = 203, 70, 32
    w, W = _weights(rng, K, C, group, BF, True)
    q_x = dict(scale=0.5, zero_point=3) if dtype == I8 else None
    for offset, stride in ((0, C), (1, C + 1), (3, 2 * C), (8, 256), (2, 208)):
        base = _inputs(rng, (offset + M * stride,), dtype).cuda()
        x = base[offset:].as_strided((M, C), (stride, 1))
        out_dtype = F32 if dtype == I8 else dtype
        room = torch.full((M, K + 9), 7.0, dtype=out_dtype, device="cuda")
        y = layer.linear_w4(x, w, None, q_x, out=room[:, 5:5 + K])
        assert y.data_ptr() == room[:, 5:].data_ptr()
        assert (room[:, :5] == 7).all() and (room[:, 5 + K:] == 7).all()
        xd = x.double().cpu() if q_x is None else (x.double().cpu() - 3) * 0.5
        want, bound = ref.linear(xd, W, None, group, 3 if dtype == F32 else 1)
        _check(y, want, bound, out_dtype)


@pytest.mark.parametrize("shape", [(40,), (2, 3, 40), (0, 40), (4, 0, 40)])
def test_linear_shapes(shape):
    rng = np.random.default_rng(1)
    w, W = _weights(rng, 24, 40, 32)
    x = _inputs(rng, shape, BF)
    y = layer.linear_w4(x.cuda(), w)
    assert y.shape == (*shape[:-1], 24)
    want, bound = ref.linear(x.double().reshape(-1, 40), W, None, 32)
    _check(y.reshape(-1, 24), want, bound, BF)


def test_linear_transposed_input_is_copied():
    rng = np.random.default_rng(2)
    w, W = _weights(rng, 24, 40, 32)
    x = _inputs(rng, (40, 6), BF).cuda().T
    want, bound = ref.linear(x.double().cpu(), W, None, 32)
    _check(layer.linear_w4(x, w), want, bound, BF)


@pytest.mark.parametrize("x_dtype", [BF, I8])
def test_linear_to_other_types(x_dtype):
    rng = np.random.default_rng(3)
    M, C, K = 5, 260, 40
    w, W = _weights(rng, K, C, 128)
    x = _inputs(rng, (M, C), x_dtype)
    q_x = dict(scale=0.02, zero_point=-5) if x_dtype == I8 else None
    xd = x.double() if q_x is None else (x.double() + 5) * np.float64(np.float32(0.02))
    b = torch.from_numpy(rng.normal(0, 1, K)).float()
    want, bound = ref.linear(xd, W, b, 128)
    for dtype in (F32, BF, HF):
        _check(layer.linear_w4(x.cuda(), w, b.cuda(), q_x, out_dtype=dtype), want, bound, dtype)
    # int8 codes: the quantizer of the real value, up to one step where the value is next to a border
    q_Y = dict(scale=0.03, zero_point=4, qmin=-100, qmax=90)
    got = layer.linear_w4(x.cuda(), w, b.cuda(), q_x, q_Y).cpu().double()
    assert got.min() >= -100 and got.max() <= 90
    v = want / np.float64(np.float32(0.03))
    code = (torch.round(v) + 4).clamp(-100, 90)
    near = (v - torch.floor(v) - 0.5).abs() < bound / 0.03 + 4 * ref.U * v.abs()
    assert (got == code)[~near].all() and ((got - code).abs() <= 1).all()
    assert (~near).float().mean() > 0.9 and got.unique().numel() > 50


def test_linear_rows_do_not_mix_and_infinities_stay():
    rng = np.random.default_rng(4)
    M, C, K = 6, 300, 40
    w, W = _weights(rng, K, C, 64)
    for dtype in (BF, HF, F32):
        x = _inputs(rng, (M, C), dtype)
        clean = layer.linear_w4(x.cuda(), w).cpu()
        bad = x.clone()
        bad[1, 7], bad[3, 299], bad[4, 0] = float("nan"), float("inf"), float("-inf")
        y = layer.linear_w4(bad.cuda(), w).cpu()
        for m in (0, 2, 5):
            assert torch.equal(y[m], clean[m])
        want = bad.double() @ W.T          # inf * 0 is NaN there as here
        for m in (1, 3, 4):
            assert torch.equal(torch.isnan(y[m]), torch.isnan(want[m]))
            fine = ~torch.isnan(want[m])
            assert (torch.sign(y[m].double())[fine] == torch.sign(want[m])[fine]).all()


def test_linear_f32_extremes_are_exact():
    # one input at a time: its product with the weight, exactly, over the range of 32-bit floats
    C = 64
    q = torch.randint(0, 16, (16, C), generator=torch.Generator().manual_seed(0))
    w = _on_gpu(layer.pack_w4(q, torch.ones(16, 1).bfloat16(), None, 128))
    values = [1.0 + 2.0 ** -23, 3.14159274, -1e30, 1e-30, 2.0 ** -100 * (1 + 2.0 ** -20), 1.7e37, 16777215.0]
    x = torch.zeros(len(values), C)
    for m, v in enumerate(values):
        x[m, 5 * m] = v
    y = layer.linear_w4(x.cuda(), w).cpu()
    for m, v in enumerate(values):
        want = (q[:, 5 * m].double() - 8) * x[m, 5 * m].double()
        assert ((y[m].double() - want).abs() <= 2 * ref.U * want.abs()).all(), v


def test_linear_padding_of_codes_does_not_matter():
    rng = np.random.default_rng(5)
    M, C, K, group = 3, 200, 20, 64
    w, W = _weights(rng, K, C, group)
    x = _inputs(rng, (M, C), BF).cuda()
    y = layer.linear_w4(x, w)
    q, s, _ = layer.unpack_w4(w)
    full = torch.randint(0, 16, (32, 256), device="cuda", dtype=torch.uint8)
    full[:K, :C] = q
    noisy = layer.pack_w4(full, torch.ones(32, 4, device="cuda").bfloat16(), None, group)
    codes = layer.W4(noisy.codes, w.scales, None, K, C, group)
    assert torch.equal(layer.linear_w4(x, codes), y)


# --- quantizer ---------------------------------------------------------------------------
def _quantize_reference(w, group, symmetric, scale_dtype):
    """In 64 bits, the borders rounded as in 32: w's values and the scales have few enough bits that a quotient
    next to a border is on the same side in both (bf16 and fp16 weights)."""
    K, C = w.shape
    groups = -(-C // group)
    q, s_all = torch.empty(K, C, dtype=torch.uint8), torch.empty(K, groups, dtype=scale_dtype)
    z_all = torch.empty(K, groups, dtype=torch.uint8)
    for g in range(groups):
        part = w[:, g * group:(g + 1) * group].double()
        lo, hi = part.amin(1).clamp(max=0), part.amax(1).clamp(min=0)
        span = torch.maximum(hi, -lo) / 7 if symmetric else (hi - lo) / 15
        s = span.clamp(max=torch.finfo(scale_dtype).max).float().to(scale_dtype)
        d = s.double()
        safe = torch.where(d > 0, d, 1.0)
        z = torch.full_like(d, 8) if symmetric else torch.round(-lo / safe).clamp(0, 15)
        z = torch.where(d > 0, z, 8.0)
        code = torch.where((d > 0)[:, None], torch.round(part / safe[:, None]) + z[:, None], z[:, None]).clamp(0, 15)
        q[:, g * group:(g + 1) * group] = code.to(torch.uint8)
        s_all[:, g], z_all[:, g] = s, z.to(torch.uint8)
    return q, s_all, z_all


@pytest.mark.parametrize("scale_dtype", [BF, HF])
@pytest.mark.parametrize("symmetric", [True, False])
@pytest.mark.parametrize("K,C,group,dtype", [
    (1, 1, 32, BF), (16, 128, 128, BF), (33, 200, 32, HF), (20, 333, 64, BF), (50, 640, 256, HF), (7, 300, 384, BF),
    (5, 100, 1024, HF), (130, 1024, 128, HF)])
def test_quantize(K, C, group, dtype, symmetric, scale_dtype):
    gen = torch.Generator().manual_seed(K + C)
    w = torch.randn(K, C, generator=gen).to(dtype)
    if K > 4:
        w[1] = 0                                # a row of zeros
        w[2, : C // 2] = w[2, : C // 2].abs()   # groups without negative values
        w[3] *= 1e-6 if dtype == HF else 1e-30  # scales that are small, or nothing in fp16
        w[4] *= 3e4 if dtype == HF else 1e30    # scales beyond the largest of fp16
    got, values = layer.quantize_w4(w.cuda(), group, symmetric, scale_dtype, values=True)
    q, s, z = _quantize_reference(w, group, symmetric, scale_dtype)
    q2, s2, z2 = layer.unpack_w4(got)
    assert torch.equal(s2.cpu(), s)
    assert (z2 is None) == symmetric
    if not symmetric:
        assert torch.equal(z2.cpu(), z)
    assert torch.equal(q2.cpu(), q)
    want = ref.matrix(q, s, None if symmetric else z, group).to(dtype)
    assert torch.equal(values.cpu(), want)
    pad = got.scales.shape[-3] * 16 - K
    if pad:      # rows beyond K: scale 0, zero 8
        rest = got.scales.transpose(-1, -2).reshape(-1, got.scales.shape[-2])[K:]
        assert (rest == 0).all()


@pytest.mark.parametrize("symmetric", [True, False])
def test_quantize_f32_strided_and_batched(symmetric):
    gen = torch.Generator().manual_seed(9)
    base = torch.randn(3, 40, 170, generator=gen)
    w = base.cuda()[:, :, 3:160]
    got, values = layer.quantize_w4(w, 64, symmetric, HF, values=True)
    assert got.codes.shape == (3, 3, 2, 16, 4, 16) and values.shape == w.shape and values.dtype == F32
    for e in range(3):
        one, v = layer.quantize_w4(w[e], 64, symmetric, HF, values=True)   # a strided view
        assert torch.equal(one.codes, got.codes[e]) and torch.equal(one.scales, got.scales[e])
        assert torch.equal(v, values[e])
        # half a step of the scale, and what rounding the scale to 11 bits cuts off at the end of the range
        s = layer.unpack_w4(one)[1].double().repeat_interleave(64, -1)[:, : w.shape[2]]
        assert ((v.double() - w[e].double()).abs() <= s * (0.5 + 15 * 2.0 ** -10)).all()


# --- experts -----------------------------------------------------------------------------
def _experts_case(T, D, I, E, k, dtype, group=(64, 64), zeros=False, bias=True, normalize=True, seed=0, scale_dtype=BF):
    rng = np.random.default_rng(seed + T + D + I + E)
    gate, G = _weights(rng, I, D, group[0], scale_dtype, zeros, (E,))
    up, Up = _weights(rng, I, D, group[0], scale_dtype, zeros, (E,))
    down, Dn = _weights(rng, D, I, group[1], scale_dtype, zeros, (E,))
    x = _inputs(rng, (T, D), dtype)
    router = torch.from_numpy(rng.normal(0, 1, (E, D)) / np.sqrt(D)).to(dtype)
    b = torch.from_numpy(rng.normal(0, 0.5, E)).float() if bias else None
    y, ids, weights = layer.experts_w4(x.cuda(), router.cuda(), gate, up, down, k, None if b is None else b.cuda(), normalize)
    want, order, w, off = ref.experts(x.double(), router.double(), b, G, Up, Dn, group, k, normalize, dtype)
    assert torch.equal(ids.cpu().long(), order)
    size = float((x.double().abs() @ router.double().abs().T).max())
    assert ((weights.double().cpu() - w).abs() <= w * (2 * (D / 32 + 16) * ref.U * size + 16 * ref.U)).all()
    _check(y, want, off, dtype)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("T,D,I,E,k,group,zeros", [
    (1, 128, 128, 4, 2, (128, 128), False),
    (1, 300, 100, 8, 8, (32, 64), True),
    (2, 64, 16, 3, 1, (32, 32), False),
    (5, 200, 360, 12, 3, (64, 128), True),
    (9, 257, 130, 5, 2, (256, 32), False),
    (20, 128, 48, 2, 2, (128, 64), True),       # every expert takes every token
    (33, 96, 40, 40, 4, (32, 64), False),
    (64, 64, 32, 6, 2, (64, 32), False),
    (70, 136, 24, 9, 3, (128, 128), True),      # more than go through at once
])
def test_experts(T, D, I, E, k, group, zeros, dtype):
    _experts_case(T, D, I, E, k, dtype, group, zeros)


@pytest.mark.parametrize("T", [1, 12])
def test_experts_larger(T):
    _experts_case(T, 1024, 512, 64, 8, BF, (128, 128))


@pytest.mark.parametrize("E,k", [(512, 16), (33, 16), (16, 16), (1, 1)])
def test_experts_many_and_one(E, k):
    _experts_case(3, 72, 16, E, k, BF, (32, 32), normalize=False)


def test_experts_without_normalization_or_bias():
    _experts_case(6, 128, 64, 10, 3, HF, normalize=False, bias=False, scale_dtype=HF)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("at_once", [1, 2, 64])
def test_experts_inner_values(at_once, dtype):
    """5 h_a - 3 h_b of two inner values with one gate and up products 3 x and 5 x: nothing is left of them but what
    the way between the two products loses of each, at most 2^-17 (two bf16 rounded to nearest), for one or two
    tokens nothing."""
    T, D, I = 64, 32, 16
    code = lambda rows, **at: torch.tensor([[at.get(f"r{r}", {}).get(c, 8) for c in range(32)] for r in range(rows)])  # noqa: E731
    gate = code(I, r0={1: 9}, r1={1: 9})
    up = code(I, r0={0: 11}, r1={0: 13})
    down = torch.full((D, I), 8)
    down[:, 0], down[:, 1] = 13, 5
    pack = lambda q: _on_gpu(layer.pack_w4(q[None], torch.ones(1, q.shape[0], 1).to(BF), None, 32))  # noqa: E731
    rng = np.random.default_rng(41)
    x = torch.zeros(T, D, dtype=dtype)
    x[:, 0], x[:, 1] = _inputs(rng, (T,), dtype), _inputs(rng, (T,), dtype)
    router = torch.zeros(1, D, dtype=dtype, device="cuda")
    weights = pack(gate), pack(up), pack(down)
    parts = [layer.experts_w4(p, router, *weights, 1) for p in x.cuda().split(at_once)]
    y, w = torch.cat([p[0] for p in parts]), torch.cat([p[2] for p in parts])
    assert (w == 1).all()
    v, g = x[:, 0].double(), x[:, 1].double()
    h = (g * torch.sigmoid(g) * v).abs()
    # 5 |h_a| + 3 |h_b| = 30 |h|; the products silu * up are rounded to 2^-24 each, silu itself is common to both
    lost = 0.0 if at_once <= 2 else 2.0 ** -17
    bound = 30 * h * (lost + 2.0 ** -23) * (1 + 2.0 ** -20) * (1 + ref.half_step(dtype)) + torch.finfo(dtype).tiny * ref.half_step(dtype)
    assert (y.double().cpu().abs() <= bound[:, None]).all()
    assert (y != 0).any()


def _small_layer(rng, E=6, D=64, I=32, dtype=BF):
    gate, _ = _weights(rng, I, D, 32, batch=(E,))
    up, _ = _weights(rng, I, D, 32, batch=(E,))
    down, _ = _weights(rng, D, I, 32, batch=(E,))
    return gate, up, down


def test_experts_ties_masks_and_nan():
    rng = np.random.default_rng(11)
    E, D = 6, 64
    gate, up, down = _small_layer(rng)
    x = _inputs(rng, (5, D), BF).cuda()
    router = torch.zeros(E, D, dtype=BF, device="cuda")
    # all logits equal: the lowest indices, equal weights
    y, ids, w = layer.experts_w4(x, router, gate, up, down, 3)
    assert (ids.cpu() == torch.tensor([0, 1, 2])).all() and torch.allclose(w.cpu(), torch.full((5, 3), 1 / 3))
    # experts taken out, fewer left than top_k: the rest have weight 0 and add nothing
    b = torch.tensor([0.0, float("-inf"), 0.0, float("-inf"), float("-inf"), float("-inf")], device="cuda")
    y2, ids2, w2 = layer.experts_w4(x, router, gate, up, down, 3, b)
    assert (ids2.cpu() == torch.tensor([0, 2, 1])).all() and (w2.cpu() == torch.tensor([0.5, 0.5, 0.0])).all()
    y3, _, _ = layer.experts_w4(x, router, gate, up, down, 2, b)
    assert torch.equal(y2, y3)
    # nothing left at all
    y4, ids4, w4 = layer.experts_w4(x, router, gate, up, down, 2, torch.full((E,), float("-inf"), device="cuda"))
    assert (y4 == 0).all() and (w4 == 0).all() and (ids4.cpu() == torch.tensor([0, 1])).all()
    # a token of NaN, one whose logit is infinite: NaN for them, the others as before
    bad = x.clone()
    bad[2, 5] = float("nan")
    router[4, :] = 1.0
    bad[3, :] = 3e38
    y5, ids5, w5 = layer.experts_w4(x, router, gate, up, down, 2)
    y6, ids6, w6 = layer.experts_w4(bad, router, gate, up, down, 2)
    for t in (0, 1, 4):
        assert torch.equal(y5[t], y6[t]) and torch.equal(ids5[t], ids6[t]) and torch.equal(w5[t], w6[t])
    for t in (2, 3):
        assert torch.isnan(y6[t]).all() and torch.isnan(w6[t]).all() and (ids6[t].cpu() == torch.tensor([0, 1])).all()


def test_experts_shapes_strides_and_out():
    rng = np.random.default_rng(12)
    gate, up, down = _small_layer(rng, dtype=F32)
    router = torch.from_numpy(rng.normal(0, 1, (6, 64))).float().cuda()
    base = torch.from_numpy(rng.normal(0, 1, (7, 67))).float().cuda()
    x = base[:, 3:]
    room = torch.full((7, 70), 7.0, device="cuda")
    y, ids, w = layer.experts_w4(x, router, gate, up, down, 2, out=room[:, 1:65])
    y2, ids2, w2 = layer.experts_w4(x.contiguous(), router, gate, up, down, 2)
    assert torch.equal(y, y2) and torch.equal(ids, ids2) and torch.equal(w, w2)
    assert (room[:, 0] == 7).all() and (room[:, 65:] == 7).all()
    for shape in ((64,), (0, 64), (1, 7, 64)):
        z = x.contiguous().reshape(-1)[: int(np.prod(shape))].reshape(shape)
        y3, ids3, w3 = layer.experts_w4(z, router, gate, up, down, 2)
        assert y3.shape == shape and ids3.shape == (*shape[:-1], 2) and w3.shape == ids3.shape
        assert torch.equal(y3.reshape(-1, 64), y2[: y3.numel() // 64])


# --- calls -------------------------------------------------------------------------------
def test_same_bits_every_time_on_streams_and_in_graphs():
    rng = np.random.default_rng(13)
    E, D, I = 12, 256, 192
    gate, up, down = (_weights(rng, a, b, 64, batch=(E,))[0] for a, b in ((I, D), (I, D), (D, I)))
    head, _ = _weights(rng, 100, D, 64)
    router = torch.from_numpy(rng.normal(0, 1, (E, D)) / 16).to(BF).cuda()
    xs = [_inputs(rng, (M, D), BF).cuda() for M in (1, 4, 20)]
    wide, _ = _weights(rng, 40000, D, 64)                  # twenty rows: the tcgen05 kernel

    def run(x):
        y, ids, w = layer.experts_w4(x, router, gate, up, down, 4)
        return y, ids, w, layer.linear_w4(y, head), layer.linear_w4(y, wide)
    want = [run(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(5):                                    # calls that overlap: workspaces of their own
        for x, st in zip(xs, streams):
            with torch.cuda.stream(st):
                got.append(run(x))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        for u, v in zip(r, want[i % len(xs)]):
            assert torch.equal(u, v)
    # two captured graphs, replayed at the same time
    graphs, outs = [], []
    for x, st in zip(xs[:2], streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            outs.append(run(x))
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            for v in o:
                v.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for o, v in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, v))


def test_a_kernel_right_behind_the_one_that_makes_its_inputs():
    # quantize, multiply, quantize again into other weights: every launch reads what the one before wrote
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(3, 512, generator=gen, device="cuda").to(BF)
    ws = [torch.randn(512, 512, generator=gen, device="cuda").mul_(0.05).to(BF) for _ in range(6)]

    def chain(wait):
        v = x
        for w in ws:
            q = layer.quantize_w4(w, 64)
            if wait:
                torch.cuda.synchronize()
            v = layer.linear_w4(v, q)
            if wait:
                torch.cuda.synchronize()
        return v
    want = chain(True)
    for _ in range(10):
        assert torch.equal(chain(False), want)


@pytest.mark.parametrize("group", [1 << 24, (1 << 31) - 128])
def test_a_group_far_longer_than_a_row(group):
    """One scale an output, whatever the group's length: C + group passes 32 bits."""
    rng = np.random.default_rng(17)
    E, D, I, near = 3, 300, 260, 384
    for symmetric in (True, False):
        m = _inputs(rng, (40, D), BF).cuda()
        a, va = layer.quantize_w4(m, near, symmetric, values=True)
        b, vb = layer.quantize_w4(m, group, symmetric, values=True)
        assert b.group == group and all(torch.equal(u, v) for u, v in zip(a[:3], b[:3]) if u is not None) and torch.equal(va, vb)
        for M in (1, 20, 70):
            x = _inputs(rng, (M, D), BF).cuda()
            assert torch.equal(layer.linear_w4(x, a), layer.linear_w4(x, b))
    wide, _ = _weights(rng, 5000, D, near, zeros=True)
    x = _inputs(rng, (70, D), BF).cuda()                    # the tcgen05 kernel
    assert torch.equal(layer.linear_w4(x, wide), layer.linear_w4(x, wide._replace(group=group)))
    ws = [_weights(rng, *s, near, batch=(E,))[0] for s in ((I, D), (I, D), (D, I))]
    router = _inputs(rng, (E, D), BF).cuda()
    for T in (1, 9):
        x = _inputs(rng, (T, D), BF).cuda()
        for u, v in zip(layer.experts_w4(x, router, *ws, 2), layer.experts_w4(x, router, *(w._replace(group=group) for w in ws), 2)):
            assert torch.equal(u, v)


def test_dual_tensors_are_refused():
    fwd = torch.autograd.forward_ad
    rng = np.random.default_rng(18)
    w, _ = _weights(rng, 24, 64, 32)
    gate, up, down = _small_layer(rng)
    x, r = _inputs(rng, (2, 64), BF).cuda(), torch.zeros(6, 64, dtype=BF, device="cuda")
    bias, mask, out = torch.zeros(24, device="cuda"), torch.zeros(6, device="cuda"), torch.zeros(2, 24, dtype=BF, device="cuda")
    want, (want_e, _, _) = layer.linear_w4(x, w, bias), layer.experts_w4(x, r, gate, up, down, 2, mask)
    with fwd.dual_level():
        dual = lambda v: fwd.make_dual(v, torch.ones_like(v))  # noqa: E731
        for bad in (lambda: layer.linear_w4(dual(x), w), lambda: layer.linear_w4(x, w, dual(bias)),
                    lambda: layer.linear_w4(x, w, out=dual(out)), lambda: layer.experts_w4(dual(x), r, gate, up, down, 2),
                    lambda: layer.experts_w4(x, r, gate, up, down, 2, dual(mask))):
            with pytest.raises(ValueError, match="tangent"):
                bad()
        assert torch.equal(layer.linear_w4(fwd.unpack_dual(dual(x)).primal, w, bias), want)
    assert torch.equal(layer.linear_w4(x, w, bias), want)
    assert torch.equal(layer.experts_w4(x, r, gate, up, down, 2, mask)[0], want_e)


def test_pending_negations():
    rng = np.random.default_rng(19)
    w, _ = _weights(rng, 24, 64, 32)
    gate, up, down = _small_layer(rng)
    r = _inputs(rng, (6, 64), F32).cuda()
    z = torch.complex(_inputs(rng, (3, 64), F32), _inputs(rng, (3, 64), F32)).cuda()
    for x in (torch._neg_view(z.real.clone()), z.conj().imag, torch._neg_view(z.real.clone())[1]):
        assert x.is_neg()
        plain = x.resolve_neg().contiguous()
        assert torch.equal(layer.linear_w4(x, w), layer.linear_w4(plain, w))
        for u, v in zip(layer.experts_w4(x, r, gate, up, down, 2), layer.experts_w4(plain, r, gate, up, down, 2)):
            assert torch.equal(u, v)
    weight = torch._neg_view(_inputs(rng, (20, 64), BF).cuda())
    for u, v in zip(layer.quantize_w4(weight, 32, False), layer.quantize_w4(weight.resolve_neg(), 32, False)):
        assert torch.equal(u, v) if isinstance(u, torch.Tensor) else u == v
    x, neg = plain.clone(), torch._neg_view
    for bad in (lambda: layer.linear_w4(x, w, neg(torch.zeros(24, device="cuda"))),
                lambda: layer.linear_w4(x, w, out=neg(torch.zeros(24, device="cuda"))),
                lambda: layer.experts_w4(x, r, gate, up, down, 2, neg(torch.zeros(6, device="cuda")))):
        with pytest.raises(ValueError, match="resolve_neg"):
            bad()


def test_quantizer_fields_are_whole_numbers():
    rng = np.random.default_rng(20)
    w, _ = _weights(rng, 24, 64, 32)
    x = _inputs(rng, (3, 64), I8).cuda()
    for bad in (dict(q_x=dict(scale=0.1, zero_point=3.7)), dict(q_x=dict(scale=0.1, qmin=-0.5)),
                dict(q_x=dict(scale=0.1), q_Y=dict(scale=0.1, zero_point=-0.25)),
                dict(q_x=dict(scale=0.1), q_Y=dict(scale=0.1, qmax=99.5)), dict(q_x=dict(scale=0.1, zero_point=float("nan")))):
        with pytest.raises(ValueError):
            layer.linear_w4(x, w, **bad)
    want = layer.linear_w4(x, w, q_x=dict(scale=0.1, zero_point=3))
    for three in (3.0, np.int64(3), np.float32(3)):
        assert torch.equal(layer.linear_w4(x, w, q_x=dict(scale=0.1, zero_point=three)), want)


def test_other_threads_run_while_a_batch_is_quantized():
    """One launch an expert, and the queue holds about a thousand: a call that waits for room lets others run."""
    import sys
    import threading
    import time
    w = torch.randn(6000, 16, 64, device="cuda").to(BF)
    layer.quantize_w4(w[:2], 32)
    torch.cuda.synchronize()
    turns, over, interval = [0], threading.Event(), sys.getswitchinterval()

    def other():
        while not over.is_set():
            turns[0] += 1
            time.sleep(0)                  # hands the interpreter on by itself
    thread = threading.Thread(target=other)
    sys.setswitchinterval(30.0)            # nobody takes it from the caller
    try:
        thread.start()
        before = turns[0]
        got = layer.quantize_w4(w, 32)
        after = turns[0]
    finally:
        over.set()
        sys.setswitchinterval(interval)
        thread.join()
    assert after > before
    for e in (0, 2999, 5999):
        assert torch.equal(got.codes[e], layer.quantize_w4(w[e], 32).codes)


def test_refusals_on_the_gpu():
    rng = np.random.default_rng(14)
    w, _ = _weights(rng, 24, 40, 32)
    x = _inputs(rng, (2, 40), BF).cuda()
    z = torch.zeros
    for bad in (lambda: layer.linear_w4(x[:, :39], w), lambda: layer.linear_w4(x.double(), w),
                lambda: layer.linear_w4(x, w._replace(codes=w.codes.cpu())),
                lambda: layer.linear_w4(x, w._replace(scales=w.scales.float())),
                lambda: layer.linear_w4(x, w._replace(group=64)), lambda: layer.linear_w4(x, w._replace(K=40)),
                lambda: layer.linear_w4(x, w._replace(group=33)), lambda: layer.linear_w4(x, w._replace(K=-1)),
                lambda: layer.linear_w4(x, w._replace(zeros=z(3, dtype=torch.uint8, device="cuda"))),
                lambda: layer.linear_w4(x, w, z(23, device="cuda")), lambda: layer.linear_w4(x, w, z(24)),
                lambda: layer.linear_w4(x, w, z(24, dtype=BF, device="cuda")),
                lambda: layer.linear_w4(x, w, q_x=dict(scale=1.0)), lambda: layer.linear_w4(x.to(I8), w),
                lambda: layer.linear_w4(x, w, out_dtype=I8), lambda: layer.linear_w4(x, w, out_dtype=torch.float64),
                lambda: layer.linear_w4(x, w, out=z(2, 25, dtype=BF, device="cuda")),
                lambda: layer.linear_w4(x, w, out=z(2, 24, device="cuda")),
                lambda: layer.linear_w4(x, w, out=z(24, 2, dtype=BF, device="cuda").T),
                lambda: layer.linear_w4(x.float().requires_grad_(), w),
                lambda: layer.quantize_w4(x, 48), lambda: layer.quantize_w4(x, 32, True, F32),
                lambda: layer.quantize_w4(x.double(), 32), lambda: layer.quantize_w4(x[0], 32)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(binding.WinoError) as e:
        layer.linear_w4(x.to(I8), w, q_x=dict(scale=-1.0))
    assert e.value.code == binding.ERR_INVALID
    with torch.no_grad():
        layer.linear_w4(x.float().requires_grad_(), w)
    gate, up, down = _small_layer(rng)
    xe, r = _inputs(rng, (2, 64), BF).cuda(), z(6, 64, dtype=BF, device="cuda")
    layer.experts_w4(xe, r, gate, up, down, 2)
    for bad in (lambda: layer.experts_w4(xe, r, gate, up, gate, 2), lambda: layer.experts_w4(xe, r[:5], gate, up, down, 2),
                lambda: layer.experts_w4(xe, r.float(), gate, up, down, 2), lambda: layer.experts_w4(xe, r, gate, up, down, 7),
                lambda: layer.experts_w4(xe, r, gate, up, down, 0), lambda: layer.experts_w4(xe.float(), r, gate, up, down, 2),
                lambda: layer.experts_w4(xe, r, gate, up, down, 2, z(5, device="cuda")),
                lambda: layer.experts_w4(xe[:, :63], r, gate, up, down, 2)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("dtype,C,K", [(F32, 33, 3), (BF, 40, 17)])
def test_more_rows_than_a_grid_has_slices(dtype, C, K):
    """Each row's result depends on that row alone: the same bits as in a small call with the same rows."""
    rng = np.random.default_rng(C)
    w, _ = _weights(rng, K, C, 32)
    M = 524288 + 5
    few = _inputs(rng, (41, C), dtype).cuda()
    x = few[torch.arange(M, device="cuda") % 41]
    out = torch.full((M, K + 2), 7.0, dtype=dtype, device="cuda")
    layer.linear_w4(x, w, out=out[:, :K])
    want = layer.linear_w4(few.repeat(128, 1), w)          # rows enough for the same kernel
    assert torch.equal(out[:, :K], want[torch.arange(M, device="cuda") % 41])
    assert (out[:, K:] == 7).all()


def test_out_beside_x():
    """out and x as columns of one tensor; a shared byte is refused; autograd learns that out was written."""
    rng = np.random.default_rng(31)
    w, _ = _weights(rng, 24, 40, 32)
    both = torch.zeros(3, 72, dtype=BF, device="cuda")
    x, y, gap = both[:, 8:48], both[:, 48:72], both[:, :8].clone()
    x.copy_(_inputs(rng, (3, 40), BF))
    want, version = layer.linear_w4(x.clone(), w), both._version
    assert layer.linear_w4(x, w, out=y) is y and both._version == version + 1
    assert torch.equal(y, want) and torch.equal(both[:, :8], gap)
    flat = torch.zeros(400, dtype=BF, device="cuda")
    for bad in (lambda: layer.linear_w4(x, w, out=both[:, 47:71]), lambda: layer.linear_w4(x, w, out=both[:, :24]),
                lambda: layer.linear_w4(x, w, out=x[:, :24]),
                lambda: layer.linear_w4(flat[:120].view(3, 40), w, out=flat[119:191].view(3, 24)),
                lambda: layer.linear_w4(flat[71:191].view(3, 40), w, out=flat[:72].view(3, 24)),
                lambda: layer.linear_w4(x, w._replace(scales=w.scales.clone().requires_grad_()))):
        with pytest.raises(ValueError):
            bad()
    layer.linear_w4(flat[:120].view(3, 40), w, out=flat[120:192].view(3, 24))
    layer.linear_w4(flat[72:192].view(3, 40), w, out=flat[:72].view(3, 24))
    gate, up, down = _small_layer(rng)
    xe, r = _inputs(rng, (2, 64), BF).cuda(), torch.zeros(6, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        layer.experts_w4(xe, r, gate, up, down, 2, out=xe)


def test_out_beside_the_other_operands():
    """out between or next to weights, router and biases in one allocation is taken, a shared byte refused."""
    rng = np.random.default_rng(32)
    M, C, K = 3, 40, 24
    w, _ = _weights(rng, K, C, 32, zeros=True)
    x = _inputs(rng, (M, C), F32).cuda()
    bias = _inputs(rng, (K,), F32).cuda()
    want = layer.linear_w4(x, w, bias)
    rows = torch.zeros(M, 64, device="cuda")               # out in columns 0..23, the bias right behind or in a gap
    for at in (24, 40, 64 + 24, 2 * 64 + 24):
        flat = torch.zeros(M * 64 + K, device="cuda")
        b, out = flat[at:at + K], flat[:M * 64].view(M, 64)[:, :K]
        b.copy_(bias)
        layer.linear_w4(x, w, b, out=out)
        assert torch.equal(out, want) and torch.equal(b, bias)
    for at in (0, 1, 23, 41, 63, 64, 2 * 64 + 23):
        flat = torch.zeros(M * 64 + K, device="cuda")
        version = flat._version
        with pytest.raises(ValueError, match="overlap"):
            layer.linear_w4(x, w, flat[at:at + K], out=flat[:M * 64].view(M, 64)[:, :K])
        assert flat._version == version
    one = torch.zeros(K, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        layer.linear_w4(x[0], w, one, out=one)
    for v in (w.codes, w.scales, w.zeros):
        whole = torch.zeros(v.numel() * v.element_size() + 4 * M * K, dtype=torch.uint8, device="cuda")
        part = whole[:v.numel() * v.element_size()].view(v.dtype).view(v.shape)
        part.copy_(v)
        moved = layer.W4(*(part if u is v else u for u in w))
        behind = whole[part.numel() * part.element_size():].view(F32).view(M, K)
        assert torch.equal(layer.linear_w4(x, moved, bias, out=behind), want) and torch.equal(part, v)
        with pytest.raises(ValueError, match="overlap"):
            layer.linear_w4(x, moved, bias, out=whole[-4 * M * K - 4:-4].view(F32).view(M, K))
    E, D = 6, 64
    gate, up, down = _small_layer(rng)
    xe, both = _inputs(rng, (2, D), BF).cuda(), torch.zeros(E + 2, D, dtype=BF, device="cuda")
    both[:E].copy_(_inputs(rng, (E, D), BF))
    want, ids, weights = layer.experts_w4(xe, both[:E].clone(), gate, up, down, 2)
    y, ids2, weights2 = layer.experts_w4(xe, both[:E], gate, up, down, 2, out=both[E:])
    assert torch.equal(y, want) and torch.equal(ids, ids2) and torch.equal(weights, weights2)
    mask = torch.zeros(E, device="cuda")
    for bad in (lambda: layer.experts_w4(xe, both[:E], gate, up, down, 2, out=both[E - 1:E + 1]),
                lambda: layer.experts_w4(xe.float(), both[:E].float(), gate, up, down, 2, rows.view(-1)[:E], out=rows.view(-1)[:2 * D].view(2, D)),
                lambda: layer.experts_w4(xe, both[:E], gate, up, down, 2, mask, out=down.scales.view(-1)[:2 * D].view(2, D)),
                lambda: layer.experts_w4(xe, both[:E], gate, up, down, 2, mask, out=up.codes.view(-1)[-4 * D:].view(BF).view(2, D))):
        with pytest.raises(ValueError, match="overlap"):
            bad()


def test_out_between_rows_of_x():
    """Rows of x and of out at different strides in one tensor: taken where no byte is shared."""
    rng = np.random.default_rng(33)
    w, _ = _weights(rng, 40, 40, 32)
    rows = torch.zeros(10, 40, dtype=BF, device="cuda")
    for x, out in (((0, 9, 4), (1, 4, 1)), ((0, 9, 4), (5, 8, 1)), ((1, 4, 1), (0, 10, 4)), ((0, 10, 3), (1, 8, 2))):
        xs, outs = list(range(*x))[:3], list(range(*out))[:3]
        rows.copy_(_inputs(rng, (10, 40), BF))
        before, v, y = rows.clone(), rows[x[0]:x[1]:x[2]][:3], rows[out[0]:out[1]:out[2]][:3]
        if set(xs) & set(outs):
            with pytest.raises(ValueError, match="overlap"):
                layer.linear_w4(v, w, out=y)
            assert torch.equal(rows, before)
            continue
        layer.linear_w4(v, w, out=y)
        assert torch.equal(y, layer.linear_w4(before[xs], w))
        rest = [r for r in range(10) if r not in outs]
        assert torch.equal(rows[rest], before[rest])
    flat = torch.zeros(400, dtype=BF, device="cuda")
    with pytest.raises(ValueError, match="overlap"):       # their second rows are the same elements
        layer.linear_w4(flat[:200].view(2, 100)[:, :40], w, out=flat[40:160].view(2, 60)[:, :40])


def test_a_network_with_its_head():
    """The library's convolution, pooled int8 codes, the 4-bit classifier, and an experts layer on real values."""
    gen = torch.Generator().manual_seed(21)
    N, C, K = 4, 64, 128
    x = torch.randint(0, 100, (N, 8, 8, C), dtype=I8, generator=gen)
    wc = torch.randint(-60, 60, (K, 3, 3, C), dtype=I8, generator=gen)
    s_x, s_w, s_y = 1 / 32, 0.002, 0.25
    y = torch.empty(N, 8, 8, K, dtype=I8, device="cuda")
    binding.direct_conv_forward(N, C, 8, 8, K, 1, dict(scale=s_x), dict(scale=s_w), dict(scale=s_y, qmin=0), x.cuda(),
                                wc.cuda(), None, y)
    pooled = y.float().mean((1, 2)).round().to(I8)          # codes of scale s_y
    assert pooled.float().std() > 0
    weight = torch.randn(10, K, generator=gen).mul(0.1)
    head, values = layer.quantize_w4(weight.cuda(), 32, False, BF, values=True)
    bias = torch.randn(10, generator=gen)
    logits = layer.linear_w4(pooled, head, bias.cuda(), dict(scale=s_y))
    want, bound = ref.linear(pooled.cpu().double() * s_y, values.cpu().double(), bias, 32)
    # `values` are rounded to 32 bits, the product's own are not
    _check(logits, want, bound + ref.U * (pooled.cpu().double().abs() * s_y) @ values.cpu().double().abs().T, F32)
    E, I = 4, 64
    mats = [torch.randn(E, a, b, generator=gen).mul(0.1).cuda() for a, b in ((I, K), (I, K), (K, I))]
    packed = [layer.quantize_w4(m, 32, values=True) for m in mats]
    router = torch.randn(E, K, generator=gen).mul(0.1)
    feats = pooled.float() * s_y
    out, ids, w = layer.experts_w4(feats, router.cuda(), *(p[0] for p in packed), 2)
    want, order, _, off = ref.experts(feats.cpu().double(), router.double(), None, *(p[1].cpu().double() for p in packed),
                                      (32, 32), 2, True, F32)
    assert torch.equal(ids.cpu().long(), order)
    _check(out, want, off + 8 * ref.U * want.abs().max(), F32)


def test_latency_table_has_the_head():
    from paper_2002_10711_b200 import latency_table
    assert latency_table.head_latency(2, 64, 10, sets=2) > 0
