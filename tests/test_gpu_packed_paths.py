"""Layers with 4-bit weights on the GPU: the launch shapes that large and lopsided calls take, which kernel a call
takes, the quantizer of 32-bit weights bit by bit, and the C entry points called by address."""
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
    worst = ((got - want).abs() / tol.clamp_min(1e-300)).max()
    assert worst <= 1.0, f"{float(worst)} times the bound"


def _kernels(call):
    """Names and grids of the kernels that a call launches, from a captured graph's nodes."""
    driver = pytest.importorskip("cuda.bindings.driver")

    def ok(r):
        assert r[0] == driver.CUresult.CUDA_SUCCESS, r[0]
        return r[1:] if len(r) > 2 else r[1]
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        keep = call()
    raw = driver.CUgraph(graph.raw_cuda_graph())
    count = ok(driver.cuGraphGetNodes(raw))[1]
    nodes = ok(driver.cuGraphGetNodes(raw, count))[0]
    names = []
    for node in nodes[:count]:
        if ok(driver.cuGraphNodeGetType(node)) == driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            p = ok(driver.cuGraphKernelNodeGetParams(node))
            name = ok(driver.cuFuncGetName(p.func)) if int(p.func) else ok(driver.cuKernelGetName(p.kern))
            names.append((name.decode(), (p.gridDimX, p.gridDimY)))
    del keep
    return names


# --- which kernel ------------------------------------------------------------------------
@pytest.mark.parametrize("M,C,K,dtype,kernel", [
    (8, 8192, 8192, BF, "k_linear_rows"),           # eight rows stay with the warp MMAs
    (9, 8192, 6200, BF, "k_linear_tc"),
    (16, 6184, 8201, HF, "k_linear_tc"),
    (16, 4096, 4096, BF, "k_linear_rows"),          # little work
    (64, 2048, 2600, BF, "k_linear_tc"),
    (64, 2044, 2600, BF, "k_linear_rows"),          # rows that are not on 16-byte boundaries
    (64, 2048, 2600, F32, "k_linear_rows"),
    (64, 2048, 2600, I8, "k_linear_rows"),
])
def test_which_kernel_a_call_takes(M, C, K, dtype, kernel):
    rng = np.random.default_rng(M + C)
    w = layer.quantize_w4(torch.randn(K, C, device="cuda"))
    x = _inputs(rng, (M, C), dtype).cuda()
    q_x = dict(scale=0.1) if dtype == I8 else None
    names = _kernels(lambda: layer.linear_w4(x, w, None, q_x))
    assert len(names) == 1 and kernel in names[0][0], names


# --- clusters of eight that share the inputs -----------------------------------------------
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("M,C,K,group,zeros,bias", [
    (32, 16384, 1024, 128, False, True),
    (64, 2944, 1792, 128, True, False),         # 23 chunks: two or three a block
    (16, 32768, 1700, 64, True, True),
    (448, 2904, 250, 256, False, False),        # seven slices of rows, a last chunk of 88 inputs
    (31, 24000, 500, 32, False, True),
])
def test_linear_clusters_of_eight(M, C, K, group, zeros, bias, dtype):
    rng = np.random.default_rng(M + C + K)
    w, W = _weights(rng, K, C, group, HF if K % 4 else BF, zeros)
    x = _inputs(rng, (M, C), dtype)
    b = _inputs(rng, (K,), F32) if bias else None
    run = lambda: layer.linear_w4(x.cuda(), w, None if b is None else b.cuda())  # noqa: E731
    want, bound = ref.linear(x.double(), W, b, group)
    y = run()
    _check(y, want, bound, dtype)
    assert torch.equal(run(), y) and binding.direct_last_status() == 0
    xg, bg = x.cuda(), None if b is None else b.cuda()
    (name, grid), = _kernels(lambda: layer.linear_w4(xg, w, bg))
    assert "k_linear_tc" in name and grid[0] == 8 * -(-K // 128), (name, grid)


@pytest.mark.parametrize("M", [12, 40, 64])
def test_tcgen05_kernel_to_other_types(M):
    rng = np.random.default_rng(M)
    C, K, group = 2056, 3300 if M > 16 else 25000, 128
    w, W = _weights(rng, K, C, group, BF, True)
    x, b = _inputs(rng, (M, C), BF), _inputs(rng, (K,), F32)
    want, bound = ref.linear(x.double(), W, b, group)
    xg, bg = x.cuda(), b.cuda()
    assert "k_linear_tc" in _kernels(lambda: layer.linear_w4(xg, w, bg, out_dtype=F32))[0][0]
    for dtype in (F32, BF, HF):
        _check(layer.linear_w4(xg, w, bg, out_dtype=dtype), want, bound, dtype)
    s, zero, lo, hi = float(np.float32(0.03)), 4, -100, 90
    q_Y = dict(scale=s, zero_point=zero, qmin=lo, qmax=hi)
    room = torch.full((M, K + 6), 77, dtype=I8, device="cuda")
    got = layer.linear_w4(xg, w, bg, q_Y=q_Y, out=room[:, 3:3 + K]).cpu().double()
    assert (room[:, :3] == 77).all() and (room[:, 3 + K:] == 77).all()
    v = want / s
    code = (torch.round(v) + zero).clamp(lo, hi)
    # 1 / s_Y, the bias over s_Y and their sum are rounded to 32 bits each
    near = (v - torch.floor(v) - 0.5).abs() < bound / s + 4 * ref.U * (v.abs() + b.double().abs() / s)
    assert (got == code)[~near].all() and ((got - code).abs() <= 1).all()
    assert (~near).double().mean() > 0.9 and got.unique().numel() > 50


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("M,C,K,stride", [(64, 2043, 2600, 2048), (20, 3337, 3200, 3352), (3, 1021, 200, 1024)])
def test_rows_with_gaps(M, C, K, stride, dtype):
    """Rows of odd length on 16-byte boundaries: what stands between them is nobody's."""
    rng = np.random.default_rng(C)
    w, W = _weights(rng, K, C, 128, BF, True)
    base = torch.full((M, stride), float("nan"), dtype=dtype)
    base[:, :C] = _inputs(rng, (M, C), dtype)
    x = base.cuda()[:, :C]
    want, bound = ref.linear(base[:, :C].double(), W, None, 128)
    _check(layer.linear_w4(x, w), want, bound, dtype)
    assert ("k_linear_tc" if M > 8 else "k_linear_rows") in _kernels(lambda: layer.linear_w4(x, w))[0][0]
    assert torch.equal(layer.linear_w4(x.contiguous()[:3], w), layer.linear_w4(x[:3], w))


# --- experts -------------------------------------------------------------------------------
@pytest.mark.parametrize("T,D,I,E,k,dtype,bias", [
    (16, 256, 1024, 64, 8, BF, 0.0),        # 512 items of the gate and up products on 296 blocks
    (16, 256, 1024, 64, 8, HF, 6.0),        # some experts have all 16 tokens, eight at a time
    (64, 256, 1024, 64, 8, BF, 6.0),        # 16 at a time, some have 64
    (12, 264, 1600, 48, 6, F32, 6.0),
    (24, 136, 1536, 40, 6, BF, 6.0),
])
def test_experts_several_items_a_block(T, D, I, E, k, dtype, bias):
    rng = np.random.default_rng(T + I)
    group = (128, 64)
    gate, G = _weights(rng, I, D, group[0], BF, True, (E,))
    up, Up = _weights(rng, I, D, group[0], BF, True, (E,))
    down, Dn = _weights(rng, D, I, group[1], BF, False, (E,))
    x = _inputs(rng, (T, D), dtype)
    router = torch.from_numpy(rng.normal(0, 1, (E, D)) / np.sqrt(D)).to(dtype)
    b = torch.from_numpy(rng.normal(0, 0.5, E)).float()
    b[[1, E // 2, E - 1]] += bias
    y, ids, weights = layer.experts_w4(x.cuda(), router.cuda(), gate, up, down, k, b.cuda())
    want, order, w, off = ref.experts(x.double(), router.double(), b, G, Up, Dn, group, k, True, dtype)
    assert torch.equal(ids.cpu().long(), order)
    _check(y, want, off, dtype)
    tokens = torch.bincount(order.flatten(), minlength=E)
    at_once = 8 if T * k <= 6 * E or T <= 8 else 16
    items = int((tokens > 0).sum()) * -(-I // 128)               # (eight row tiles of 16 a block)
    assert items > 2 * torch.cuda.get_device_properties(0).multi_processor_count
    assert bias == 0 or (tokens > at_once).any()
    again = layer.experts_w4(x.cuda(), router.cuda(), gate, up, down, k, b.cuda())
    assert torch.equal(again[0], y)


# --- quantizer ---------------------------------------------------------------------------
def _quantize_32(w, group, symmetric, scale_dtype):
    """The documented rules step by step in 32-bit floats: codes, scales and zeros have to be the same bits."""
    K, C = w.shape
    groups = -(-C // group)
    p = torch.nn.functional.pad(w, (0, groups * group - C)).view(K, groups, group)
    lo, hi = p.amin(-1, keepdim=True).clamp(max=0), p.amax(-1, keepdim=True).clamp(min=0)
    span = torch.maximum(hi, -lo) / torch.tensor(7.0) if symmetric else (hi - lo) / torch.tensor(15.0)
    s = span.clamp(max=torch.finfo(scale_dtype).max).to(scale_dtype)
    f = s.float()
    z = torch.full_like(f, 8) if symmetric else torch.where(f > 0, torch.round(-lo / f).clamp(0, 15), 8.0)
    q = torch.where(f > 0, (torch.round(p / f) + z).clamp(0, 15), z)
    return q.view(K, -1)[:, :C].to(torch.uint8), s[..., 0], z[..., 0].to(torch.uint8), ((q - z) * f).view(K, -1)[:, :C]


@pytest.mark.parametrize("scale_dtype", [BF, HF])
@pytest.mark.parametrize("symmetric", [True, False])
@pytest.mark.parametrize("K,C,group", [(64, 512, 32), (100, 1024, 64), (33, 640, 128), (17, 768, 256), (16, 896, 1024),
                                       (40, 157, 64), (5, 1001, 32), (9, 500, 384)])
def test_quantize_32_bit_weights(K, C, group, symmetric, scale_dtype):
    gen = torch.Generator().manual_seed(K + C)
    w = torch.randn(K, C, generator=gen)
    w[1], w[2], w[3], w[4] = 0.0, w[2].abs(), w[3] * 1e-30, w[4] * 1e30
    w[0, ::7] = 0.5 * torch.round(w[0, ::7] * 4)             # quotients on borders among them
    got, values = layer.quantize_w4(w.cuda(), group, symmetric, scale_dtype, values=True)
    q, s, z, v = _quantize_32(w, group, symmetric, scale_dtype)
    q2, s2, z2 = layer.unpack_w4(got)
    assert torch.equal(s2.cpu(), s) and torch.equal(q2.cpu(), q) and torch.equal(values.cpu(), v)
    assert z2 is None if symmetric else torch.equal(z2.cpu(), z)


# --- by address ----------------------------------------------------------------------------
def test_c_entry_points():
    rng = np.random.default_rng(50)
    K, C, M, group = 40, 192, 5, 64
    codes = {F32: binding.FLOAT, BF: binding.BF16, HF: binding.FP16, I8: binding.INT8}
    stream = torch.cuda.Stream()
    weight = _inputs(rng, (K, C + 9), HF).cuda()[:, :C]
    like, values = layer.quantize_w4(weight, group, False, HF, values=True)
    mine = [torch.empty_like(v) for v in (like.codes, like.scales, like.zeros, values)]
    packed = binding.packed(K, C, group, codes[HF], *mine[:3])
    assert mine[0].numel() == binding.packed_code_bytes(K, C) and mine[1].numel() == binding.packed_scale_count(K, C, group)
    x = _inputs(rng, (M, C), I8).cuda()
    bias = _inputs(rng, (K,), F32).cuda()
    y = torch.full((M, K + 2), 9.0, dtype=BF, device="cuda")
    q_x = dict(scale=0.05, zero_point=-3)
    torch.cuda.synchronize()
    binding.quantize_weights(packed, weight, codes[HF], C + 9, mine[3], stream=stream)
    binding.linear_forward(M, codes[I8], codes[BF], C, K + 2, packed, x, bias, y, q_x, stream=stream)
    stream.synchronize()
    for u, v in zip(mine, (like.codes, like.scales, like.zeros, values)):
        assert torch.equal(u, v)
    assert torch.equal(y[:, :K], layer.linear_w4(x, like, bias, q_x, out_dtype=BF)) and (y[:, K:] == 9).all()
    T, D, I, E, k = 70, 64, 40, 5, 2                            # 64 tokens, then six more
    gate, up, down = (_weights(rng, *s, 32, batch=(E,))[0] for s in ((I, D), (I, D), (D, I)))
    x, router, mask = _inputs(rng, (T, D), BF).cuda(), _inputs(rng, (E, D), BF).cuda(), _inputs(rng, (E,), F32).cuda()
    out, ids, weights = torch.empty_like(x), torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    desc = binding.experts_desc(T, D, I, E, k, codes[BF], D, D, *(binding.packed(v.K, v.C, v.group, codes[BF], v.codes, v.scales)
                                                                  for v in (gate, up, down)), normalize=False)
    size = binding.experts_workspace_bytes(desc)
    ws = torch.full((size + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    binding.experts_forward(desc, x, router, mask, out, ids, weights, ws, stream=stream)
    stream.synchronize()
    want = layer.experts_w4(x, router, gate, up, down, k, mask, False)
    assert all(torch.equal(u, v) for u, v in zip((out, ids, weights), want))
    assert (ws[size:] == 0xAB).all()                            # no byte beyond what was asked for
    for few in (1, 2, 3):
        d = binding.experts_desc(few, D, I, E, k, codes[BF], D, D, desc.gate, desc.up, desc.down)
        ws.fill_(0xAB)
        size = binding.experts_workspace_bytes(d)
        binding.experts_forward(d, x, router, mask, out, ids, weights, ws)
        torch.cuda.synchronize()
        assert (ws[size:] == 0xAB).all()
        assert torch.equal(out[:few], layer.experts_w4(x[:few], router, gate, up, down, k, mask)[0])
