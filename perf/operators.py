"""Layers with 4-bit weights and group scales, as cases to be timed and compared.

A case is a dict of plain values with an "op":
  quantize  weights to 4-bit codes with one scale (and zero point) per group of inputs, and the
            values that the codes stand for (layer.quantize_w4)
  linear    y = x W^T + b for one to some hundred rows of x (layer.linear_w4)
  experts   a mixture-of-experts layer for a few tokens: router, the chosen experts' gate, up and
            down products, weighted sum (layer.experts_w4)

Packed weights of K outputs and C inputs, both rounded up (K to 16, C to 128), in groups of G
inputs: `codes`, uint8 [K/16][C/128][16][4][16], holds the 32 codes of row 16 a + r and of inputs
128 b + 32 i + 8 t + e (i = 0..3, e = 0..7) in the 16 bytes at [a][b][r][t]: 32-bit word i, with
the code of e in nibble e / 2 (e even) or 4 + e / 2 (e odd).  `scales` and `zeros` are
[K/16][groups][16] (rows beyond K: scale 0, zero 8).  A code q stands for (q - zero) * scale; without zeros, zero is 8.
"""
import math

import torch

own = False

BF16, FP16, FP32, INT8 = "bfloat16", "float16", "float32", "int8"


def _quantize(name, K, C, group, dtype, symmetric, scale_dtype=BF16):
    return dict(name=name, op="quantize", K=K, C=C, group=group, dtype=dtype, symmetric=symmetric,
                scale_dtype=scale_dtype)


def _linear(name, M, C, K, group, dtype, zeros=False, bias=False, scale_dtype=BF16):
    return dict(name=name, op="linear", M=M, C=C, K=K, group=group, dtype=dtype, zeros=zeros, bias=bias,
                scale_dtype=scale_dtype)


def _experts(name, T, D, I, E, top_k, group, dtype, zeros=False, scale_dtype=BF16):
    return dict(name=name, op="experts", T=T, D=D, I=I, E=E, top_k=top_k, group=group, dtype=dtype, zeros=zeros,
                scale_dtype=scale_dtype)


def listed():
    return [
        # a small layer's weights after an update, kept in 32 bits
        _quantize("quantize_512x512_g64", 512, 512, 64, FP32, True),
        # the weights of a large layer, zero points
        _quantize("quantize_8192x8192_g128_zeros", 8192, 8192, 128, BF16, False),
        # the classifier behind a convolutional network: 512 pooled int8 codes of one image, ten classes
        _linear("linear_1x512_10_int8", 1, 512, 10, 32, INT8, bias=True),
        # one token through a square projection: latency
        _linear("linear_1x4096_4096", 1, 4096, 4096, 128, BF16),
        # one token, few outputs and a long sum, small groups with zero points
        _linear("linear_1x16384_2048_g64_zeros", 1, 16384, 2048, 64, FP16, zeros=True, scale_dtype=FP16),
        # one token over a vocabulary: the largest matrix
        _linear("linear_1x8192_32768", 1, 8192, 32768, 128, BF16),
        # sizes that fill no tile, real inputs in 32 bits
        _linear("linear_5x2000_1001_g32_f32", 5, 2000, 1001, 32, FP32, zeros=True, bias=True),
        # a batch of tokens, one from each sequence that is being served
        _linear("linear_16x8192_8192", 16, 8192, 8192, 128, BF16, bias=True),
        # a larger batch, or a short prompt
        _linear("linear_64x8192_8192_zeros", 64, 8192, 8192, 128, BF16, zeros=True),
        # one token through eight of 64 small experts
        _experts("experts_1x2048_1024_64_k8", 1, 2048, 1024, 64, 8, 128, BF16),
        # sizes that fill no tile, few experts
        _experts("experts_5x1000_360_12_k3_f16", 5, 1000, 360, 12, 3, 32, FP16, zeros=True, scale_dtype=FP16),
        # a batch of tokens: most experts are chosen by someone
        _experts("experts_16x2048_1024_64_k8", 16, 2048, 1024, 64, 8, 128, BF16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A multiple of 128 or 8, or any number."""
    n, kind = _log_int(rng, lo, hi), rng.random()
    return max(128, n // 128 * 128) if kind < 0.55 and n >= 128 else max(8, n // 8 * 8) if kind < 0.8 else n


def draw(rng):
    kind = rng.random()
    group = rng.choice([32, 64, 128, 128])
    scale_dtype = rng.choice([BF16, FP16])
    if kind < 0.15:
        while True:
            K, C = _size(rng, 64, 16384), _size(rng, 64, 16384)
            if K * C <= 8192 * 8192:
                c = _quantize("", K, C, group, rng.choice([BF16, FP16, FP32]), rng.random() < 0.5, scale_dtype)
                break
    elif kind < 0.65:
        while True:
            M, C, K = _log_int(rng, 1, 64), _size(rng, 64, 16384), _size(rng, 10, 32768)
            if C * K <= 8192 * 32768 and M * C * K <= 64 * 8192 * 8192:
                c = _linear("", M, C, K, group, rng.choice([BF16, BF16, FP16, FP32, INT8]), rng.random() < 0.4,
                            rng.random() < 0.4, scale_dtype)
                break
    else:
        while True:
            T, D, I, E = _log_int(rng, 1, 32), _size(rng, 128, 4096), _size(rng, 64, 4096), _log_int(rng, 4, 128)
            k = min(E, rng.choice([1, 2, 2, 4, 6, 8]))
            if E * D * I <= 64 * 2048 * 1024 and T * k <= 16 * 8 * 2:
                c = _experts("", T, D, I, E, k, group, rng.choice([BF16, BF16, FP16, FP32]), rng.random() < 0.3,
                             scale_dtype)
                break
    del c["name"]
    return c


# --- inputs ------------------------------------------------------------------------------
def _type(name):
    return getattr(torch, name)


def _round_up(n, to):
    return -(-n // to) * to


def _groups(C, group):
    return -(-C // group)


def _packed(gen, case, K, C, batch=()):
    """Random packed weights (codes, scales, zeros, K, C, group), bell-shaped as trained ones are:
    the largest of a group is at the end of the range or next to it."""
    group = case["group"]
    rt, nc, ng = _round_up(K, 16) // 16, _round_up(C, 128) // 128, _groups(C, group)
    shape = (*batch, rt, nc, 16, 4, 16)
    zeros = None
    if case["zeros"]:
        zeros = torch.randint(5, 11, (*batch, rt, ng, 16), generator=gen, device="cuda", dtype=torch.uint8)
    lo, hi = (torch.empty(shape, dtype=torch.float16, device="cuda").normal_(8.0, 2.6, generator=gen).round_()
              .clamp_(0.0, 15.0).to(torch.uint8) for _ in range(2))
    codes = hi.mul_(16).add_(lo)
    # a layer's outputs are about as large as its inputs
    scales = torch.randn((*batch, rt, ng, 16), generator=gen, device="cuda").mul_(0.25).exp_().div_(2.6 * math.sqrt(C))
    return codes, scales.to(_type(case["scale_dtype"])), zeros, K, C, group


def _activations(gen, M, C, dtype):
    x = torch.randn((M, C), generator=gen, device="cuda")
    x *= torch.where(torch.rand(C, generator=gen, device="cuda") < 0.01, 8.0, 1.0)   # some channels are larger
    return x.to(_type(dtype))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "quantize":
        w = torch.randn((case["K"], case["C"]), generator=gen, device="cuda").mul_(0.02)
        return dict(op="quantize", w=w.to(_type(case["dtype"])), group=case["group"], symmetric=case["symmetric"],
                    scale_dtype=_type(case["scale_dtype"]))
    if case["op"] == "linear":
        M, C, K = case["M"], case["C"], case["K"]
        state = dict(op="linear", w=_packed(gen, case, K, C), q_x=None,
                     bias=torch.randn(K, generator=gen, device="cuda") if case["bias"] else None)
        if case["dtype"] == INT8:      # codes of a layer's output behind a rectifier
            x = torch.randn((M, C), generator=gen, device="cuda").abs_().mul_(32.0).round_().clamp_(0, 120)
            state.update(x=(x - 5).to(torch.int8), q_x=dict(scale=1.0 / 32.0, zero_point=-5))
        else:
            state["x"] = _activations(gen, M, C, case["dtype"])
        return state
    T, D, I, E = case["T"], case["D"], case["I"], case["E"]
    router = torch.randn((E, D), generator=gen, device="cuda").div_(math.sqrt(D)).to(_type(case["dtype"]))
    return dict(op="experts", x=_activations(gen, T, D, case["dtype"]), router=router,
                router_bias=torch.randn(E, generator=gen, device="cuda").mul_(0.1), top_k=case["top_k"],
                gate=_packed(gen, case, I, D, (E,)), up=_packed(gen, case, I, D, (E,)),
                down=_packed(gen, case, D, I, (E,)))


# --- one pass ----------------------------------------------------------------------------
def _unpack(w):
    """The values of packed weights in 32 bits: [..., K, C]."""
    codes, scales, zeros, K, C, group = w
    *batch, rt, nc, _, _, _ = codes.shape
    nibbles = torch.stack((codes & 15, codes >> 4), -1)                     # of byte 4 i + j: 2 j and 2 j + 1
    q = nibbles.view(*batch, rt, nc, 16, 4, 4, 2, 4)                        # a b r t i h n: e = 2 n + h
    n = len(batch)
    q = q.permute(*range(n), n, n + 2, n + 1, n + 4, n + 3, n + 6, n + 5).reshape(*batch, rt * 16, nc * 128)
    q = q[..., :K, :C].float()
    ng = _groups(C, group)

    def spread(v):                                                          # per group -> per input
        v = v.transpose(-1, -2).reshape(*batch, rt * 16, ng)[..., :K, :]
        return v.float().repeat_interleave(group, -1)[..., :C]
    return q.sub_(8.0 if zeros is None else spread(zeros)).mul_(spread(scales))


def _by_tiles(v, fill):
    """[K][groups] as in packed weights: [K/16][groups][16], rows beyond K filled."""
    K, ng = v.shape
    v = torch.nn.functional.pad(v, (0, 0, 0, -K % 16), value=fill)
    return v.view(-1, 16, ng).transpose(1, 2).contiguous()


def _plain_quantize(state):
    w, group = state["w"].float(), state["group"]
    K, C = w.shape
    ng = _groups(C, group)
    w = torch.nn.functional.pad(w, (0, ng * group - C)).view(K, ng, group)
    largest = torch.finfo(state["scale_dtype"]).max
    if state["symmetric"]:
        span, parts = w.abs().amax(-1, keepdim=True), 7.0
    else:
        low = w.amin(-1, keepdim=True).clamp_(max=0.0)
        span, parts = w.amax(-1, keepdim=True).clamp_(min=0.0) - low, 15.0
    s = (span / torch.full_like(span, parts)).clamp_(max=largest).to(state["scale_dtype"])
    s32 = s.float()
    by = torch.where(s32 > 0, s32, 1.0)
    z = torch.full_like(s32, 8.0) if state["symmetric"] else (-low / by).round_().clamp_(0.0, 15.0)
    z = torch.where(s32 > 0, z, 8.0)
    q = torch.where(s32 > 0, (w / by).round_() + z, z).clamp_(0.0, 15.0)
    values = ((q - z) * s32).view(K, ng * group)[:, :C].to(state["w"].dtype)
    return dict(values=values, scales=_by_tiles(s[..., 0], 0.0),
                zeros=None if state["symmetric"] else _by_tiles(z[..., 0], 8.0).to(torch.uint8))


def _plain_linear(state):
    x = state["x"].float()
    if state["q_x"] is not None:
        x = (x - state["q_x"]["zero_point"]) * state["q_x"]["scale"]
    y = x @ _unpack(state["w"]).T
    if state["bias"] is not None:
        y = y + state["bias"]
    return y if state["q_x"] is not None else y.to(state["x"].dtype)


def _plain_experts(state):
    x, k = state["x"].float(), state["top_k"]
    p = torch.softmax(x @ state["router"].float().T + state["router_bias"], -1)
    weights, ids = torch.sort(p, dim=-1, descending=True, stable=True)
    weights, ids = weights[:, :k], ids[:, :k]
    weights = weights / weights.sum(-1, keepdim=True)
    gate, up = x @ _unpack(state["gate"]).transpose(1, 2), x @ _unpack(state["up"]).transpose(1, 2)
    out = (gate / (1.0 + torch.exp(-gate)) * up) @ _unpack(state["down"]).transpose(1, 2)   # [E, T, D]
    share = torch.zeros_like(p).scatter_(1, ids, weights)
    y = (out * share.T[:, :, None]).sum(0)
    return dict(y=y.to(state["x"].dtype), ids=ids.to(torch.int32), weights=weights)


def run(state):
    op = state["op"]
    if own:
        from paper_2002_10711_b200 import layer
        if op == "quantize":
            w, values = layer.quantize_w4(state["w"], state["group"], state["symmetric"], state["scale_dtype"],
                                          values=True)
            return dict(values=values, scales=w.scales, zeros=w.zeros)
        if op == "linear":
            return layer.linear_w4(state["x"], state["w"], state["bias"], state["q_x"])
        y, ids, weights = layer.experts_w4(state["x"], state["router"], state["gate"], state["up"], state["down"],
                                           state["top_k"], state["router_bias"])
        return dict(y=y, ids=ids, weights=weights)
    return _plain_quantize(state) if op == "quantize" else _plain_linear(state) if op == "linear" \
        else _plain_experts(state)


# --- what a pass cannot do without -------------------------------------------------------
_BYTES = {BF16: 2, FP16: 2, FP32: 4, INT8: 1}


def _weight_bytes(case, K, C):
    return K * C // 2 + K * _groups(C, case["group"]) * (3 if case["zeros"] else 2)


def work(case):
    size = _BYTES[case["dtype"]]
    if case["op"] == "quantize":
        K, C = case["K"], case["C"]
        scales = K * _groups(C, case["group"]) * (2 if case["symmetric"] else 3)
        return dict(bytes=K * C * (2 * size + 0.5) + scales, flops=5 * K * C)
    if case["op"] == "linear":
        M, C, K = case["M"], case["C"], case["K"]
        return dict(bytes=_weight_bytes(case, K, C) + M * C * size + M * K * (4 if size == 1 else size)
                    + (4 * K if case["bias"] else 0), flops=2 * M * C * K)
    T, D, I, E, k = (case[n] for n in ("T", "D", "I", "E", "top_k"))
    chosen = E * (1.0 - (1.0 - k / E) ** T)          # distinct experts, on average
    return dict(bytes=chosen * (2 * _weight_bytes(case, I, D) + _weight_bytes(case, D, I)) + E * D * size + 4 * E
                + 2 * T * D * size + 8 * T * k, flops=2 * T * E * D + 6 * T * k * D * I)


# --- the definition in 64 bits -------------------------------------------------------------
def _exact_matrix(codes, scales, zeros, K, C, group):
    """One matrix in 64 bits, code by code from its place in the packed form."""
    rt, nc = codes.shape[0], codes.shape[1]
    words = codes.contiguous().view(torch.int32).reshape(-1)               # [a][b][r][t][i]
    row = torch.arange(K, device="cuda")[:, None]
    col = torch.arange(C, device="cuda")[None, :]
    unit = (((row // 16) * nc + col // 128) * 16 + row % 16) * 4 + col // 8 % 4
    e = col % 8
    shift = 4 * (e // 2 + 4 * (e % 2))
    q = (words[unit * 4 + col // 32 % 4] >> shift) & 15
    ng = scales.shape[1]
    at = ((row // 16) * ng + col // group) * 16 + row % 16
    z = 8 if zeros is None else zeros.reshape(-1)[at].to(torch.float64)
    return (q.to(torch.float64) - z) * scales.reshape(-1)[at].to(torch.float64)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quantize":
        w = state["w"].to(torch.float64)
        K, C = w.shape
        group, kind = case["group"], state["scale_dtype"]
        ng, tiles = _groups(C, group), -(-K // 16)
        values = torch.empty_like(w)
        scales = torch.zeros((tiles * 16, ng), dtype=torch.float64, device="cuda")
        zeros = torch.full((tiles * 16, ng), 8, dtype=torch.uint8, device="cuda")
        for g in range(ng):
            part = w[:, g * group:(g + 1) * group]
            if case["symmetric"]:
                s = part.abs().max(1).values / 7
            else:
                low, high = part.min(1).values.clamp(max=0), part.max(1).values.clamp(min=0)
                s = (high - low) / 15
            s = s.to(kind).to(torch.float64)
            scales[:K, g] = s
            safe = torch.where(s > 0, s, torch.ones_like(s))
            z = torch.full_like(s, 8) if case["symmetric"] else torch.round(-low / safe).clamp(0, 15)
            zeros[:K, g] = torch.where(s > 0, z, 8.0).to(torch.uint8)
            q = (torch.round(part / safe[:, None]) + z[:, None]).clamp(0, 15)
            values[:, g * group:(g + 1) * group] = torch.where(s[:, None] > 0, (q - z[:, None]) * s[:, None], 0.0)
        place = [v.view(tiles, 16, ng).transpose(1, 2).contiguous() for v in (scales, zeros)]
        return dict(values=values, scales=place[0], zeros=None if case["symmetric"] else place[1])
    x = state["x"].to(torch.float64)
    if case["op"] == "linear":
        codes, scales, zeros, K, C, group = state["w"]
        if state["q_x"] is not None:
            x = (x - state["q_x"]["zero_point"]) * state["q_x"]["scale"]
        y = torch.empty((x.shape[0], K), dtype=torch.float64, device="cuda")
        step = max(16, (1 << 26) // C // 16 * 16)                           # outputs at a time
        for k in range(0, K, step):
            a, b = k // 16, -(-min(K, k + step) // 16)
            part = _exact_matrix(codes[a:b], scales[a:b], None if zeros is None else zeros[a:b],
                                 min(K, k + step) - k, C, group)
            y[:, k:k + step] = x @ part.T
        return y if state["bias"] is None else y + state["bias"].to(torch.float64)
    k = case["top_k"]
    logits = x @ state["router"].to(torch.float64).T + state["router_bias"].to(torch.float64)
    y = torch.zeros_like(x)
    order = torch.argsort(-logits, dim=-1, stable=True)[:, :k]
    chosen = torch.gather(logits, 1, order)
    weights = torch.exp(chosen - torch.logsumexp(chosen, -1, keepdim=True))

    def product(v, w, e):
        codes, scales, zeros, K, C, group = w
        return v @ _exact_matrix(codes[e], scales[e], None if zeros is None else zeros[e], K, C, group).T
    for e in range(case["E"]):
        share = (weights * (order == e)).sum(-1)
        rows = torch.nonzero((order == e).any(-1))[:, 0]
        if rows.numel():
            gate, up = product(x[rows], state["gate"], e), product(x[rows], state["up"], e)
            y[rows] += share[rows, None] * product(gate * torch.sigmoid(gate) * up, state["down"], e)
    return dict(y=y, ids=order.to(torch.int32), weights=weights)
