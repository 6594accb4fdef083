"""Plain references in 64 bits of the layers with 4-bit weights, on the CPU, with bounds on what a
32-bit kernel may be off."""
import numpy as np
import torch

U = 2.0 ** -23        # one truncated 32-bit addition


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def code_at(codes, k, c):
    """The code of output k, input c, by the documented layout: codes numpy uint8 [K/16][C/128][16][4][16]."""
    b = c % 128
    i, t, e = b // 32, b // 8 % 4, b % 8
    unit = codes[k // 16, c // 128, k % 16, t]
    word = int.from_bytes(unit[4 * i:4 * i + 4].tobytes(), "little")
    nibble = e // 2 if e % 2 == 0 else 4 + e // 2
    return word >> (4 * nibble) & 15


def matrix(q, scales, zeros, group):
    """(codes - zeros) * scales in 64 bits; q [K, C], scales and zeros [K, groups] tensors."""
    C = q.shape[-1]
    spread = lambda v: v.double().repeat_interleave(group, -1)[..., :C]  # noqa: E731
    return (q.double() - (8.0 if zeros is None else spread(zeros))) * spread(scales)


def steps(C, group, parts=1):
    """Roundings on the way of a product into its sum: inside a 16-wide MMA at most 17, one for every later
    MMA of its group, one per 128-input tile or group of a warp, warps and blocks that are joined, the last multiplication."""
    g = min(group, 128)
    return 17 + parts * g // 16 + 2 * (-(-C // g)) + 8 + 8 + 2


def linear(x, W, bias, group, parts=1, rows=None):
    """(y, bound of a 32-bit sum's error), all 64 bits."""
    y, size = x @ W.T, x.abs() @ W.abs().T
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, steps(W.shape[1], group, parts) * U * size


def experts(x, router, bias, gate, up, down, groups, top_k, normalize, dtype):
    """(y, ids, weights, bound of y): gate, up, down [E, ., .] in 64 bits."""
    logits = x @ router.T + (0 if bias is None else bias.double())
    order = torch.argsort(-logits, dim=-1, stable=True)[:, :top_k]
    p = torch.softmax(logits, -1)
    w = torch.gather(p, 1, order)
    if normalize:
        w = w / w.sum(-1, keepdim=True)
    w = torch.nan_to_num(w, 0.0) if not torch.isnan(logits).any() else w
    y, off = torch.zeros_like(x), torch.zeros_like(x)
    parts = 3 if dtype == torch.float32 else 1
    kept = 2.0 ** -22 if dtype == torch.float32 else 2.0 ** -15      # h as a sum of three or two bf16
    for t in range(x.shape[0]):
        for j in range(top_k):
            e = int(order[t, j])
            a = float(w[t, j])
            if a == 0.0:
                continue
            g, dg = linear(x[t:t + 1], gate[e], None, groups[0], parts)
            u, du = linear(x[t:t + 1], up[e], None, groups[0], parts)
            s = g * torch.sigmoid(g)
            h = s * u
            # |silu'| < 1.1; exp, quotient and products: a few steps of 32 bits each
            dh = 1.1 * dg * u.abs() + s.abs() * du + (kept + 16 * U) * h.abs()
            v, dv = linear(h, down[e], None, groups[1], 3)
            y[t] += a * v[0]
            # the weight itself: exp of a logit's difference, whose error is the logits' own
            dl = 2 * (x.shape[1] / 32 + 16) * U * float((x[t].abs() @ router.abs().T).max())
            off[t] += a * (dv + dh @ down[e].abs().T)[0] + a * (dl + 16 * U) * v[0].abs() * 2
    return y, order, w, off


def random_packed(rng, K, C, group, scale_dtype=torch.bfloat16, zeros=False, batch=()):
    """(codes, scales, zeros) of layer.pack_w4, on the CPU."""
    groups = -(-C // group)
    q = torch.from_numpy(rng.integers(0, 16, (*batch, K, C), dtype=np.uint8))
    s = torch.from_numpy(np.exp(rng.normal(0, 0.5, (*batch, K, groups))) / (5 * np.sqrt(C))).to(scale_dtype)
    z = torch.from_numpy(rng.integers(0, 16, (*batch, K, groups), dtype=np.uint8)) if zeros else None
    return q, s, z
