"""The 4-bit cache and its rows in 64 bits, from their definitions, for the tests."""
import math

import torch

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def encode(x):
    """(codes uint8 [..., D/2], scales uint8 [..., D/32]) of rows [..., D]."""
    g = x.detach().cpu().double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    fine = torch.isfinite(g).all(-1)
    m, e = torch.frexp(torch.where(fine, top, 1.0))            # top = m * 2^e, m in [0.5, 1)
    e = torch.where(m < 0.875, e - 3, e - 2)                   # the least e with top < 7 * 2^e
    e = torch.where(top == 0, -127, e).clamp(-127, 125)
    y = torch.where(fine.unsqueeze(-1), g.abs() * torch.exp2(-e.double()).unsqueeze(-1), 0.0)
    d = (y.unsqueeze(-1).clamp(max=6.0) - MAGNITUDES).abs()
    near = d == d.amin(-1, keepdim=True)                       # one magnitude, or two on a tie
    even = torch.arange(8) % 2 == 0
    code = torch.where(near.sum(-1, keepdim=True) > 1, near & even, near).to(torch.uint8).argmax(-1)
    code = torch.where(fine.unsqueeze(-1), code + 8 * torch.signbit(g), 0).to(torch.uint8).flatten(-2)
    scale = torch.where(fine, e + 127, 255).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def decode(codes, scales):
    """float64 rows [..., D]."""
    codes, scales = codes.cpu(), scales.cpu()
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = MAGNITUDES[c & 7] * torch.where(c >= 8, -1.0, 1.0).double()
    s = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
    return v * s.repeat_interleave(32, -1)


def attention(k, v, q, n, rows, scale):
    """One unit's output [G, t, D] of queries [G, t, D] over values [C, D], with
    the weighted mean of |v| and, over the cached rows that a query row sees, the
    largest sum |q_c k_c| and the largest sum of |k_c| times the largest |q| of c's
    32 channels."""
    G, t, D = q.shape
    out, size = torch.zeros((G, t, D)).double(), torch.zeros((G, t, D)).double()
    prod, most = torch.zeros((G, t, 1)).double(), torch.zeros((G, t, 1)).double()
    top = q.abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
    for i in range(rows):
        m = max(0, n - rows + 1 + i)
        if m:
            w = torch.softmax(q[:, i] @ k[:m].T * scale, -1)
            out[:, i], size[:, i] = w @ v[:m], w @ v[:m].abs()
            prod[:, i, 0] = (q[:, i].abs() @ k[:m].abs().T).amax(-1)
            most[:, i, 0] = (top[:, i] @ k[:m].abs().T).amax(-1)
    return out, size, prod, most


def scores(x, variant):
    """float64 scores of one unit's scored rows [n, D]."""
    form = variant.replace("key_", "")
    mean = x.mean(0)
    if form == "norm":
        return x.norm(dim=-1)
    if form == "l2":
        return (x - mean).norm(dim=-1)
    both = x.norm(dim=-1) * mean.norm()
    return torch.where(both > 0, 1 - (x @ mean) / torch.where(both > 0, both, 1.0), 1.0)


def kept(score, N, variant):
    """The slots that stay: the N best, equal ones by the lower slot."""
    order = sorted(range(len(score)), key=lambda j: (score[j] if variant == "key_norm" else -score[j], j))
    return sorted(order[:N])


def moves(keep, n, N):
    """(from, to) slots of the gather."""
    keep = set(keep)
    holes = [j for j in range(min(N, n)) if j not in keep]
    movers = [j for j in range(N, n) if j in keep]
    return list(zip(movers, holes))


def rope(x, w, pos, inv_freq, eps, interleaved):
    """float64 [S, L, H, t, D], with the size of each output's terms."""
    y = x.double()
    if w is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()[None, :, None, None, :]
    R = 2 * inv_freq.numel()
    i = torch.arange(R // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    angle = (pos.double().unsqueeze(-1) * inv_freq.double())[:, None, None]
    out, size = y.clone(), y.abs()
    out[..., a] = y[..., a] * angle.cos() - y[..., b] * angle.sin()
    out[..., b] = y[..., b] * angle.cos() + y[..., a] * angle.sin()
    size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, size
