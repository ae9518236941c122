"""Norm and rotation of query and key rows against their formulas in 64 bits."""
import pytest
import torch

import mx4_ref as ref
from paper_2609_23314_amd import vd

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rows(shape, dtype, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * 2).to(dtype)


def _inv_freq(R, base=10000.0):
    return (base ** (-torch.arange(0, R, 2).double() / R)).float()


def _check(out, x, w, pos, inv_freq, eps, interleaved):
    """fp32 arithmetic: the norm is a sum of D squares, added 8 in a lane and by
    halves over the lanes, a square root, a division and two products (together
    within 20 * 2^-24 of y); cos and sin are off by the angle's rounding to fp32
    (2^-24 * pi) and two steps, the sum of two products by one more: within 12 * 2^-24
    of the terms' sizes.  The angle in turns is three fp64 products of its size."""
    want, size = ref.rope(x, w, pos, inv_freq, eps, interleaved)
    far = float(pos.abs().max()) * float(inv_freq.abs().max()) * 4 * 2.0 ** -53
    tol = (32 * 2.0 ** -24 + far) * size
    tol = tol + (torch.finfo(out.dtype).eps / 2) * (want.abs() + tol) + 1e-37
    err = (out.cpu().double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,R", [(64, 64), (64, 8), (128, 128), (128, 32), (256, 256), (256, 72)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["both", "q", None])
def test_norm_rope(dtype, D, R, interleaved, norm):
    S, L, H, G, t = 2, 3, 2, 3, 5
    q, k = _rows((S, L, H * G, t, D), dtype, 1), _rows((S, L, H, t, D), dtype, 2)
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(0, 5000, (S, t), generator=g).int()
    wt = dtype if D != 128 else torch.float32
    qw = (1 + 0.3 * torch.randn((L, D), generator=g)).to(wt) if norm else None
    kw = (1 + 0.3 * torch.randn((L, D), generator=g)).to(wt) if norm == "both" else None
    f = _inv_freq(R)
    to = lambda x: None if x is None else x.to(DEV)  # noqa: E731
    outs = vd.vd_qk_norm_rope(to(q), to(k), to(pos), to(f), to(qw), to(kw), eps=1e-5, interleaved=interleaved)
    for out, x, w in zip(outs, (q, k), (qw, kw)):
        assert out.dtype == dtype and out.shape == x.shape
        _check(out, x, w, pos, f, 1e-5, interleaved)


@pytest.mark.parametrize("S,L,H,G,t", [(1, 1, 1, 1, 1), (1, 1, 2, 4, 1000), (17, 1, 1, 3, 1), (1, 40, 8, 4, 9), (3, 2, 5, 7, 67)])
def test_shapes_and_mixed_types(S, L, H, G, t):
    """Few tokens and many; fp32 queries beside bf16 keys, the keys straight into a cache's slots."""
    D = 128
    q, k = _rows((S, L, H * G, t, D), torch.bfloat16, 4), _rows((S, L, H, t, D), torch.bfloat16, 5)
    pos = torch.arange(S * t).int().view(S, t) + 77
    w = torch.ones(L, D)
    cache = torch.full((S, L, H, t + 6, D), 3.0, dtype=torch.bfloat16, device=DEV)
    qo = torch.empty(q.shape, dtype=torch.float32, device=DEV)
    qo, ko = vd.vd_qk_norm_rope(q.to(DEV), k.to(DEV), pos.to(DEV), _inv_freq(D).to(DEV), w.to(DEV), w.to(DEV), qo,
                                cache[:, :, :, 4:4 + t])
    _check(qo, q, w, pos, _inv_freq(D), 1e-6, False)
    _check(cache[:, :, :, 4:4 + t], k, w, pos, _inv_freq(D), 1e-6, False)
    assert cache[:, :, :, :4].eq(3).all() and cache[:, :, :, 4 + t:].eq(3).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_fused_projection_in_place(dtype):
    """Query and key parts of one [token, heads * D] projection, in place; the value part is left alone."""
    T, H, G, D = 37, 2, 4, 64
    qkv = _rows((1, T, (G + 2) * H, D), dtype, 6)
    d = qkv.to(DEV)
    view = lambda a, b, x: x[:, :, a:b].permute(0, 2, 1, 3).unsqueeze(1)  # noqa: E731
    q, k = view(0, G * H, d), view(G * H, (G + 1) * H, d)
    pos, f, w = torch.arange(T).int().view(1, T), _inv_freq(D), torch.full((1, D), 0.7)
    vd.vd_qk_norm_rope(q, k, pos.to(DEV), f.to(DEV), w.to(DEV), w.to(DEV), q, k)
    _check(q, view(0, G * H, qkv), w, pos, f, 1e-6, False)
    _check(k, view(G * H, (G + 1) * H, qkv), w, pos, f, 1e-6, False)
    assert torch.equal(d[:, :, (G + 1) * H:].cpu(), qkv[:, :, (G + 1) * H:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_and_one_side(interleaved):
    D = 64
    q = _rows((1, 1, 2, 6, D), torch.float32, 7)
    pos = torch.tensor([[0, 1, 10 ** 6, 2 ** 24 + 1, 2 ** 31 - 1, -5]]).int()
    out, none = vd.vd_qk_norm_rope(q.to(DEV), None, pos.to(DEV), _inv_freq(D).to(DEV), interleaved=interleaved)
    assert none is None
    _check(out, q, None, pos, _inv_freq(D), 0.0, interleaved)
    none, out = vd.vd_qk_norm_rope(None, q.to(DEV), pos.to(DEV), _inv_freq(D).to(DEV), interleaved=interleaved)
    assert none is None
    _check(out, q, None, pos, _inv_freq(D), 0.0, interleaved)


def test_zero_rows_and_nonfinite_ones():
    """A row of zeros stays zero (eps > 0); a row with NaN or an infinity spoils itself alone."""
    D = 128
    x = _rows((1, 1, 3, 4, D), torch.float32, 8)
    x[0, 0, 0, 0] = 0
    w = torch.ones(1, D, device=DEV)
    pos, f = torch.arange(4).int().view(1, 4).to(DEV), _inv_freq(D).to(DEV)
    clean, _ = vd.vd_qk_norm_rope(x.to(DEV), None, pos, f, w)
    assert not clean[0, 0, 0, 0].any() and torch.isfinite(clean).all()
    y = x.clone()
    y[0, 0, 1, 2, 9] = float("nan")
    out, _ = vd.vd_qk_norm_rope(y.to(DEV), None, pos, f, w)
    assert out[0, 0, 1, 2].isnan().all()
    out[0, 0, 1, 2] = clean[0, 0, 1, 2]
    assert torch.equal(out, clean)
