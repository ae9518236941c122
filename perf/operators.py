"""The operators around a KV cache held in 4 bits, as measurable cases.

The rows that go into a cache are made by the norms of queries and keys and
their rotation; a 4-bit cache (e2m1 codes with one power of two per 32 channels)
is filled, read back, attended to and evicted from.  Every case is one of these
calls, at the shapes of the repository's workloads or at generic sizes of the
same ranges.

``own`` false: the plain forms, elementary torch operations on the same bytes.
``own`` true: the calls of the library.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}
GROUP = 32   # channels that share a scale


def listed():
    return [
        # One layer's decode step, sixteen sequences: the smallest call, latency and launches.
        dict(name="rope_decode", kind="rope", seqs=16, layers=1, heads=8, group=4, dim=128, rows=1, dtype="bf16",
             out="f32", rotary=128, interleaved=False, norm=True, start=30000),
        # An 8B model's prompt block, the q and k rows of all layers.
        dict(name="rope_prefill", kind="rope", seqs=1, layers=32, heads=8, group=4, dim=128, rows=512, dtype="bf16",
             out="bf16", rotary=128, interleaved=False, norm=True, start=2048),
        # Wide heads, an odd block, a quarter of the channels rotated in neighbouring pairs, far positions.
        dict(name="rope_partial_wide", kind="rope", seqs=3, layers=13, heads=4, group=2, dim=256, rows=333, dtype="f32",
             out="f32", rotary=64, interleaved=True, norm=False, start=1000000),
        # One decode step's rows of every layer into the cache, sixteen sequences.
        dict(name="append_decode", kind="append", seqs=16, layers=32, heads=8, group=1, dim=128, rows=1, dtype="bf16",
             capacity=1025),
        # A prompt block's rows of every layer into the cache.
        dict(name="append_prefill", kind="append", seqs=1, layers=32, heads=8, group=1, dim=128, rows=512, dtype="bf16",
             capacity=2560),
        # Decode at a full budget, all layers, fp32 queries as the decode step of the uncompressed cache has them.
        dict(name="attention_decode_b16", kind="attention", seqs=16, layers=32, heads=8, group=4, dim=128, rows=1,
             dtype="f32", n=4097, ragged=False),
        # One layer of it with sequences of different lengths: a call as an engine makes it, layer by layer.
        dict(name="attention_layer_ragged", kind="attention", seqs=16, layers=1, heads=8, group=4, dim=128, rows=1,
             dtype="bf16", n=4097, ragged=True),
        # A single long sequence that nothing was evicted from: few units, split over the rows.
        dict(name="attention_single_long", kind="attention", seqs=1, layers=1, heads=8, group=8, dim=128, rows=1,
             dtype="bf16", n=131072, ragged=False),
        # Block prompt processing: a block of 512 rows attends to the budget and to itself.
        dict(name="attention_block", kind="attention", seqs=1, layers=32, heads=8, group=4, dim=128, rows=512,
             dtype="bf16", n=2560, ragged=False),
        # Wide heads, few sequences, an odd block.
        dict(name="attention_block_wide", kind="attention", seqs=4, layers=2, heads=4, group=2, dim=256, rows=777,
             dtype="bf16", n=4873, ragged=True),
        # The pass at a prompt boundary: 512 of 2560 rows go.
        dict(name="evict_prefill", kind="evict", seqs=1, layers=32, heads=8, group=1, dim=128, n=2560, budget=2048,
             variant="l2", ragged=False),
        # The pass at a decode step: one row of each unit goes.
        dict(name="evict_decode", kind="evict", seqs=16, layers=8, heads=8, group=1, dim=128, n=4097, budget=4096,
             variant="l2", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# what a drawn case reads, writes and computes at most (below the largest listed cases)
_MOST_BYTES, _MOST_FLOPS = 1.2e9, 5.0e11


def draw(rng):
    kind = rng.choice(["rope", "append", "attention", "attention", "block", "evict"])
    c = dict(kind="attention" if kind == "block" else kind, seqs=_log_int(rng, 1, 17), layers=_log_int(rng, 1, 33),
             heads=rng.choice([1, 2, 3, 4, 5, 8]), group=rng.choice([1, 2, 3, 4, 8]) if kind != "evict" else 1,
             dim=rng.choice([64, 128, 256]))
    if kind == "rope":
        c |= dict(rows=_log_int(rng, 1, 1025), dtype=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]),
                  rotary=c["dim"] // rng.choice([1, 1, 2, 4]), interleaved=rng.random() < 0.4,
                  norm=rng.random() < 0.7, start=_log_int(rng, 1, 1000000))
    elif kind == "append":
        c |= dict(rows=_log_int(rng, 1, 1025), dtype=rng.choice(["bf16", "f32"]), capacity=_log_int(rng, 1100, 5000))
    elif kind == "attention":
        c |= dict(rows=1, dtype=rng.choice(["bf16", "f32"]), n=_log_int(rng, 1, 40000), ragged=rng.random() < 0.5)
    elif kind == "block":
        c |= dict(rows=_log_int(rng, 2, 1025), dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.5)
        c["n"] = c["rows"] + _log_int(rng, 1, 5000)
    else:
        budget = _log_int(rng, 16, 8000)
        c |= dict(n=budget + rng.choice([1, _log_int(rng, 1, 1025)]), budget=budget,
                  variant=rng.choice(["l2", "l2", "dir", "norm", "key_l2"]), ragged=rng.random() < 0.5)
    for key in ("seqs", "layers", "rows", "n"):
        while c.get(key, 1) > (1 if key != "n" else max(c.get("rows", 1), c.get("budget", 0) + 1)):
            w = work(c)
            if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS:
                return c
            c[key] = max(c[key] // 2, 1 if key != "n" else max(c.get("rows", 1), c.get("budget", 0) + 1))
    return c


def _lengths(c):
    """The sequences' cached tokens: all n, or ragged ones between a quarter of it and n."""
    S, n = c["seqs"], c["n"]
    if not c["ragged"] or S == 1:
        return [n] * S
    least = max(1, n // 4, c.get("rows", 1), c.get("budget", 0) // 4)
    return [n - (n - least) * s // (S - 1) for s in range(S)]


def _budgets(c):
    """One row to evict at a decode step, the share of the longest sequence else."""
    more = c["n"] - c["budget"]
    return [max(1, n - more) for n in _lengths(c)]


def _row_bytes(c):
    """Bytes of a row in 4 bits: its codes and its scales."""
    return c["dim"] // 2 + c["dim"] // GROUP


def work(c):
    units, D, G = c["seqs"] * c["layers"] * c["heads"], c["dim"], c["group"]
    if c["kind"] == "rope":
        values = units * (G + 1) * c["rows"] * D
        return {"bytes": values * (ESIZE[c["dtype"]] + ESIZE[c["out"]]), "flops": 8 * values}
    if c["kind"] == "append":     # the rows in, the codes and scales, the values that they read back as
        values = 2 * units * c["rows"] * D
        return {"bytes": values * (ESIZE[c["dtype"]] + 2) + 2 * units * c["rows"] * _row_bytes(c), "flops": 4 * values}
    per_layer = c["layers"] * c["heads"]
    if c["kind"] == "attention":
        t = c["rows"]
        rows = sum(_lengths(c)) * per_layer
        seen = sum(t * (n - t) + t * (t + 1) // 2 for n in _lengths(c)) * per_layer * G
        return {"bytes": 2 * rows * _row_bytes(c) + 2 * units * G * t * D * ESIZE[c["dtype"]], "flops": 4 * D * seen}
    rows = sum(_lengths(c)) * per_layer
    gone = sum(n - N for n, N in zip(_lengths(c), _budgets(c))) * per_layer
    # the scored rows, the scores and the mask, and what moves: some of the new rows, K and V, into the evicted rows' slots
    moved = sum((n - N) * N // n for n, N in zip(_lengths(c), _budgets(c))) * per_layer
    return {"bytes": rows * (_row_bytes(c) + 5) + 4 * moved * _row_bytes(c) + 4 * gone, "flops": 4 * rows * D}


# ------------------------------------------------------------------ the 4-bit format, in torch

_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _encode(x):
    """Codes [..., D/2] and scales [..., D/32] (uint8) of rows [..., D]: the scale
    is the least power of two whose sevenfold is above the group's largest
    magnitude, a code the nearest magnitude, ties to the even code."""
    g = x.float().unflatten(-1, (-1, GROUP))
    m, e = torch.frexp(g.abs().amax(-1))
    e = torch.where(m > 0, e - 3 + (m >= 0.875), -127).clamp(-127, 125)
    y = g.abs() * ((127 - e) << 23).view(torch.float32).unsqueeze(-1)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    code = (code + 8 * torch.signbit(g)).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | (code[..., 1] << 4), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    """fp32 rows [..., D] of codes and scales."""
    one = torch.tensor(_MAGNITUDES + tuple(-m for m in _MAGNITUDES), device=codes.device)
    pair = torch.stack([one.repeat(16), one.repeat_interleave(16)], -1)
    x = pair[codes.int()].flatten(-2).unflatten(-1, (-1, GROUP))
    return (x * (scales.int() << 23).clamp(min=0x00400000).view(torch.float32).unsqueeze(-1)).flatten(-2)


# ------------------------------------------------------------------ inputs

def _rows(g, shape, dtype, seed_scale=0.5):
    """Rows as a model makes them: normal, some channels larger, one token in a hundred an outlier."""
    S, L, H, t, D = shape
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(seed_scale * torch.randn((1, L, H, 1, D), generator=g, device=DEV))
    x *= torch.where(torch.rand((S, 1, 1, t, 1), generator=g, device=DEV) < 0.01, 4.0, 1.0)
    return x.to(dtype)


def _cache(g, c, capacity):
    """Codes and scales of K and V, layer by layer."""
    S, L, H, D = c["seqs"], c["layers"], c["heads"], c["dim"]
    made = [torch.empty((S, L, H, capacity, D // (2 if i < 2 else GROUP)), dtype=torch.uint8, device=DEV) for i in range(4)]
    for layer in range(L):
        for i in (0, 1):
            codes, scales = _encode(_rows(g, (S, 1, H, capacity, D), torch.bfloat16))
            made[i][:, layer:layer + 1], made[2 + i][:, layer:layer + 1] = codes, scales
    return made


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    S, L, H, G, D = c["seqs"], c["layers"], c["heads"], c["group"], c["dim"]
    st = {"case": c}
    if c["kind"] == "rope":
        dt, R = DTYPE[c["dtype"]], c["rotary"]
        st["q"] = _rows(g, (S, L, H * G, c["rows"], D), dt)
        st["k"] = _rows(g, (S, L, H, c["rows"], D), dt)
        first = torch.randint(0, c["start"] + 1, (S, 1), generator=g, device=DEV)
        st["pos"] = (first + torch.arange(c["rows"], device=DEV)).int()
        st["inv_freq"] = (500000.0 ** (-torch.arange(0, R, 2, device=DEV).double() / R)).float()
        for name in ("q_weight", "k_weight"):
            st[name] = (1 + 0.2 * torch.randn((L, D), generator=g, device=DEV)) if c["norm"] else None
    elif c["kind"] == "append":
        C = max(c["capacity"], c["rows"])
        st["cache"] = [torch.zeros((S, L, H, C, D // k), dtype=torch.uint8, device=DEV) for k in (2, 2, GROUP, GROUP)]
        st["n_old"] = [(C - c["rows"]) * s // S for s in range(S)]
        st["slots"] = torch.tensor(st["n_old"], device=DEV).view(S, 1) + torch.arange(c["rows"], device=DEV)
        st["k_rows"] = _rows(g, (S, L, H, c["rows"], D), DTYPE[c["dtype"]])
        st["v_rows"] = _rows(g, (S, L, H, c["rows"], D), DTYPE[c["dtype"]])
    elif c["kind"] == "attention":
        st["cache"] = _cache(g, c, c["n"])
        st["q"] = _rows(g, (S, L, H * G, c["rows"], D), DTYPE[c["dtype"]], 0.2)
        st["n"] = _lengths(c)
        st["n_dev"] = torch.tensor(st["n"], device=DEV)
    else:
        st["cache"] = _cache(g, c, c["n"])
        st["n"], st["budget"] = _lengths(c), _budgets(c)
        st["n_dev"], st["budget_dev"] = torch.tensor(st["n"], device=DEV), torch.tensor(st["budget"], device=DEV)
        st["pos"] = torch.arange(c["n"], dtype=torch.int32, device=DEV).repeat(S * L * H, 1)
    if own:
        from paper_2609_23314_amd import vd
        vd.load()
    return st


# ------------------------------------------------------------------ the calls

def run(state):
    return {"rope": _run_rope, "append": _run_append, "attention": _run_attention, "evict": _run_evict}[state["case"]["kind"]](state)


def _run_rope(st):
    c = st["case"]
    if own:
        from paper_2609_23314_amd import vd
        q_out = torch.empty(st["q"].shape, dtype=DTYPE[c["out"]], device=DEV)
        k_out = torch.empty(st["k"].shape, dtype=DTYPE[c["out"]], device=DEV)
        return vd.vd_qk_norm_rope(st["q"], st["k"], st["pos"], st["inv_freq"], st["q_weight"], st["k_weight"], q_out, k_out,
                                  eps=1e-6, interleaved=c["interleaved"])
    return [_plain_rope(st[x], st["pos"], st["inv_freq"], st[x + "_weight"], c) for x in ("q", "k")]


def _plain_rope(x, pos, inv_freq, weight, c):
    R = c["rotary"]
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight[:, None, None, :]
    angle = pos.double().unsqueeze(-1) * inv_freq.double()    # far positions lose their angle in 32 bits
    cos, sin = [f(angle).float()[:, None, None] for f in (torch.cos, torch.sin)]
    r = y[..., :R]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :R // 2], r[..., R // 2:])
    u, w = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([u, w], -1).flatten(-2) if c["interleaved"] else torch.cat([u, w], -1)
    return torch.cat([r, y[..., R:]], -1).to(DTYPE[c["out"]])


def _run_append(st):
    """The rows into the cache, and the values that it then holds for them."""
    c, cache = st["case"], st["cache"]
    if own:
        from paper_2609_23314_amd import vd
        mx = vd.Mx4Cache(*cache)
        vd.vd_append_mx4(mx, st["n_old"], st["k_rows"], st["v_rows"])
        return vd.vd_read_mx4(mx, st["n_old"], c["rows"])
    made = [*_encode(st["k_rows"]), *_encode(st["v_rows"])]
    at = st["slots"][:, None, None, :, None].expand(-1, c["layers"], c["heads"], -1, -1)
    for i, rows in zip((0, 2, 1, 3), made):
        cache[i].scatter_(3, at.expand(*at.shape[:4], rows.shape[-1]), rows)
    back = [x.gather(3, at.expand(*at.shape[:4], x.shape[-1])) for x in cache]
    return [_decode(back[0], back[2]).bfloat16(), _decode(back[1], back[3]).bfloat16()]


def _run_attention(st):
    c, (k, v, ks, vs) = st["case"], st["cache"]
    if own:
        from paper_2609_23314_amd import vd
        return vd.vd_attention_mx4(vd.Mx4Cache(k, v, ks, vs), st["q"], st["n"])
    S, L, H, G, t, D, n = c["seqs"], c["layers"], c["heads"], c["group"], c["rows"], c["dim"], c["n"]
    q = st["q"].float().reshape(S, L, H, G * t, D) * D ** -0.5
    z = torch.matmul(q, _decode(k, ks).transpose(-1, -2)).view(S, L, H, G, t, n)
    # query row i, one of the newest t, sees the slots up to its own
    last = st["n_dev"].view(S, 1) - t + torch.arange(t, device=DEV)
    hide = torch.arange(n, device=DEV) > last.unsqueeze(-1)
    z.masked_fill_(hide.view(S, 1, 1, 1, t, n), -math.inf)
    z -= z.amax(-1, keepdim=True)
    w = z.exp_()
    w /= w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(S, L, H, G * t, n), _decode(v, vs))
    return out.view(S, L, H * G, t, D).to(DTYPE[c["dtype"]])


def _run_evict(st):
    """The scores, the mask, and the state: every byte of the cache and the token of each slot (rows are
    moved whole, so codes and scales are compared byte for byte)."""
    c, cache, pos = st["case"], st["cache"], st["pos"]
    S, L, H, n = c["seqs"], c["layers"], c["heads"], c["n"]
    U = S * L * H
    scores = torch.zeros((U, n), device=DEV)
    keep = torch.zeros((U, n), dtype=torch.uint8, device=DEV)
    if own:
        from paper_2609_23314_amd import vd
        vd.vd_evict_step_mx4(vd.Mx4Cache(*cache), st["n"], st["budget"], c["variant"], pos=pos, scores_out=scores, keep_out=keep)
        return [scores, keep, pos, *cache]
    i = 0 if c["variant"].startswith("key") else 1
    x = _decode(cache[i], cache[2 + i]).view(U, n, c["dim"]).double()     # scores next to the budget's border differ by little
    per = L * H
    nv, budget = [st[s].repeat_interleave(per).unsqueeze(-1) for s in ("n_dev", "budget_dev")]
    slot = torch.arange(n, device=DEV)
    valid = slot < nv
    mean = torch.where(valid.unsqueeze(-1), x, 0.0).sum(1, keepdim=True) / nv.unsqueeze(-1)
    form = c["variant"].replace("key_", "")
    if form == "dir":
        length = x.norm(dim=-1) * mean.norm(dim=-1)
        s = 1.0 - torch.where(length > 0, (x * mean).sum(-1) / torch.where(length > 0, length, 1.0), 0.0)
    else:
        s = (x - mean if form == "l2" else x).square().sum(-1).sqrt()
    scores = torch.where(valid, s.float(), 0.0)
    order = torch.where(valid, scores, -math.inf).sort(dim=-1, descending=True, stable=True).indices
    mask = torch.zeros_like(valid).scatter_(1, order, slot < budget) & valid
    # the k-th kept slot at or above the budget goes to the k-th evicted slot below it
    hu, hj = (~mask & (slot < torch.minimum(budget, nv))).nonzero(as_tuple=True)
    mu, mj = (mask & (slot >= budget)).nonzero(as_tuple=True)
    for y in (*cache, pos.view(S, L, H, n, 1)):
        flat = y.view(U, n, -1)
        flat[hu, hj] = flat[mu, mj]
    return [scores, mask.to(torch.uint8), pos, *cache]


# ------------------------------------------------------------------ the definitions, in 64 bits

def _values64(codes, scales):
    sign = torch.where((codes & 8) > 0, -1.0, 1.0).double()
    e, m = ((codes >> 1) & 3).double(), (codes & 1).double()
    size = torch.where(e > 0, torch.exp2(e - 1) * (1 + 0.5 * m), 0.5 * m)
    return sign * size * torch.exp2(scales.double() - 127).repeat_interleave(GROUP, -1)


def _unpack(x):
    y = torch.empty((*x.shape[:-1], 2 * x.shape[-1]), dtype=torch.uint8, device=x.device)
    y[..., 0::2], y[..., 1::2] = x & 15, x >> 4
    return y


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["kind"] == "rope":
        done = []
        for x, w in ((st["q"], st["q_weight"]), (st["k"], st["k_weight"])):
            y = x.double()
            if w is not None:
                y = y / (y.pow(2).sum(-1, keepdim=True) / c["dim"] + 1e-6).sqrt() * w.double().view(1, c["layers"], 1, 1, c["dim"])
            R = c["rotary"]
            i = torch.arange(R // 2, device=DEV)
            a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + R // 2)
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                               st["pos"].double()[:, None, None, :, None] * st["inv_freq"].double())
            z = torch.complex(y[..., a], y[..., b]) * turn
            y[..., a], y[..., b] = z.real, z.imag
            done.append(y)
        return done
    if c["kind"] == "append":
        done = []
        size = torch.tensor(_MAGNITUDES, dtype=torch.float64, device=DEV)
        middle = (size[1:] + size[:-1]) / 2
        for x in (st["k_rows"], st["v_rows"]):
            y = x.double().unflatten(-1, (-1, GROUP))
            top = y.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -130)
            unit = torch.exp2(torch.floor(torch.log2(top / 7 * (1 + 1e-12))) + 1).clamp(min=2.0 ** -127)
            r = y.abs() / unit
            low, high = torch.bucketize(r, middle, right=False), torch.bucketize(r, middle, right=True)
            at = torch.where(low % 2 == 0, low, high)     # they differ on a tie: the even one
            done.append((torch.copysign(size[at], y) * unit).flatten(-2))
        return done
    if c["kind"] == "attention":
        S, L, H, G, t, D, n = c["seqs"], c["layers"], c["heads"], c["group"], c["rows"], c["dim"], c["n"]
        q, done = st["q"].double(), torch.empty((S, L, H * G, t, D), dtype=torch.float64, device=DEV)
        k, v, ks, vs = st["cache"]
        for s in range(S):
            for layer in range(L):
                m = st["n"][s]
                kx, vx = _values64(_unpack(k[s, layer, :, :m]), ks[s, layer, :, :m]), _values64(_unpack(v[s, layer, :, :m]), vs[s, layer, :, :m])
                z = torch.matmul(q[s, layer].view(H, G * t, D), kx.transpose(1, 2).contiguous()).view(H, G, t, m) / math.sqrt(D)
                seen = torch.ones((t, m), dtype=torch.bool, device=DEV).tril(m - t)
                p = torch.softmax(torch.where(seen, z, -math.inf), -1)
                done[s, layer] = torch.matmul(p.view(H, G * t, m), vx).reshape(H * G, t, D)
        return done
    # the scores; whole numbers have no such value
    S, L, H, n = c["seqs"], c["layers"], c["heads"], c["n"]
    i = 0 if c["variant"].startswith("key") else 1
    done = torch.zeros((S, L, H, n), dtype=torch.float64, device=DEV)
    for s in range(S):
        for layer in range(L):
            m = st["n"][s]
            x = _values64(_unpack(st["cache"][i][s, layer, :, :m]), st["cache"][2 + i][s, layer, :, :m])
            mean = x.mean(1, keepdim=True)
            if c["variant"].endswith("dir"):
                u = x / x.norm(dim=-1, keepdim=True).clamp(min=1e-300)
                w = mean / mean.norm(dim=-1, keepdim=True).clamp(min=1e-300)
                d = 1 - (u * w).sum(-1)
            else:
                d = (x if c["variant"].endswith("norm") else x - mean).norm(dim=-1)
            done[s, layer, :, :m] = d
    return [done.view(S * L * H, n), None, None, None, None, None, None]
