"""The 4-bit cache and the rotated rows without a GPU: what the calls refuse (all
before any HIP call), the host side under the sanitizers, and the kernels' code."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import mx4_ref as ref
from paper_2609_23314_amd import build as lib_build
from paper_2609_23314_amd import vd
from test_sanitizers import HERE, ROCM_INCLUDE, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2609_23314_amd", "csrc")
FAKE = 0x7F0000000000   # never dereferenced: validation fails first
INVALID, UNSUPPORTED, WORKSPACE = vd.VD_ERR_INVALID_ARG, vd.VD_ERR_UNSUPPORTED, vd.VD_ERR_WORKSPACE


def _cache(**kw):
    """2 sequences, 3 layers, 4 KV heads, 16 query heads, 100 slots of 128 channels."""
    c = vd.VdMx4Cache(FAKE, FAKE + 0x100000, FAKE + 0x200000, FAKE + 0x300000, 2, 3, 4, 16, 128, 100,
                      76800, 25600, 6400, 64, 4800, 1600, 400, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _ints(x):
    return None if x is None else (ctypes.c_int32 * len(x))(*x)


def _longs(x):
    return None if x is None else (ctypes.c_int64 * len(x))(*x)


ROWS = FAKE + 0x1000000
ROW_STRIDES = (3 * 4 * 8 * 128, 4 * 8 * 128, 8 * 128, 128)
Q_STRIDES = (3 * 16 * 8 * 128, 16 * 8 * 128, 8 * 128, 128)


def _append(c, fn="vd_append_mx4", n_old=(4, 90), rows=(8, 8), max_rows=8, dtype=0, k=ROWS, ks=ROW_STRIDES, v=ROWS + 0x1000000,
            vs=ROW_STRIDES, pos=None, pos0=None):
    head = (ctypes.byref(c) if c is not None else None, _ints(n_old), _ints(rows), max_rows, dtype, k, _longs(ks), v, _longs(vs))
    return vd.load().vd_append_mx4(*head, pos, _ints(pos0), None) if fn == "vd_append_mx4" else vd.load().vd_read_mx4(*head, None)


def _attend(c, dtype=0, q=ROWS, qs=Q_STRIDES, max_rows=8, rows=(8, 8), scale=0.1, n=(50, 0), out=ROWS + 0x1000000, os_=Q_STRIDES,
            ws=None, ws_bytes=0):
    return vd.load().vd_attention_mx4(ctypes.byref(c) if c is not None else None, dtype, q, _longs(qs), max_rows, _ints(rows),
                                      scale, _ints(n), out, _longs(os_), ws, ws_bytes, None)


def _evict(c, n=(50, 60), N=(40, 40), variant=0, pos=None, scores=None, keep=None):
    return vd.load().vd_evict_step_mx4(ctypes.byref(c) if c is not None else None, _ints(n), _ints(N), variant, pos, scores, keep, None)


@pytest.mark.parametrize("call", [_append, lambda c: _append(c, "vd_read_mx4"), _attend, _evict])
@pytest.mark.parametrize("field,value,status", [
    ("k", None, INVALID), ("v", None, INVALID), ("k_scale", None, INVALID), ("v_scale", None, INVALID),
    ("num_seqs", 0, INVALID), ("num_layers", -1, INVALID), ("num_kv_heads", 0, INVALID), ("num_q_heads", 6, INVALID),
    ("head_dim", 96, UNSUPPORTED), ("head_dim", 0, INVALID), ("capacity", 0, INVALID), ("capacity", (1 << 24) + 1, UNSUPPORTED),
    ("k", FAKE + 8, INVALID), ("v", FAKE, INVALID), ("v_scale", FAKE + 0x200000, INVALID), ("k_scale", FAKE + 0x200002, INVALID),
    ("stride_slot", 48, INVALID), ("stride_slot", 72, INVALID), ("stride_head", -64, INVALID), ("stride_head", 6408, INVALID),
    ("scale_slot", 2, INVALID), ("scale_slot", 6, INVALID), ("scale_layer", -4, INVALID), ("scale_head", 402, INVALID),
    ("stride_slot", 1 << 26, UNSUPPORTED), ("stride_seq", 1 << 62, UNSUPPORTED), ("scale_seq", 1 << 60, UNSUPPORTED),
])
def test_cache_refused(call, field, value, status):
    assert call(_cache(**{field: value})) == status


def test_no_cache():
    assert _append(None) == _append(None, "vd_read_mx4") == _attend(None) == _evict(None) == INVALID


@pytest.mark.parametrize("stride", ["stride_seq", "stride_layer", "stride_head", "scale_seq", "scale_layer", "scale_head"])
def test_writers_refuse_units_that_share_memory(stride):
    c = _cache(**{stride: 0})
    assert _append(c) == _evict(c) == INVALID
    assert _attend(c, scale=float("nan")) == INVALID      # (readers may: it gets to the next check)


@pytest.mark.parametrize("fn", ["vd_append_mx4", "vd_read_mx4"])
@pytest.mark.parametrize("bad", [
    dict(n_old=None), dict(n_old=(-1, 0)), dict(n_old=(93, 0)), dict(rows=(9, 0)), dict(rows=(-1, 0)), dict(max_rows=0),
    dict(rows=None, n_old=(0, 93)), dict(dtype=2), dict(k=None), dict(v=None), dict(ks=None), dict(k=ROWS + 8),
    dict(ks=(3 * 4 * 8 * 128, 4 * 8 * 128, 8 * 128, 132)), dict(vs=(-128, 4 * 8 * 128, 8 * 128, 128)),
    dict(ks=(1 << 60, 0, 0, 128)), dict(k=FAKE + 16), dict(v=FAKE + 0x300000)])
def test_rows_refused(fn, bad):
    assert _append(_cache(), fn, **bad) == INVALID


def test_append_positions_refused():
    pos = FAKE + 0x4000000
    assert _append(_cache(), pos=pos + 2) == INVALID
    assert _append(_cache(), pos=pos, pos0=(-1, 0)) == INVALID
    assert _append(_cache(), pos=pos, pos0=(2 ** 31 - 8, 0)) == INVALID


def test_read_refuses_outputs_that_share_memory():
    assert _append(_cache(), "vd_read_mx4", v=ROWS) == INVALID
    assert _append(_cache(), "vd_read_mx4", ks=(3 * 4 * 8 * 128, 0, 8 * 128, 128)) == INVALID


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(max_rows=0), dict(rows=(9, 0)), dict(rows=(-1, 0)), dict(n=None), dict(n=(101, 0)), dict(n=(-1, 0)),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(q=None), dict(out=None), dict(qs=None), dict(q=ROWS + 4),
    dict(out=ROWS), dict(out=FAKE), dict(os_=(3 * 16 * 8 * 128, 16 * 8 * 128, 8 * 128, 0)),
    dict(qs=(3 * 16 * 8 * 128, 16 * 8 * 128, 8 * 128, 100))])
def test_attention_refused(bad):
    assert _attend(_cache(), **bad) == INVALID


def test_attention_limits_and_workspace():
    assert _attend(_cache(), max_rows=2 ** 28) == UNSUPPORTED
    size = vd.load().vd_attention_mx4_workspace_size
    c = _cache(num_seqs=1, num_layers=1, num_kv_heads=1, num_q_heads=4, capacity=8192)
    sizes = [size(ctypes.byref(c), 0, 1, n) for n in (0, 1, 100, 511, 512, 2000, 4000, 8192)]
    assert sizes[0] == 0 and sizes == sorted(sizes) and sizes[-1] > 0
    many = dict(n=(8000,), rows=(1,), max_rows=1)
    for ws, b in ((None, 1 << 40), (FAKE + 0x5000008, 1 << 40), (FAKE + 0x5000000, size(ctypes.byref(c), 0, 1, 8000) - 1)):
        assert _attend(c, ws=ws, ws_bytes=b, **many) == WORKSPACE
    assert size(ctypes.byref(c), 0, 1, 8193) == size(ctypes.byref(c), 0, 1, -1) == size(ctypes.byref(c), 5, 1, 10) == 0
    assert size(ctypes.byref(c), 0, 0, 10) == size(ctypes.byref(_cache(head_dim=96)), 0, 1, 10) == 0


@pytest.mark.parametrize("bad", [dict(n=None), dict(N=None), dict(n=(101, 5)), dict(n=(-1, 5)), dict(N=(0, 5)), dict(variant=6),
                                 dict(variant=-1), dict(pos=FAKE + 2), dict(scores=FAKE + 2)])
def test_evict_refused(bad):
    assert _evict(_cache(), **bad) == INVALID


def test_evict_capacity():
    assert _evict(_cache(capacity=vd.MAX_CAPACITY + 1)) == UNSUPPORTED


def _rope(**kw):
    """2 sequences, 3 layers, 4 + 2 heads, 8 rows of 128 channels."""
    a = vd.VdRopeArgs()
    for side, heads, at in ((a.q, 4, 0), (a.k, 2, 0x4000000)):
        side.x, side.out, side.weight, side.heads, side.out_dtype = ROWS + at, ROWS + at + 0x2000000, FAKE, heads, 0
        for st in (side.strides, side.out_strides):
            st[:] = (3 * heads * 8 * 128, heads * 8 * 128, 8 * 128, 128)
    a.pos, a.inv_freq, a.dtype, a.weight_dtype = FAKE, FAKE, 0, 1
    a.num_seqs, a.num_layers, a.rows, a.head_dim, a.rotary, a.interleaved, a.eps = 2, 3, 8, 128, 64, 0, 1e-6
    for k, v in kw.items():
        side, _, field = k.partition("_") if k[:2] in ("q_", "k_") else ("", "", k)
        setattr(getattr(a, side) if side else a, field, v)
    return vd.load().vd_qk_norm_rope(ctypes.byref(a), None)


@pytest.mark.parametrize("bad,status", [
    (dict(q_x=None, q_out=None, k_x=None, k_out=None), INVALID), (dict(q_x=None), INVALID), (dict(q_out=None), INVALID),
    (dict(pos=None), INVALID), (dict(pos=FAKE + 2), INVALID), (dict(inv_freq=None), INVALID), (dict(inv_freq=FAKE + 8), INVALID),
    (dict(dtype=3), INVALID), (dict(weight_dtype=3), INVALID), (dict(q_out_dtype=2), INVALID), (dict(k_heads=0), INVALID),
    (dict(num_seqs=0), INVALID), (dict(num_layers=0), INVALID), (dict(rows=0), INVALID), (dict(head_dim=0), INVALID),
    (dict(head_dim=96), UNSUPPORTED), (dict(rotary=0), INVALID), (dict(rotary=12), INVALID), (dict(rotary=136), INVALID),
    (dict(interleaved=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(q_weight=FAKE + 8), INVALID),
    (dict(q_x=ROWS + 8), INVALID), (dict(k_strides=(6144, 2048, 1024, 100)), INVALID), (dict(k_strides=(-128, 2048, 1024, 128)), INVALID),
    (dict(q_out_strides=(0, 4096, 1024, 128)), INVALID),                     # sequences written onto each other
    (dict(q_out=ROWS + 16), INVALID),                                        # an output that overlaps its input
    (dict(q_out=ROWS, q_out_dtype=1), INVALID),                              # in place, but of another type
    (dict(k_out=ROWS + 0x2000000), INVALID),                                 # both sides' outputs
])
def test_rope_refused(bad, status):
    for key, value in bad.items():
        if isinstance(value, tuple):
            bad = {**bad, key: (ctypes.c_int64 * 4)(*value)}
    assert _rope(**bad) == status


def test_binding_refuses_on_the_host():
    x = torch.zeros(1, 1, 2, 3, 64)
    cpu = vd.Mx4Cache.zeros(1, 1, 2, 8, 64, device="cpu")
    for call in (lambda: vd.vd_append_mx4(cpu, [0], x, x), lambda: vd.vd_read_mx4(cpu, [0], 1), lambda: vd.vd_attention_mx4(cpu, x, [1]),
                 lambda: vd.vd_evict_step_mx4(cpu, [1], [1])):
        with pytest.raises(ValueError, match="on one GPU"):
            call()
    with pytest.raises(ValueError, match="on a GPU"):
        vd.vd_qk_norm_rope(x, None, torch.zeros(1, 3, dtype=torch.int32), torch.ones(32))
    g = x.clone().requires_grad_()
    for call in (lambda: vd.vd_append_mx4(cpu, [0], g, x), lambda: vd.vd_attention_mx4(cpu, g, [1]),
                 lambda: vd.vd_qk_norm_rope(g, None, torch.zeros(1, 3, dtype=torch.int32), torch.ones(32))):
        with pytest.raises(ValueError, match="no gradient"):
            call()
    for bad in (cpu._replace(v=cpu.v[:, :, :, :4]), cpu._replace(v_scale=cpu.v_scale[:, :1]), cpu._replace(k=cpu.k[0]),
                cpu._replace(k=cpu.k[..., :24], v=cpu.v[..., :24]), cpu._replace(v=cpu.v.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises(ValueError):
            vd.mx4_desc(bad)
    with pytest.raises(IndexError):
        cpu.seq(1)
    with pytest.raises(IndexError):
        cpu.seq(-1)


def test_format_by_hand():
    """The reference's own format, on values whose codes can be said."""
    x = torch.zeros(1, 32)
    x[0, :10] = torch.tensor([6.0, -0.5, 0.25, 0.75, 5.0, -6.9, 3.5, 1.0, -0.0, 2.5])
    codes, scales = ref.encode(x)
    assert scales.tolist() == [[127]] and codes[0, :5].tolist() == [0x97, 0x20, 0xF6, 0x26, 0x48]
    assert ref.decode(codes, scales)[0, :10].tolist() == [6.0, -0.5, 0.0, 1.0, 4.0, -6.0, 4.0, 1.0, 0.0, 2.0]
    x[0, 0] = 7.0            # at seven the scale doubles
    assert ref.encode(x)[1].tolist() == [[128]]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_host_under_sanitizers(tmp_path):
    exe = str(tmp_path / "mx4_san")
    _run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
          "-o", exe, os.path.join(HERE, "sanitize", "mx4_main.cpp"), os.path.join(CSRC, "vd_mx4.cpp")])
    assert "mx4 sanitizer run ok" in _run([exe], env={**os.environ, "ASAN_OPTIONS": "detect_leaks=1"}, timeout=300)


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = {}
    for name in ("vd_mx4", "vd_rope"):
        path = tmp_path_factory.mktemp("asm") / (name + ".s")
        subprocess.run([lib_build.hipcc(), f"--offload-arch={lib_build.ARCH}", "--cuda-device-only", "-S", "-O3", "-std=c++17",
                        "-I", os.path.join(ROOT, "include"), "-I", CSRC, *lib_build.DEVICE_FLAGS,
                        os.path.join(CSRC, name + ".hip"), "-o", str(path)], check=True, capture_output=True)
        out[name] = path.read_text()
    return out


@pytest.mark.parametrize("name", ["vd_mx4", "vd_rope"])
def test_code_has_no_calls_flat_accesses_or_stack(assembly, name):
    text = assembly[name]
    assert "s_swappc" not in text
    assert not re.findall(r"^\s*(flat_\w+)", text, flags=re.M)
    assert not re.findall(r"v_pk_(?:add|mul|fma)_f32", text)
    sizes = dict(re.findall(r"\.amdhsa_kernel (\S+)\n(?:.*\n)*?\s*\.amdhsa_private_segment_fixed_size (\d+)", text))
    assert len(sizes) >= 12 and set(sizes.values()) == {"0"}, {k: v for k, v in sizes.items() if v != "0"}


def test_registers_leave_the_workgroups_their_place(assembly):
    """512 registers of a SIMD lane, in steps of 8: the eviction's workgroups of 1024 threads
    (or two of 512) need 128, the attention's blocks of bf16 queries up to 128 channels 256."""
    regs = dict(re.findall(r"\.amdhsa_kernel (\S+)\n(?:.*\n)*?\s*\.amdhsa_next_free_vgpr (\d+)", assembly["vd_mx4"]))
    for part, limit, count in (("evict_kernel", 128, 18), ("attn_block_kernelILi0ELi64", 256, 1), ("attn_block_kernelILi0ELi128", 256, 1),
                               ("attn_kernelILi0ELi128", 128, 1), ("attn_kernelILi1ELi128", 168, 1)):
        some = {k: int(v) for k, v in regs.items() if part in k}
        assert len(some) == count and max(some.values()) <= limit, some
