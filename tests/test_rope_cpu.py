"""Rotary positions and query/key norms without a GPU: the position table, and
what the C ABI refuses before any HIP call."""
import ctypes
import math

import numpy as np
import pytest
import torch

FAKE = 0x10000  # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def L():
    from paper_2608_12032_amd import losa
    return losa


@pytest.mark.parametrize("dims,lens,base", [
    ((128,), (5000,), 10000.0), ((44, 42, 42), (21, 30, 52), 10000.0), ((2, 6), (1, 7), 256.0),
    ((64,), (300_000,), 500_000.0)])
def test_table_is_cos_sin_of_the_angles(L, dims, lens, base):
    """Angles in fp64 and one rounding: half a step of fp32 (2^-24, values are at most
    1) plus what an fp64 angle of up to 3e5 can be off by (2^-53 of it, a few times)."""
    t = L.losa_rope_table(dims, lens, base, device="cpu")
    assert t.axis_dim == dims and t.axis_len == lens and t.data.dtype == torch.float32
    off = 0
    for dim, n in zip(dims, lens):
        got = t.data[off:off + n * dim].view(n, dim // 2, 2).double().numpy()
        off += n * dim
        j = np.arange(dim // 2)
        angle = np.arange(n)[:, None] * np.power(base, -2.0 * j / dim)[None, :]
        assert np.abs(got[..., 0] - np.cos(angle)).max() <= 2.0 ** -24 + 2.0 ** -31
        assert np.abs(got[..., 1] - np.sin(angle)).max() <= 2.0 ** -24 + 2.0 ** -31
    assert off == t.data.numel()


@pytest.mark.parametrize("dims,lens,base,status", [
    ((), (), 1e4, 2), ((2,) * 5, (3,) * 5, 1e4, 2), ((3,), (4,), 1e4, 2), ((0,), (4,), 1e4, 2),
    ((4,), (0,), 1e4, 2), ((4,), (4,), 0.0, 2), ((4,), (4,), math.nan, 2), ((4,), (4,), math.inf, 2)])
def test_table_refusals(L, dims, lens, base, status):
    with pytest.raises(L.LosaError) as e:
        L.losa_rope_table(dims, lens, base, device="cpu")
    assert e.value.status == status


def test_a_table_holds_its_positions(L):
    for data in (torch.zeros(75), torch.zeros(76, dtype=torch.float64), torch.zeros(152)[::2]):
        with pytest.raises(ValueError, match="76 elements"):
            L.RopeTable(data, (4, 6), (7, 8))
    with pytest.raises(AttributeError):
        L.RopeTable(torch.zeros(76), (4, 6), (7, 8)).data = torch.zeros(1)


def test_table_capacity(L):
    room = (ctypes.c_float * 8)()
    one = lambda *x: (ctypes.c_int * len(x))(*x)  # noqa: E731
    assert L.lib.losa_rope_table(1, one(4), one(3), 1e4, room, 11) == 6
    assert L.lib.losa_rope_table(1, one(4), one(3), 1e4, None, 12) == 1
    # 2^31 floats: beyond the kernels' 32-bit table index
    assert L.lib.losa_rope_table(1, one(1 << 10), one(1 << 21), 1e4, room, 1 << 40) == 2


class View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64),
                ("head", ctypes.c_int64)]


class Rotation(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int), ("axis_dim", ctypes.c_int * 4),
                ("axis_len", ctypes.c_int * 4), ("table", ctypes.c_void_p),
                ("pos", ctypes.c_void_p), ("pos_batch", ctypes.c_int64), ("pairs", ctypes.c_int)]


class QkNorm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("all_heads", ctypes.c_int), ("eps", ctypes.c_float),
                ("q_weight", ctypes.c_void_p), ("q_bias", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("k_bias", ctypes.c_void_p)]


def test_structures_are_packed_as_c_lays_them_out(L):
    """The binding passes structures as bytes: the layout a C compiler gives them."""
    ints = ctypes.c_int * 4
    assert bytes(View(1 << 40, 2, 3, 4)) == L._VIEW(1 << 40, 2, 3, 4)
    t = L.RopeTable(torch.zeros(76), (4, 6), (7, 8))
    assert bytes(Rotation(2, ints(4, 6), ints(7, 8), 1 << 33, 1 << 34, 9, 1)) == \
        t._head + L._ROTATION(1 << 33, 1 << 34, 9, 1)
    assert bytes(QkNorm(2, 1, 0.5, 1 << 33, None, 8, 1 << 50)) == \
        L._QK_NORM(2, True, 0.5, 1 << 33, 0, 8, 1 << 50)


def rotation(L, **kw):
    a = dict(n_axes=3, dim=(44, 42, 42, 0), len=(21, 30, 52, 0), table=FAKE, pos=FAKE, pos_batch=0,
             pairs=0)
    a.update(kw)
    return Rotation(a["n_axes"], (ctypes.c_int * 4)(*a["dim"]), (ctypes.c_int * 4)(*a["len"]),
                       a["table"], a["pos"], a["pos_batch"], a["pairs"])


def view(L, data=FAKE, batch=100 * 512, token=512, head=128):
    return View(data, batch, token, head)


def rope(L, x=None, y=None, rot=None, dtype=1, B=2, N=100, N_pad=100, H=4, d=128, **kw):
    x = view(L) if x is None else x
    y = view(L) if y is None else y
    rot = rotation(L, **kw) if rot is None else rot
    at = lambda s: None if s == 0 else ctypes.addressof(s)  # noqa: E731
    return L.lib.losa_rope(at(x), dtype, B, N, N_pad, H, d, at(rot), at(y), None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=0), 1), (dict(y=0), 1), (dict(rot=0), 1), (dict(table=None), 1), (dict(pos=None), 1),
    (dict(B=0), 2), (dict(N=0), 2), (dict(H=-1), 2), (dict(N_pad=99), 2), (dict(d=0), 2),
    (dict(d=96), 5), (dict(dtype=7), 5), (dict(pairs=2), 5), (dict(n_axes=0), 2),
    (dict(n_axes=5), 2), (dict(dim=(43, 42, 42, 0)), 2), (dict(dim=(64, 42, 42, 0)), 2),
    (dict(dim=(42, 42, 42, 0)), 2),                         # 126: no multiple of 8
    (dict(len=(21, 0, 52, 0)), 2), (dict(table=FAKE + 4), 4), (dict(pos=FAKE + 2), 4),
    (dict(pos_batch=-1), 2), (dict(pos_batch=299), 2), (dict(N_pad=(1 << 30) + 1), 2),
])
def test_rope_refusals(L, kw, code):
    assert rope(L, **kw) == code
    assert L.lib.losa_last_error().decode() != ""


@pytest.mark.parametrize("which", ["x", "y"])
@pytest.mark.parametrize("kw,code", [
    (dict(data=0), 1), (dict(data=FAKE + 8), 4), (dict(token=-512), 2), (dict(head=132), 4),
    (dict(token=1 << 41), 2)])
def test_view_refusals(L, which, kw, code):
    assert rope(L, **{which: view(L, **kw)}) == code


@pytest.mark.parametrize("kw", [dict(batch=0), dict(token=0), dict(head=0), dict(head=64)])
def test_overlapping_output_rows_are_refused(L, kw):
    assert rope(L, y=view(L, **kw)) == 2


@pytest.mark.parametrize("kw", [
    dict(token=128, head=256),          # heads of one token over those of the next
    dict(batch=99 * 512 + 384), dict(token=512, head=256, batch=100 * 512),
    dict(token=1 << 39, head=1 << 39, batch=1 << 39)])
def test_rows_that_step_into_each_other_are_refused(L, kw):
    assert rope(L, y=view(L, **kw)) == 2
    assert "overlap" in L.lib.losa_last_error().decode()


def test_outputs_over_other_tensors_are_refused(L):
    """An output may be its own input, the same view; nothing else starts where it does."""
    head_major = dict(batch=100 * 512, token=128, head=100 * 128)
    assert rope(L, y=view(L, **head_major)) == 2 and "same view" in L.lib.losa_last_error().decode()
    assert rope(L, N_pad=128, x=view(L, batch=128 * 512), y=view(L, batch=128 * 512)) == 2
    at = [view(L, data=FAKE + (i << 24)) for i in range(6)]
    for kw in (dict(qo=at[1]), dict(ko=at[0]), dict(vo=at[1]), dict(qo=at[4]), dict(ko=at[5]),
               dict(vo=view(L, data=at[2].data, **head_major)), dict(vo=at[2], N_pad=128)):
        n_pad = kw.get("N_pad", 100)
        t = dict(zip(("q", "k", "v", "qo", "ko", "vo"), at))
        if n_pad == 128:
            t = {x: View(y.data, 128 * 512, y.token, y.head) for x, y in t.items()}
        t.update(kw)
        assert qkn(L, **t) == 2, kw


def norms(L, kind=1, all_heads=0, eps=1e-6, qw=None, qb=None, kw=None, kb=None):
    return QkNorm(kind, all_heads, eps, qw, qb, kw, kb)


def qkn(L, q=1, k=1, v=1, qo=1, ko=1, vo=1, norm=None, rot=1, dtype=1, H=4, Hkv=2, d=128, N_pad=100):
    pick = lambda s: view(L) if isinstance(s, int) and s == 1 else s  # noqa: E731
    keep = [pick(s) for s in (q, k, v, qo, ko, vo)]
    norm = norms(L) if norm is None else norm
    rot = rotation(L) if isinstance(rot, int) and rot == 1 else rot
    at = lambda s: None if isinstance(s, int) and s == 0 else ctypes.addressof(s)  # noqa: E731
    q, k, v, qo, ko, vo = (at(s) for s in keep)
    return L.lib.losa_qk_norm_rope(q, k, v, dtype, 2, 100, N_pad, H, Hkv, d, at(norm), at(rot), qo,
                                   ko, vo, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=0), 1), (dict(k=0), 1), (dict(qo=0), 1), (dict(ko=0), 1), (dict(v=0), 1),
    (dict(vo=0), 1), (dict(Hkv=0), 2), (dict(H=0), 2), (dict(N_pad=3), 2), (dict(d=32), 5),
    (dict(dtype=-3), 5)])
def test_qk_norm_rope_refusals(L, kw, code):
    assert qkn(L, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(kind=0), 5), (dict(kind=3), 5), (dict(eps=-1e-6), 2), (dict(eps=math.nan), 2),
    (dict(eps=math.inf), 2), (dict(qw=FAKE + 4), 4), (dict(kb=FAKE + 8), 4)])
def test_norm_refusals(L, kw, code):
    assert qkn(L, norm=norms(L, **kw)) == code


def test_binding_refuses_host_tensors(L):
    x = torch.zeros((1, 4, 2, 64))
    t = L.losa_rope_table((64,), (4,), device="cpu")
    pos = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(ValueError, match="must live on"):
        L.losa_rope(x, t, pos)
    with pytest.raises(ValueError, match="must live on"):
        L.losa_qk_norm_rope(x, x)
    with pytest.raises(ValueError, match="same length"):
        L.losa_rope_table((64,), (4, 4), device="cpu")


def test_a_call_beyond_one_launch_is_refused(L):
    """2^24 workgroups of 256 threads: a launch counts its threads in 32 bits.  (Each batch
    takes one workgroup here; with q, k and v a third of them is enough.)"""
    n, one = 1 << 24, dict(batch=128, token=128, head=128)
    far = dict(one, data=FAKE + (1 << 33))
    assert rope(L, x=view(L, **one), y=view(L, **far), B=n, N=1, N_pad=1, H=1) == 2
    assert "more workgroups than one launch takes" in L.lib.losa_last_error().decode()
    x = [View(FAKE + (i << 33), 128, 128, 128) for i in range(6)]
    at = [ctypes.addressof(v) for v in x]
    norm = norms(L)
    assert L.lib.losa_qk_norm_rope(*at[:3], 1, n // 3 + 1, 1, 1, 1, 1, 128, ctypes.addressof(norm), None,
                                   *at[3:], None) == 2
    assert "more workgroups than one launch takes" in L.lib.losa_last_error().decode()
