"""The plan of the packed attention without a GPU (its units cover every row and key
once, whatever the batch), and what the C ABI refuses before any HIP call."""
import copy
import ctypes
import pickle
import random

import numpy as np
import pytest
import torch

FAKE = 0x10000  # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def L():
    from paper_2608_12032_amd import losa
    return losa


ITEM = np.dtype([("q_row", "<i8"), ("k_row", "<i8"), ("head0", "<i4"), ("rows", "<i4"), ("keys", "<i4"),
                 ("seen", "<i4"), ("part", "<i4"), ("split", "<i4")])
JOIN = np.dtype([("q_row", "<i8"), ("in_group", "<i4"), ("part", "<i4"), ("step", "<i4"), ("n", "<i4")])


def units(plan):
    raw = plan.data.numpy().tobytes()[:plan.info.bytes]
    n = plan.info.n_tiles + plan.info.n_few
    items = np.frombuffer(raw[:n * ITEM.itemsize], ITEM)
    return items[:plan.info.n_tiles], items[plan.info.n_tiles:], np.frombuffer(raw[n * ITEM.itemsize:], JOIN)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_units_cover_every_row_and_key_once(L, dtype, causal, seed):
    rng = random.Random(seed)
    G = rng.choice([1, 2, 3, 8])
    ql = [rng.choice([0, 1, 2, 5, 33, 128, 129, 400]) for _ in range(7)]
    kl = [rng.choice([0, 1, 63, 128, 129, 700, 5000, 50_000]) for _ in ql]
    p = L.losa_packed_plan(ql, kl, 2 * G, 2, dtype, causal=causal, device="cpu")
    tiles, few, joins = units(p)
    most = 32 if dtype == torch.bfloat16 else 16
    assert p.info.tile_rows in ((128,) if dtype == torch.bfloat16 else (16, 32))
    assert p.q_rows == max([0] + [sum(ql[:i + 1]) for i in range(7) if ql[i]])
    parts = []
    q0 = k0 = 0
    for q, k in zip(ql, kl):
        rows, shift = q * G, k - q
        sees = lambda t: max(0, min(k, t + shift + 1)) if causal else k  # noqa: E731
        mine = [x for x in (tiles if rows > most else few) if q0 <= x["q_row"] < q0 + q]
        block = p.info.tile_rows
        if dtype == torch.float32:  # the fewer keys, the more of a workgroup's waves have rows of their own
            split = 3 if rows <= most else sum(k > n for n in (32, 64, 128))
            assert all(x["split"] == split for x in mine)
            block = block * 8 >> split
        number = lambda x: (int(x["q_row"]) - q0) * G + int(x["head0"])  # noqa: E731
        for x in mine:
            assert int(x["rows"]) == rows - number(x)
            if x["keys"]:
                assert k0 <= x["k_row"] and x["k_row"] + x["keys"] <= k0 + k
            else:
                assert x["k_row"] == 0
            # each row's keys, as the kernels read them, are those of the formula that the
            # unit's range holds
            c0 = int(x["k_row"]) - k0 if x["keys"] else 0
            for r in (0, min(block, int(x["rows"])) - 1):
                t = (int(x["head0"]) + r) // G
                tok = int(x["q_row"]) - q0 + t
                assert max(0, min(int(x["keys"]), int(x["seen"]) + t)) == \
                    max(0, min(c0 + int(x["keys"]), sees(tok)) - c0)
        # a tile's or a few-row sequence's keys, part after part
        by_row = {}
        for x in mine:
            by_row.setdefault(number(x), []).append(x)
        assert sorted(by_row) == (list(range(0, rows, block)) if rows > most else [0][:rows])
        n = firsts = None
        for r, those in by_row.items():
            those.sort(key=lambda x: x["part"])
            last = min(q - 1, (r + block - 1) // G)
            assert sum(int(x["keys"]) for x in those) == (sees(last) if rows > most else k)
            held = [x for x in those if x["keys"]]
            assert not held or held[0]["k_row"] == k0
            assert all(a["k_row"] + a["keys"] == b["k_row"] for a, b in zip(held, held[1:]))
            assert n in (None, len(those)) and len(those) <= 256
            n = len(those)
            if n == 1:
                assert those[0]["part"] == -1
            else:
                at = [int(x["part"]) - r for x in those]
                assert firsts in (None, at[0]) and at == [at[0] + i * rows for i in range(n)]
                firsts = at[0]
        if n is not None and n > 1:
            got = [j for j in joins if q0 <= j["q_row"] < q0 + q]
            assert sorted((int(j["q_row"]) - q0) * G + int(j["in_group"]) for j in got) == list(range(rows))
            for j in got:
                r = (int(j["q_row"]) - q0) * G + int(j["in_group"])
                assert (j["part"], j["step"], j["n"]) == (firsts + r, rows, n)
            parts.append((firsts, firsts + n * rows))
        q0, k0 = q0 + q, k0 + k
    parts.sort()
    assert sum(b - a for a, b in parts) == p.info.part_rows
    assert all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
    for x in (tiles, few):  # longest first
        n = [int(y["keys"]) for y in x]
        assert n == sorted(n, reverse=True)
    assert p.workspace_bytes(128) == p.info.part_rows * 2 * 130 * 4


def test_a_sequence_is_split_alike_in_any_batch(L):
    alone = units(L.losa_packed_plan([3], [9000], 8, 2, torch.bfloat16, device="cpu"))[1]
    among = units(L.losa_packed_plan([500, 3, 1], [20, 9000, 40_000], 8, 2, torch.bfloat16, device="cpu"))[1]
    cut = lambda x, k0: sorted((int(y["k_row"]) - k0, int(y["keys"])) for y in x  # noqa: E731
                               if k0 <= y["k_row"] < k0 + 9000)
    assert cut(alone, 0) == cut(among, 20) and len(alone) > 1


def test_nothing_to_do(L):
    p = L.losa_packed_plan([], [], 4, 4, torch.float32, device="cpu")
    assert (p.info.bytes, p.q_rows, p.k_rows, p.workspace_bytes(64)) == (0, 0, 0, 0)
    p = L.losa_packed_plan([0, 0], [5, 0], 4, 4, torch.bfloat16, causal=True, device="cpu")
    assert p.info.bytes == 0 and p.k_rows == 0


@pytest.mark.parametrize("kw,status", [
    (dict(heads=0), 2), (dict(kv_heads=0), 2), (dict(heads=5, kv_heads=2), 2),
    (dict(q_lens=[3, -1]), 2), (dict(k_lens=[3, -1]), 2), (dict(k_starts=[0, -4]), 2),
    (dict(q_starts=[0, 2]), 2),                     # rows 2 of q belong to both
    (dict(q_starts=[7, 5]), 2), (dict(q_lens=[1 << 30, 1 << 30], heads=4, kv_heads=2), 2),
    (dict(q_starts=[0, 1 << 41]), 2), (dict(q_lens=[(1 << 30) + 1, 3]), 2),
    # more workgroups than a launch takes
    (dict(q_lens=[1 << 30, 3], heads=1 << 9, kv_heads=1 << 9), 2)])
def test_plan_refusals(L, kw, status):
    args = dict(q_lens=[3, 3], k_lens=[5, 5], heads=4, kv_heads=2, dtype=torch.bfloat16, device="cpu")
    args.update(kw)
    with pytest.raises(L.LosaError) as e:
        L.losa_packed_plan(**args)
    assert e.value.status == status and str(e.value)


def test_plan_argument_checks(L):
    with pytest.raises(TypeError, match="dtype"):
        L.losa_packed_plan([1], [1], 1, 1, torch.float16, device="cpu")
    with pytest.raises(ValueError, match="entries"):
        L.losa_packed_plan([1], [1, 2], 1, 1, torch.float32, device="cpu")
    with pytest.raises(ValueError, match="32 bits"):
        L.losa_packed_plan([1 << 31], [1], 1, 1, torch.float32, device="cpu")
    info = L._PackedInfo()
    one = (ctypes.c_int32 * 1)(4)
    call = lambda **k: L.lib.losa_packed_plan(  # noqa: E731
        None, k.get("q", one), None, one, k.get("n", 1), k.get("dtype", 1), 2, 1, 0, k.get("plan"),
        k.get("room", 0), k.get("info", ctypes.addressof(info)))
    assert call() == 0 and info.bytes == ITEM.itemsize
    assert call(info=None) == 1 and call(q=None) == 1 and call(n=-1) == 2 and call(dtype=9) == 5
    room = (ctypes.c_int64 * 8)()
    at = ctypes.addressof(room)
    assert call(plan=at, room=ITEM.itemsize - 1) == 6 and call(plan=at + 4, room=64) == 4
    assert call(plan=at, room=64) == 0


class View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64),
                ("head", ctypes.c_int64)]


def view(L, data=FAKE, token=512, head=128):
    return View(data, 0, token, head)


def fwd(L, q=1, k=1, v=1, o=1, q_rows=40, k_rows=4000, plan=FAKE, d=128, scale=0.1, lse=None,
        lse_head=40, ws=FAKE, wsb=1 << 30, info=None, dtype=torch.bfloat16, lens=([4, 30], [3000, 30])):
    if info is None:
        info = L.losa_packed_plan(*lens, 4, 2, dtype, device="cpu").info
    q, k, v, o = (view(L) if isinstance(x, int) and x == 1 else x for x in (q, k, v, o))
    at = lambda x: None if isinstance(x, int) else ctypes.addressof(x)  # noqa: E731
    return L.lib.losa_packed_attn_fwd(at(q), at(k), at(v), q_rows, k_rows, at(info), plan, d, scale,
                                      at(o), lse, lse_head, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=0), 1), (dict(k=0), 1), (dict(v=0), 1), (dict(o=0), 1), (dict(info=0), 1),
    (dict(plan=None), 1), (dict(plan=FAKE + 4), 4), (dict(q_rows=33), 2), (dict(k_rows=3029), 2),
    (dict(d=0), 2), (dict(d=96), 5), (dict(scale=0.0), 2), (dict(scale=float("nan")), 2),
    (dict(scale=float("inf")), 2), (dict(lse=FAKE + 2), 4), (dict(lse=FAKE, lse_head=33), 2),
    (dict(ws=None), 1), (dict(ws=FAKE + 8), 4), (dict(wsb=100), 6)])
def test_forward_refusals(L, kw, code):
    assert fwd(L, **kw) == code
    assert L.lib.losa_last_error().decode() != ""


@pytest.mark.parametrize("which", ["q", "k", "v", "o"])
@pytest.mark.parametrize("kw,code", [(dict(data=0), 1), (dict(data=FAKE + 8), 4), (dict(token=516), 4),
                                     (dict(head=-128), 2)])
def test_forward_view_refusals(L, which, kw, code):
    assert fwd(L, **{which: view(L, **kw)}) == code


def test_forward_stride_refusals(L):
    assert fwd(L, o=view(L, token=64)) == 2 and fwd(L, o=view(L, head=0)) == 2
    for which in "qo":  # row offsets are products of 32-bit numbers
        assert fwd(L, **{which: view(L, head=1 << 31)}) == 2
        assert fwd(L, **{which: view(L, token=1 << 31)}) == 2
    for which in "kv":
        assert fwd(L, **{which: view(L, token=64)}) == 2
        assert fwd(L, **{which: view(L, token=(1 << 25) + 8)}) == 2


def test_an_output_over_other_tensors_is_refused(L):
    at = [view(L, data=FAKE + (i << 24)) for i in range(4)]
    args = dict(zip("qkvo", at))
    for kw in (dict(o=view(L, data=at[0].data, token=128, head=5120)), dict(o=at[1]), dict(o=at[2])):
        assert fwd(L, **{**args, **kw}) == 2 and "may lie over" in L.lib.losa_last_error().decode()


def test_forward_refuses_what_is_no_info(L):
    info = L.losa_packed_plan([4], [300], 4, 2, torch.bfloat16, device="cpu").info
    for name, value in (("H", 5), ("H_kv", 0), ("n_tiles", 3), ("bytes", 8), ("dtype", 4), ("n_few", -1), ("tile_rows", 64)):
        bad = L._PackedInfo.from_buffer_copy(info)
        setattr(bad, name, value)
        assert fwd(L, info=bad) == 2, name


def test_forward_of_nothing_launches_nothing(L):
    assert fwd(L, lens=([0, 0], [5, 0]), plan=None, q_rows=0, k_rows=0, ws=None, wsb=0) == 0


def test_binding_refuses_host_tensors(L):
    p = L.losa_packed_plan([4], [4], 2, 1, torch.float32, device="cpu")
    q = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError, match="must live on"):
        L.losa_packed_attn_fwd(q, q[:, :1], q[:, :1], p)
    with pytest.raises(TypeError, match="PackedPlan"):
        L.losa_packed_attn_fwd(q, q, q, None)


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda p: pickle.loads(pickle.dumps(p))],
                         ids=["copy", "deepcopy", "pickle"])
def test_a_copied_plan_holds_its_own_sizes(L, monkeypatch, again):
    """What a call passes as the plan's sizes is the copy's own, also once the original
    and its memory have gone to other plans."""
    plan = L.losa_packed_plan([4, 30], [3000, 30], 4, 2, torch.bfloat16, device="cpu")
    want, units_of = bytes(plan.info), plan.data.clone()
    twin = again(plan)
    del plan
    others = [L.losa_packed_plan([n], [n], 8, 8, torch.bfloat16, device="cpu") for n in range(1, 200)]
    passed = []

    def seen(q, k, v, q_rows, k_rows, info, *rest):  # what the library would read
        passed.append(ctypes.string_at(info, ctypes.sizeof(L._PackedInfo)))
        return 0

    monkeypatch.setattr(L, "_call", lambda dev, fn, *args: seen(*args))
    monkeypatch.setattr(L, "_packed_view", lambda *a: b"")
    monkeypatch.setattr(L, "_arg", lambda t, *a, **k: t)
    on_gpu = type("OnGpu", (torch.Tensor,), {"is_cuda": property(lambda t: True)})
    q, k = torch.zeros(34, 4, 128).as_subclass(on_gpu), torch.zeros(3030, 2, 128)
    L.losa_packed_attn_fwd(q, k, k, twin, out=torch.zeros(34, 4, 128))
    assert passed == [want] and bytes(twin.info) == want and len(others) == 199
    assert torch.equal(twin.data, units_of) and twin.workspace_bytes(128) > 0
    assert (twin.q_rows, twin.k_rows, twin.heads, twin.kv_heads) == (34, 3030, 4, 2)


def test_a_plan_is_what_was_planned(L):
    """A plan's sizes and units are not replaced, and fit each other."""
    plan = L.losa_packed_plan([4, 30], [3000, 30], 4, 2, torch.bfloat16, device="cpu")
    for name in ("info", "data", "dtype", "q_rows", "k_rows", "heads", "kv_heads"):
        with pytest.raises(AttributeError):
            setattr(plan, name, getattr(plan, name))
    plan.info.n_tiles = 1 << 20  # a copy's
    assert plan.info.n_tiles < 100
    for data in (plan.data[:-1], plan.data.int(), plan.data.repeat(2)[::2]):
        with pytest.raises(ValueError, match="int64"):
            L.PackedPlan(plan.info, data, plan.dtype)
    with pytest.raises(ValueError, match="dtype"):
        L.PackedPlan(plan.info, plan.data, torch.float32)
    assert L.PackedPlan(plan.info, plan.data, plan.dtype).workspace_bytes(64) == plan.workspace_bytes(64)


@pytest.mark.parametrize("dtype,heads,kv_heads,q_lens,k_len", [
    (torch.bfloat16, 2, 2, [(1 << 30) - 128], 1),           # tiles, 256 threads a workgroup
    (torch.float32, 2, 2, [(1 << 30) - 256], 1),            # 512
    (torch.bfloat16, 16, 16, [1] * ((1 << 20) - 1), 1),     # few-row parts
    (torch.float32, 8, 8, [1] * ((1 << 20) - 1), 1),
    (torch.bfloat16, 2048, 64, [1] * ((1 << 15) - 1), 512),  # joins, eight rows a workgroup
], ids=["tiles", "tiles-f32", "few", "few-f32", "joins"])
def test_a_plan_beyond_one_launch_is_refused(L, dtype, heads, kv_heads, q_lens, k_len):
    """A launch counts its threads in 32 bits: one unit more than fits is refused by the
    plan, not by the launch, which may be the call's second."""
    def status(q_lens):
        n = len(q_lens)
        q, k = np.array(q_lens, np.int32), np.full(n, k_len, np.int32)
        info = L._PackedInfo()
        st = L.lib.losa_packed_plan(None, q.ctypes.data, None, k.ctypes.data, n, L._DTYPES[dtype], heads,
                                    kv_heads, 0, None, 0, ctypes.addressof(info))
        if st == 0:
            threads = 256 if dtype == torch.bfloat16 else 512
            units = (info.n_tiles + info.n_few) * kv_heads
            joins = info.n_wide * kv_heads + -(-(info.n_joins - info.n_wide) * kv_heads // 8)
            assert units * threads < 1 << 32 and joins * 512 < 1 << 32
            # the next unit is the first too many
            assert (units + kv_heads) * threads >= 1 << 32 or joins * 512 + kv_heads * 32 * 64 >= 1 << 32
        return st

    assert status(q_lens) == 0
    assert status([q_lens[0] + 128 * (2 if dtype == torch.float32 else 1)] if len(q_lens) == 1
                  else q_lens + [1]) == 2
    assert "launch" in L.lib.losa_last_error().decode()


@pytest.mark.parametrize("q_lens,q_starts,run", [
    ([4, 30], None, 34), ([4, 30], [0, 100], 30), ([4, 0, 30], [30, 7, 0], 34), ([1, 1, 1], [0, 2, 4], 1),
    ([3, 0], None, 3), ([0], [9], 0), ([2, 5, 1, 6], [20, 40, 22, 23], 9)])
def test_longest_run_of_neighbouring_rows(L, q_lens, q_starts, run):
    p = L.losa_packed_plan(q_lens, [3000] * len(q_lens), 4, 2, torch.bfloat16, q_starts=q_starts, device="cpu")
    assert p.info.q_run == run


@pytest.mark.parametrize("token,head,starts,code", [
    # (with no workspace: 1 is the next check)
    (128, 128, None, 2), (128, 128, [0, 5], 2), (256, 384, None, 2), (384, 512, None, 2), (136, 40 * 136, None, 1),
    (136, 2 * 136, None, 2), (136, 33 * 136 + 128, None, 1), (136, 29 * 136, [0, 40], 2), (136, 30 * 136, [0, 40], 1),
    (512, 128, None, 1), (128 * 7, 256, None, 1), (128 * 6, 256, None, 2), (128, 40 * 128, None, 1), (128, 34 * 128, None, 1),
    (128, 33 * 128, None, 2)])
def test_output_rows_that_share_memory_are_refused(L, token, head, starts, code):
    """Rows of one run of neighbours, 34 or the longer of two, 4 heads: each pair compared."""
    run = 34 if starts is None else 30
    at = sorted(r * token + h * head for r in range(run) for h in range(4))
    assert (min(b - a for a, b in zip(at, at[1:])) < 128) == (code == 2)
    info = L.losa_packed_plan([4, 30], [3000, 30], 4, 2, torch.bfloat16, q_starts=starts, device="cpu").info
    assert fwd(L, info=info, q_rows=80, o=view(L, token=token, head=head, data=FAKE + (1 << 30)), ws=None,
               lse_head=80) == code
    assert code == 1 or "overlap" in L.lib.losa_last_error().decode()
