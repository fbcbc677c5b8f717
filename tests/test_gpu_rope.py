"""Rotary positions and query/key norms on the GPU against plain arithmetic in
64 bits, element by element.

Tolerances.  The output is rounded once: half a step, finfo.eps / 2 relative to
the value.  Before that everything is fp32, u = 2^-24 per operation: a sum of
squares takes 8 fma, up to 4 exchanges and (over all heads) one addition per
head and wave, so its relative error is under (16 + H) u, half of that after
the root; root, division, weight and bias add one each, the rotation two
products, a sum and two roundings of the table.  That is under (16 + H) / 2 + 12
< 24 + H steps of the terms' size (the sum of the absolute values that a result
is made of).  A layer norm subtracts the mean: its error, under 16 u of the row's
largest value, scales with weight / std.
"""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2608_12032_amd import losa
    return losa


def turn(y, size, dims, lens, pos, halves, base):
    """Rotation of y [B, N, H, d] (fp64, CPU) and of the size of its terms."""
    B, N = y.shape[:2]
    rot = sum(dims)
    angle = []
    for a, dim in enumerate(dims):
        p = pos[:, a] if pos.dim() == 3 else pos[a][None].expand(B, N)
        f = base ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
        ang = p.double()[:, :, None] * f
        ang = torch.where((p < 0)[:, :, None], 0.0, ang)
        angle.append(torch.where((p >= lens[a])[:, :, None], torch.nan, ang))
    angle = torch.cat(angle, 2)[:, :, None, :]
    if halves:
        i, j = torch.arange(rot // 2), torch.arange(rot // 2) + rot // 2
    else:
        i, j = torch.arange(0, rot, 2), torch.arange(1, rot, 2)
    c, s = angle.cos(), angle.sin()
    out, big = y.clone(), size.clone()
    out[..., i], out[..., j] = y[..., i] * c - y[..., j] * s, y[..., i] * s + y[..., j] * c
    big[..., i] = big[..., j] = size[..., i] + size[..., j]
    return out, big


def normed(x, kind, over, w, b, eps):
    """Norm of x [B, N, H, d] in fp64 and the size of its terms."""
    dims = (3,) if over == "head" else (2, 3)
    span = lambda t, fill: (torch.full(x.shape[3:], fill).double() if t is None else  # noqa: E731
                            t.double().cpu() if over == "head" else t.double().cpu().view(x.shape[2:]))
    mean = x.mean(dims, keepdim=True) if kind == "layer" else torch.zeros(1).double()
    z = x - mean
    inv = 1.0 / torch.sqrt((z * z).mean(dims, keepdim=True) + eps)
    y = z * inv * span(w, 1.0) + span(b, 0.0)
    size = (x.abs() + mean.abs()) * inv * span(w, 1.0).abs() + span(b, 0.0).abs()
    if kind == "layer":
        size = size + x.abs().amax(dims, keepdim=True) * inv * span(w, 1.0).abs()
    return y, size


def check(got, ref, size, N, H):
    """got [B, H, n_pad, d] against ref [B, N, H, d]."""
    g = got.cpu().double().transpose(1, 2)
    assert not g[:, N:].any(), "padding rows"
    g = g[:, :N]
    assert torch.equal(torch.isnan(g), torch.isnan(ref))
    bound = torch.finfo(got.dtype).eps / 2 * ref.abs() + (24 + H) * U * size
    err = (g - ref).abs()
    ok = (err <= bound) | torch.isnan(ref)
    assert ok.all(), ((err - bound).nan_to_num().max(), err.nan_to_num().max())


def randn(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def grid(T, Hg, Wg, text=0):
    g = torch.stack([x.flatten() for x in torch.meshgrid(
        torch.arange(T), torch.arange(Hg), torch.arange(Wg), indexing="ij")])
    return torch.cat([torch.full((3, text), -1), g], 1).to(torch.int32)


ROPE_CASES = [  # dtype, d, halves, dims, grid, text, B, H, pad
    ("bf16", 128, False, (44, 42, 42), (3, 5, 7), 0, 1, 12, 128),
    ("bf16", 128, True, (32, 48, 48), (2, 3, 5), 9, 2, 3, 64),
    ("bf16", 64, False, (16, 24, 24), (3, 4, 11), 5, 2, 5, 1),
    ("bf16", 64, True, (48,), (1, 1, 67), 0, 1, 1, 1),          # 16 dims unturned
    ("bf16", 128, False, (24, 32), (1, 6, 9), 0, 3, 2, 128),    # 72 dims unturned
    ("f32", 128, False, (44, 42, 42), (2, 5, 7), 3, 2, 7, 1),
    ("f32", 128, True, (128,), (1, 1, 130), 0, 1, 4, 64),
    ("f32", 64, False, (8, 8, 8, 8), (2, 3, 5), 0, 1, 3, 1),    # four axes
    ("f32", 64, True, (16, 24, 24), (3, 3, 3), 1, 2, 40, 128),
    ("bf16", 64, True, (6, 10), (1, 5, 9), 2, 1, 3, 1),         # pairs of a lane on two axes
    ("bf16", 128, False, (2, 2, 4), (2, 3, 4), 1, 1, 2, 1),
    ("f32", 128, True, (10, 2, 44), (3, 2, 7), 0, 2, 6, 128),
    ("bf16", 128, False, (128,), (1, 1, 1), 0, 1, 1, 1),        # one token, one head
    ("f32", 64, False, (64,), (1, 1, 1), 0, 5, 2, 1),
]


@pytest.mark.parametrize("case", ROPE_CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_rope(L, case):
    dtype, d, halves, dims, (T, Hg, Wg), text, B, H, pad = case
    print(f"[gpu-rope] {case}", flush=True)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pos = grid(T, Hg, Wg, text)
    pos = {1: pos[2:], 2: pos[1:], 3: pos, 4: torch.cat([pos[:1], pos])}[len(dims)].contiguous()
    lens = [int(p.max()) + 1 for p in pos]
    N = pos.shape[1]
    n_pad = -(-N // pad) * pad
    x = randn(B, N, H, d, seed=1).to(tt)
    y = L.losa_rope(x.cuda(), L.losa_rope_table(dims, lens), pos.cuda(), n_pad=n_pad,
                    pairing="halves" if halves else "interleaved")
    assert y.shape == (B, H, n_pad, d)
    ref, size = turn(x.double(), x.double().abs(), dims, lens, pos, halves, 10000.0)
    check(y, ref, size, N, H)
    # unturned dims come through as they are
    assert torch.equal(y[:, :, :N, sum(dims):].cpu(), x[..., sum(dims):].transpose(1, 2))


NORM_CASES = list(itertools.product(["bf16", "f32"], [64, 128], ["rms", "layer"], ["head", "all"],
                                    [(1, 1, 3, 3), (37, 2, 4, 2), (130, 1, 17, 1), (9, 1, 40, 40)]))


@pytest.mark.parametrize("case", NORM_CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_qk_norm_rope(L, case):
    dtype, d, kind, over, (N, B, H, Hkv) = case
    print(f"[gpu-qknorm] {case}", flush=True)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n_pad = -(-N // 64) * 64
    # one fused projection; channels of uneven size and mean
    x = (randn(B, N, H + 2 * Hkv, d, seed=2) * (1 + randn(d, seed=3).abs()) + 0.5 * randn(d, seed=4)).to(tt)
    xg = x.cuda()
    span = [h * d if over == "all" else d for h in (H, Hkv)]
    qw, kw = 1 + 0.3 * randn(span[0], seed=5), 1 + 0.3 * randn(span[1], seed=6)
    qb = 0.2 * randn(span[0], seed=7) if kind == "layer" else None
    pos = torch.stack([torch.arange(N) % 7, torch.arange(N) // 7]).to(torch.int32)
    pos[:, N // 2:N // 2 + 3] = -1
    dims, lens = (d // 2, d // 2), (7, N // 7 + 1)
    halves = H % 2 == 0
    q, k, v = L.losa_qk_norm_rope(
        xg[:, :, :H], xg[:, :, H:H + Hkv], xg[:, :, H + Hkv:], norm=kind, over=over,
        q_weight=qw.cuda(), q_bias=None if qb is None else qb.cuda(), k_weight=kw.cuda(),
        eps=1e-5, table=L.losa_rope_table(dims, lens, 1000.0), pos=pos.cuda(), n_pad=n_pad,
        pairing="halves" if halves else "interleaved")
    for got, part, w, b in ((q, x[:, :, :H], qw, qb), (k, x[:, :, H:H + Hkv], kw, None)):
        y, size = normed(part.double(), kind, over, w, b, 1e-5)
        ref, size = turn(y, size, dims, lens, pos, halves, 1000.0)
        check(got, ref, size, N, H)
    assert torch.equal(v[:, :, :N].cpu(), x[:, :, H + Hkv:].transpose(1, 2))
    assert not v[:, :, N:].any()


def test_norm_alone_and_layout_alone(L):
    """norm without a rotation, without weights; neither (a change of layout); no values."""
    x = randn(2, 50, 6, 128, seed=8).to(torch.bfloat16)
    xg = x.cuda()
    q, k = L.losa_qk_norm_rope(xg[:, :, :4], xg[:, :, 4:], norm="rms")
    for got, part in ((q, x[:, :, :4]), (k, x[:, :, 4:])):
        y, size = normed(part.double(), "rms", "head", None, None, 1e-6)
        check(got, y, size, 50, 4)
    q, k = L.losa_qk_norm_rope(xg[:, :, :4], xg[:, :, 4:], norm=None, n_pad=64)
    assert torch.equal(q[:, :, :50].cpu(), x[:, :, :4].transpose(1, 2))
    assert torch.equal(k[:, :, :50].cpu(), x[:, :, 4:].transpose(1, 2)) and not k[:, :, 50:].any()


def test_positions_by_batch_and_out_of_the_table(L):
    """Each batch has its own positions; one outside the table gives NaN in its axis'
    dims and nowhere else, one below 0 leaves them as they are."""
    x = randn(3, 6, 2, 64, seed=9)
    pos = torch.tensor([[[0, 1, 2, 3, 4, 99], [5, 4, 3, 2, 1, 0]],
                        [[4, -1, 4, 4, 4, 4], [-7, 1, 2, 8, 2, 1]],
                        [[2 ** 31 - 1, 1, 1, 1, 1, 1], [-2 ** 31, 1, 2, 3, 4, 5]]],
                       dtype=torch.int32)
    dims, lens = (24, 32), (5, 6)
    y = L.losa_rope(x.cuda(), L.losa_rope_table(dims, lens), pos.cuda())
    ref, size = turn(x.double(), x.double().abs(), dims, lens, pos, False, 10000.0)
    check(y, ref, size, 6, 2)
    assert torch.isnan(y).any() and torch.equal(y[..., 56:].cpu(), x[..., 56:].transpose(1, 2))


@pytest.mark.parametrize("tt", [torch.bfloat16, torch.float32])
def test_strides(L, tt):
    """Head-major and token-major views on both sides, a broadcast input, in place."""
    x = randn(2, 40, 4, 128, seed=10).to(tt).cuda()
    pos = (torch.arange(40, dtype=torch.int32) * 3)[None].cuda()
    t = L.losa_rope_table((128,), (118,))
    want = L.losa_rope(x, t, pos)
    head_major = x.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(L.losa_rope(head_major, t, pos), want)
    room = torch.full((2, 40, 9, 128), 5.0, dtype=tt, device="cuda")
    L.losa_rope(x, t, pos, out=room[:, :, 3:7].transpose(1, 2))
    assert torch.equal(room[:, :, 3:7].transpose(1, 2), want)
    assert (room[:, :, :3] == 5).all() and (room[:, :, 7:] == 5).all()
    wide = x[:1, :, :1].expand(2, 40, 4, 128)
    assert torch.equal(L.losa_rope(wide, t, pos), L.losa_rope(wide.contiguous(), t, pos))
    y = x.clone()
    L.losa_rope(y, t, pos, out=y.transpose(1, 2))
    assert torch.equal(y.transpose(1, 2), want)
    y = x.clone()
    a, b = L.losa_qk_norm_rope(x[:, :, :3], x[:, :, 3:], over="all", table=t, pos=pos)
    L.losa_qk_norm_rope(y[:, :, :3], y[:, :, 3:], over="all", table=t, pos=pos,
                        q_out=y[:, :, :3].transpose(1, 2), k_out=y[:, :, 3:].transpose(1, 2))
    assert torch.equal(y[:, :, :3].transpose(1, 2), a) and torch.equal(y[:, :, 3:].transpose(1, 2), b)


def test_a_head_gives_the_same_bits_alone(L):
    x = randn(1, 700, 20, 128, seed=11).to(torch.bfloat16).cuda()
    pos = torch.arange(700, dtype=torch.int32)[None].cuda()
    t = L.losa_rope_table((96,), (700,))
    q, k = L.losa_qk_norm_rope(x, x[:, :, :1], norm="layer", table=t, pos=pos)
    for h in (0, 7, 19):
        a, _ = L.losa_qk_norm_rope(x[:, :, h:h + 1], x[:, :, :1], norm="layer", table=t, pos=pos)
        assert torch.equal(a[:, 0], q[:, h])
    a, _ = L.losa_qk_norm_rope(x[:, 100:107], x[:, 100:107, :1], norm="layer", table=t,
                               pos=pos[:, 100:107].contiguous())
    assert torch.equal(a, q[:, :, 100:107])


def test_non_finite_values_stay_in_their_rows(L):
    x = randn(1, 33, 3, 64, seed=12)
    x[0, 4, 1, 10], x[0, 20, 2, 3], x[0, 7, 0, 60] = float("inf"), float("nan"), -float("inf")
    pos = torch.arange(33, dtype=torch.int32)[None]
    pos[0, 7] = -1
    clean = x.nan_to_num(0.0, 0.0, 0.0)
    t = L.losa_rope_table((48,), (33,))
    y = L.losa_rope(x.cuda(), t, pos.cuda()).cpu()
    z = L.losa_rope(clean.cuda(), t, pos.cuda()).cpu()
    bad = ~torch.isfinite(y)
    assert bad.sum() == 5  # two pairs, and one value of an unturned dim
    assert bad[0, 1, 4, 10:12].all() and bad[0, 2, 20, 2:4].all() and y[0, 0, 7, 60] == -float("inf")
    assert torch.equal(torch.where(bad, 0.0, y), torch.where(bad, 0.0, z))
    q, _ = L.losa_qk_norm_rope(x.cuda(), x.cuda(), table=t, pos=pos.cuda())
    bad = ~torch.isfinite(q.cpu()).all(3)
    want = torch.zeros(1, 3, 33, dtype=torch.bool)
    want[0, 1, 4] = want[0, 2, 20] = want[0, 0, 7] = True
    assert torch.equal(bad, want)


def test_streams_and_graph(L):
    x = randn(1, 257, 6, 128, seed=13).to(torch.bfloat16).cuda()
    w = (1 + 0.1 * randn(4 * 128, seed=14)).cuda()
    pos = torch.arange(257, dtype=torch.int32)[None].cuda()
    t = L.losa_rope_table((128,), (257,))
    out = [torch.empty(1, h, 320, 128, dtype=x.dtype, device="cuda") for h in (4, 1, 1)]

    def call():
        L.losa_qk_norm_rope(x[:, :, :4], x[:, :, 4:5], x[:, :, 5:], over="all", q_weight=w,
                            table=t, pos=pos, n_pad=320, q_out=out[0], k_out=out[1], v_out=out[2])
        L.losa_rope(x[:, :, :4], t, pos, n_pad=320, out=room)

    room = torch.empty_like(out[0])
    call()
    torch.cuda.synchronize()
    ref = [o.clone() for o in out] + [room.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(3):
        for o in out + [room]:
            o.fill_(rep)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out + [room], ref)), rep


def test_prepared_tensors_feed_the_sparse_path(L):
    """Projections -> norm and rotation -> construction step, selection, sparse forward:
    the padded layout is what the path reads, and its padding rows are 0."""
    T, Hg, Wg, H, d, C = 2, 9, 15, 3, 64, 64
    N = T * Hg * Wg
    n_pad = L.padded_len(N, C, C)
    x = randn(1, N, 3 * H, d, seed=15).to(torch.bfloat16).cuda()
    pos = grid(T, Hg, Wg).cuda()
    t = L.losa_rope_table((16, 24, 24), (T, Hg, Wg))
    q, k, v = L.losa_qk_norm_rope(x[:, :, :H], x[:, :, H:2 * H], x[:, :, 2 * H:], table=t, pos=pos,
                                  n_pad=n_pad)
    o, mass = L.losa_construct(q, k, v, N, C, C)
    rp, ci = L.losa_select_blocks(mass, N, C, C, 1.0)
    o2 = L.losa_sparse_attn_fwd(q, k, v, N, C, C, rp, ci)
    assert torch.equal(o, o2)
    qf, kf, vf = (a[0, :, :N].double().cpu() for a in (q, k, v))
    ref = torch.softmax(qf @ kf.transpose(1, 2) / d ** 0.5, 2) @ vf
    assert (o[0, :, :N].double().cpu() - ref).abs().max() <= 2e-2


def test_device_argument_checks(L):
    x = torch.zeros(1, 5, 2, 64, device="cuda")
    t = L.losa_rope_table((64,), (5,))
    pos = torch.zeros(1, 5, dtype=torch.int32, device="cuda")
    w = torch.ones(64, device="cuda")
    cases = [
        (lambda: L.losa_rope(x[0], t, pos), ValueError, "B, N, H, d"),
        (lambda: L.losa_rope(x.half(), t, pos), TypeError, "dtype"),
        (lambda: L.losa_rope(x.transpose(2, 3), t, pos), ValueError, "contiguous rows"),
        (lambda: L.losa_rope(x, t.data, pos), TypeError, "RopeTable"),
        (lambda: L.losa_rope(x, t, pos.long()), TypeError, "pos must be"),
        (lambda: L.losa_rope(x, t, pos[:, :4]), ValueError, "contiguous|pos must have shape"),
        (lambda: L.losa_rope(x, t, pos.cpu()), ValueError, "must live on"),
        (lambda: L.losa_rope(x, t, pos, pairing="thirds"), ValueError, "pairing"),
        (lambda: L.losa_rope(x, t, pos, n_pad=4), L.LosaError, "N_pad"),
        (lambda: L.losa_rope(x, t, pos, out=torch.empty(1, 2, 6, 64, device="cuda")), ValueError,
         "out must have shape"),
        (lambda: L.losa_qk_norm_rope(x, x[:, :4]), ValueError, "k must have shape"),
        (lambda: L.losa_qk_norm_rope(x, x.bfloat16()), TypeError, "k must be"),
        (lambda: L.losa_qk_norm_rope(x, x, norm="batch"), ValueError, "norm must be"),
        (lambda: L.losa_qk_norm_rope(x, x, over="rows"), ValueError, "over must be"),
        (lambda: L.losa_qk_norm_rope(x, x, q_weight=w, over="all"), ValueError, "q_weight"),
        (lambda: L.losa_qk_norm_rope(x, x, q_weight=w.bfloat16()), TypeError, "q_weight"),
        (lambda: L.losa_qk_norm_rope(x, x, norm=None, q_weight=w), ValueError, "need a norm"),
        (lambda: L.losa_qk_norm_rope(x, x, table=t), ValueError, "table and pos"),
        (lambda: L.losa_qk_norm_rope(x, x, v_out=x.transpose(1, 2)), ValueError, "v_out needs v"),
        (lambda: L.losa_rope(x.flatten()[4:4 + 256].view(1, 2, 2, 64)[..., :64], t, pos[:, :2].contiguous()), None, ""),
        (lambda: L.losa_rope(x.flatten()[1:257].view(1, 2, 2, 64), t, pos[:, :2].contiguous()),
         L.LosaError, "ALIGNMENT"),
    ]
    for fn, exc, msg in cases:
        if exc is None:
            fn()
            continue
        with pytest.raises(exc, match=msg):
            fn()


# Calls of a layer's size: outputs of 32 MiB and more go past the caches, and a wave takes
# several groups of four heads one after another.  Sampled tokens against 64 bits; every
# token bitwise against calls on a few hundred tokens, which do neither.
SLICE = 250


def large_positions(N, T):
    return torch.stack([torch.arange(N) % T, torch.arange(N) // T]).to(torch.int32)


def sampled(N):
    return torch.cat([torch.tensor([0, 1, N - 2, N - 1]),
                      torch.randint(0, N, (40,), generator=torch.Generator().manual_seed(16))])


LARGE_ROPE = [  # dtype, d, halves, rot, B, N, H, pad
    ("bf16", 128, False, 128, 1, 11_003, 12, 128), ("bf16", 128, True, 96, 1, 11_003, 13, 1),
    ("bf16", 64, True, 64, 2, 5_501, 26, 64), ("bf16", 64, False, 48, 1, 22_001, 12, 1),
    ("f32", 128, True, 128, 1, 11_003, 13, 64), ("f32", 128, False, 64, 3, 1_801, 14, 1),
    ("f32", 64, False, 64, 1, 11_003, 13, 128), ("f32", 64, True, 32, 1, 16_381, 9, 1)]


@pytest.mark.parametrize("case", LARGE_ROPE, ids=lambda c: "-".join(map(str, c)))
def test_rope_of_a_layer(L, case):
    dtype, d, halves, rot, B, N, H, pad = case
    print(f"[gpu-rope] {case}", flush=True)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n_pad = -(-N // pad) * pad
    assert B * H * n_pad * d * tt.itemsize >= 32 << 20
    gen = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn(B, N, 2 * H, d, generator=gen, device="cuda").to(tt)[:, :, H:]
    dims, lens = (rot // 2, rot // 2), (101, N // 101 + 1)
    pos, t = large_positions(N, 101), L.losa_rope_table(dims, lens)
    pos[:, N // 3:N // 3 + 77] = -1
    pg, pairing = pos.cuda(), "halves" if halves else "interleaved"
    y = L.losa_rope(x, t, pg, n_pad=n_pad, pairing=pairing)
    at = sampled(N)
    xs = x[:, at.cuda()].double().cpu()
    ref, size = turn(xs, xs.abs(), dims, lens, pos[:, at], halves, 10000.0)
    check(y[:, :, at.cuda()], ref, size, len(at), H)
    assert not y[:, :, N:].any()
    for a in range(0, N, SLICE):
        s = slice(a, min(N, a + SLICE))
        small = L.losa_rope(x[:, s], t, pg[:, s].contiguous(), pairing=pairing)
        assert torch.equal(y[:, :, s], small), a
    z = x.contiguous()  # in place
    L.losa_rope(z, t, pg, pairing=pairing, out=z.transpose(1, 2))
    assert torch.equal(z.transpose(1, 2), y[:, :, :N])


LARGE_NORM = [  # dtype, d, kind, over, halves, B, N, H, Hkv, pad
    ("bf16", 128, "rms", "head", False, 1, 9_001, 12, 12, 128), ("bf16", 64, "layer", "head", True, 2, 4_603, 24, 8, 1),
    ("bf16", 128, "layer", "all", False, 1, 9_001, 12, 6, 64), ("bf16", 64, "rms", "all", True, 1, 22_001, 16, 4, 1),
    ("bf16", 128, "layer", "all", True, 1, 4_603, 40, 40, 64), ("bf16", 128, "rms", "all", False, 2, 11_003, 4, 1, 1),
    ("f32", 128, "layer", "head", True, 1, 4_603, 12, 6, 64), ("f32", 64, "rms", "head", False, 1, 9_001, 13, 13, 1),
    ("f32", 128, "rms", "all", True, 1, 4_603, 12, 3, 128), ("f32", 64, "layer", "all", False, 1, 4_603, 17, 17, 1),
    ("f32", 128, "layer", "all", False, 1, 9_001, 4, 2, 1)]


@pytest.mark.parametrize("case", LARGE_NORM, ids=lambda c: "-".join(map(str, c)))
def test_qk_norm_rope_of_a_layer(L, case):
    dtype, d, kind, over, halves, B, N, H, Hkv, pad = case
    print(f"[gpu-qknorm] {case}", flush=True)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n_pad = -(-N // pad) * pad
    assert B * (H + 2 * Hkv) * n_pad * d * tt.itemsize >= 32 << 20
    gen = torch.Generator(device="cuda").manual_seed(18)
    x = torch.randn(B, N, H + 2 * Hkv, d, generator=gen, device="cuda")
    x = (x * (1 + randn(d, seed=19).abs()).cuda() + 0.5 * randn(d, seed=20).cuda()).to(tt)
    cut = lambda t: (t[:, :, :H], t[:, :, H:H + Hkv], t[:, :, H + Hkv:])  # noqa: E731
    span = [h * d if over == "all" else d for h in (H, Hkv)]
    qw, kw = 1 + 0.3 * randn(span[0], seed=21), 1 + 0.3 * randn(span[1], seed=22)
    qb = 0.2 * randn(span[0], seed=23) if kind == "layer" else None
    dims, lens = (d // 2, d // 4), (101, N // 101 + 1)
    pos, t = large_positions(N, 101), L.losa_rope_table(dims, lens)
    pg = pos.cuda()
    args = dict(norm=kind, over=over, q_weight=qw.cuda(), k_weight=kw.cuda(),
                q_bias=None if qb is None else qb.cuda(), eps=1e-5, table=t,
                pairing="halves" if halves else "interleaved")
    got = L.losa_qk_norm_rope(*cut(x), pos=pg, n_pad=n_pad, **args)
    at = sampled(N)
    q, k, v = (p[:, at.cuda()].double().cpu() for p in cut(x))
    for g, part, w, b, h in ((got[0], q, qw, qb, H), (got[1], k, kw, None, Hkv)):
        y, size = normed(part, kind, over, w, b, 1e-5)
        ref, size = turn(y, size, dims, lens, pos[:, at], halves, 10000.0)
        check(g[:, :, at.cuda()], ref, size, len(at), h)
    assert torch.equal(got[2][:, :, :N], cut(x)[2].transpose(1, 2))
    assert not any(g[:, :, N:].any() for g in got)
    for a in range(0, N, SLICE):
        s = slice(a, min(N, a + SLICE))
        small = L.losa_qk_norm_rope(*cut(x[:, s]), pos=pg[:, s].contiguous(), **args)
        assert all(torch.equal(g[:, :, s], z) for g, z in zip(got, small)), a
    parts = cut(x.clone())  # in place
    L.losa_qk_norm_rope(*parts, pos=pg, q_out=parts[0].transpose(1, 2), k_out=parts[1].transpose(1, 2),
                        v_out=parts[2].transpose(1, 2), **args)
    assert all(torch.equal(p.transpose(1, 2), g[:, :, :N]) for p, g in zip(parts, got))
