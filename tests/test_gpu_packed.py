"""Packed attention on the GPU against plain attention in 64 bits, element by element.

Tolerances, from the arithmetic.  With w the softmax weights of a row, A = sum_j w_j |v_j|
and Z = scale * sum |q_i k_ji| at its largest, an output is off by at most
  half a step of the output, finfo.eps / 2 * |o|;
  bf16: half a step of every probability in P V, 2^-8 A;
  scores summed over d in fp32 (u = 2^-24 a term, both in p and in the sum): 4 (d + 8) u Z A;
  fp32 sums over the keys, taken 4 or more at a time, and their joins: (k / 4 + 128) u A.
lse: 2 (d + 8) u Z + (k / 4 + 128) u + 8 u |lse|.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2608_12032_amd import losa
    return losa


def randn(*shape, seed, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def reference(q, k, v, causal, scale):
    """One sequence: o and its bound [lq, H, d], lse and its bound [H, lq], in fp64."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    lq, H, d = q.shape
    lk, G = k.shape[0], H // k.shape[1]
    o, size = torch.zeros(lq, H, d).double(), torch.zeros(lq, H, d).double()
    lse, z = torch.full((H, lq), -math.inf).double(), torch.zeros(H, lq).double()
    seen = torch.ones(lq, lk, dtype=torch.bool)
    if causal:
        seen = torch.arange(lk)[None] <= torch.arange(lq)[:, None] + lk - lq
    some = seen.any(1)
    for h in range(H if lk else 0):
        s = (q[:, h] @ k[:, h // G].t() * scale).masked_fill(~seen, -math.inf)
        z[h] = (q[:, h].abs() @ k[:, h // G].abs().t() * scale).masked_fill(~seen, 0.0).amax(1)
        lse[h] = torch.logsumexp(s, 1)
        w = torch.where(seen, torch.exp(s - torch.where(some, lse[h], 0.0)[:, None]), 0.0)
        o[:, h], size[:, h] = w @ v[:, h // G], w @ v[:, h // G].abs()
    return o, size, lse, z


def check(got, got_lse, ref, lk, d):
    o, size, lse, z = ref
    u_keys = (lk / 4 + 128) * U
    zt = z.t()[:, :, None]
    p_step = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    bound = torch.finfo(got.dtype).eps / 2 * o.abs() + size * (p_step + 4 * (d + 8) * U * zt + u_keys)
    err = (got.double().cpu() - o).abs()
    assert (err <= bound).all(), ((err - bound).max(), err.max())
    if got_lse is not None:
        g = got_lse.double().cpu()
        empty = torch.isinf(lse)
        assert torch.equal(torch.isinf(g), empty) and (g[empty] < 0).all()
        lb = 2 * (d + 8) * U * z + u_keys + 8 * U * lse.abs()
        assert ((g - lse).abs() <= lb)[~empty].all(), (g - lse)[~empty].abs().max()


def call(L, q, k, v, ql, kl, causal, scale=None, **kw):
    plan = L.losa_packed_plan(ql, kl, q.shape[1], k.shape[1], q.dtype, causal=causal,
                              **{x: kw.pop(x) for x in ("q_starts", "k_starts") if x in kw})
    ws = plan.workspace(q.shape[2])
    if ws is not None:
        ws.fill_(255)  # every float a NaN
    return L.losa_packed_attn_fwd(q, k, v, plan, scale=scale, want_lse=True, workspace=ws, **kw)


BF, F = torch.bfloat16, torch.float32
CASES = [  # dtype, d, H, Hkv, causal, q_lens, k_lens
    # each tile, sub-tile and half of the loop, one off either way
    (BF, 128, 2, 2, False, (1, 31, 32, 33, 127, 128, 129, 300), (1, 31, 32, 33, 63, 64, 65, 300)),
    (BF, 64, 3, 3, False, (129, 64, 257, 40), (95, 96, 97, 161)),
    (BF, 128, 2, 2, True, (1, 31, 33, 128, 129, 300, 513), None),
    (BF, 64, 4, 2, True, (65, 1, 200, 127, 400), None),
    # grouped heads, groups that do not divide a tile
    (BF, 128, 6, 2, True, (100, 43, 1, 257), None), (BF, 64, 10, 2, True, (77, 5, 130), None),
    (BF, 128, 8, 1, False, (70, 4, 3, 200), (300, 1000, 129, 64)),
    # a block of new tokens over a cache; a cache shorter than the queries (rows that see nothing)
    (BF, 128, 2, 1, True, (160, 200, 130), (500, 90, 7)), (BF, 64, 2, 2, True, (300, 40, 140), (1000, 39, 0)),
    # few rows: single tokens, parts, ragged ends, nothing to see
    (BF, 128, 8, 2, True, (1, 1, 1, 1, 1, 1), (1, 127, 128, 129, 3000, 40_001)),
    (BF, 64, 4, 4, True, (1, 2, 7, 32, 5, 1, 3), (5000, 300, 1000, 700, 3, 0, 1)),
    (BF, 128, 24, 1, False, (1, 1, 1), (513, 7000, 64)), (BF, 128, 96, 3, True, (1, 1), (900, 31)),
    (BF, 64, 5, 1, False, (6, 1), (20_000, 70_000)),
    # tiles whose keys are split: drafted tokens and chunks over a cache
    (BF, 128, 8, 1, True, (7, 5, 33, 16), (9000, 2048, 4111, 2047)),
    (BF, 64, 8, 2, True, (100, 9, 256), (6000, 20_003, 2600)), (BF, 128, 6, 2, False, (43, 11), (2049, 30_000)),
    # mixed
    (BF, 128, 4, 2, True, (0, 1, 600, 3, 0, 17, 64), (4, 900, 600, 3, 0, 2100, 64)),
    (F, 128, 2, 2, False, (1, 15, 16, 17, 31, 32, 33, 150), (1, 31, 32, 33, 255, 256, 257, 300)),
    # few keys: 1, 2, 4 or 8 waves to a row set
    (F, 128, 2, 2, False, (300, 257, 150, 90, 33, 129), (32, 100, 200, 64, 33, 7)),
    (F, 64, 6, 2, True, (64, 100, 65, 129, 31, 20), None), (F, 128, 3, 1, True, (50, 90, 30), (64, 128, 7)),
    (F, 64, 6, 2, True, (100, 1, 333, 64), None), (F, 128, 3, 1, True, (40, 130), (300, 60)),
    (F, 128, 4, 1, True, (20, 5, 64), (3001, 9000, 2048)), (F, 64, 3, 1, False, (90, 6), (2050, 7000)),
    (F, 64, 8, 2, True, (1, 4, 2, 1), (3000, 511, 513, 20_011)),
    (F, 128, 4, 4, True, (1, 16, 3, 0, 9), (0, 2000, 2, 5, 1100)),
    (F, 128, 32, 2, False, (1, 1), (700, 5000)),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", "").replace("torch.", ""))
def test_against_plain_attention(L, case):
    dtype, d, H, Hkv, causal, ql, kl = case
    kl = ql if kl is None else kl
    print(f"[gpu-packed] {case}", flush=True)
    q = randn(sum(ql), H, d, seed=1, dtype=dtype).cuda()
    kv = randn(sum(kl), 2 * Hkv, d, seed=2, dtype=dtype).cuda()
    k, v = kv[:, :Hkv], kv[:, Hkv:]
    o, lse = call(L, q, k, v, ql, kl, causal)
    a = b = 0
    for x, y in zip(ql, kl):
        if x:
            ref = reference(q[a:a + x], k[b:b + y], v[b:b + y], causal, d ** -0.5)
            check(o[a:a + x], lse[:, a:a + x], ref, y, d)
        a, b = a + x, b + y


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("causal", [False, True])
def test_peaked_and_shifted_scores(L, dtype, causal):
    """Score gaps of hundreds, all scores far from 0, a maximum that keeps rising."""
    d, ql = 128, (200, 1, 90)
    for kind in ("peaked", "shifted", "rising"):
        q = randn(sum(ql), 2, d, seed=3, dtype=F)
        k = randn(sum(ql), 2, d, seed=4, dtype=F)
        if kind == "peaked":
            q, k = q * 10, k * 10
        elif kind == "shifted":
            q, k = q + 4, k - 4
        else:
            q[:] = 2.0
            k = k * 0.1 + torch.linspace(-3, 3, len(k))[:, None, None]
        q, k, v = q.to(dtype).cuda(), k.to(dtype).cuda(), randn(sum(ql), 2, d, seed=5, dtype=dtype).cuda()
        o, lse = call(L, q, k, v, ql, ql, causal, scale=0.2)
        a = 0
        for x in ql:
            ref = reference(q[a:a + x], k[a:a + x], v[a:a + x], causal, 0.2)
            check(o[a:a + x], lse[:, a:a + x], ref, x, d)
            a += x


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_sequence_gives_the_same_bits_alone_and_packed(L, dtype):
    d, ql, kl = 128, (300, 1, 2, 150, 1), (300, 9000, 400, 700, 64)
    q = randn(sum(ql), 4, d, seed=6, dtype=dtype).cuda()
    k, v = (randn(sum(kl), 2, d, seed=s, dtype=dtype).cuda() for s in (7, 8))
    o, lse = call(L, q, k, v, ql, kl, True)
    a = b = 0
    for x, y in zip(ql, kl):
        o1, l1 = call(L, q[a:a + x], k[b:b + y], v[b:b + y], [x], [y], True)
        assert torch.equal(o1, o[a:a + x]) and torch.equal(l1, lse[:, a:a + x])
        o1, _ = call(L, q[a:a + x, 2:], k[b:b + y, 1:], v[b:b + y, 1:], [x], [y], True)
        assert torch.equal(o1, o[a:a + x, 2:])  # a head's group alone
        a, b = a + x, b + y


def test_fp32_rows_give_the_same_bits_in_a_large_call(L):
    """A call of many units takes row sets of 32 rows, a small one of 16."""
    d, ql, kl = 64, (130, 77, 40, 90_000), (20, 60, 200, 31)
    q = randn(sum(ql), 4, d, seed=80, dtype=F).cuda()
    k, v = (randn(sum(kl), 2, d, seed=s, dtype=F).cuda() for s in (81, 82))
    for causal in (False, True):
        o, lse = call(L, q, k, v, ql, kl, causal)
        a = b = 0
        for x, y in zip(ql[:3], kl):
            o1, l1 = call(L, q[a:a + x], k[b:b + y], v[b:b + y], [x], [y], causal)
            assert torch.equal(o1, o[a:a + x]) and torch.equal(l1, lse[:, a:a + x])
            a, b = a + x, b + y


@pytest.mark.parametrize("dtype", [BF, F])
def test_layouts_gaps_and_shared_keys(L, dtype):
    """Starts with gaps and in any order, keys shared by sequences, head-major tensors;
    rows that no sequence owns stay as they were."""
    d, H, Hkv = 64, 4, 2
    ql, kl = [140, 1, 60], [200, 333, 200]
    qs, ks = [300, 7, 100], [50, 400, 50]
    q = randn(500, H, d, seed=9, dtype=dtype).cuda()
    k, v = (randn(800, Hkv, d, seed=s, dtype=dtype).cuda() for s in (10, 11))
    out = torch.full_like(q, 3.0)
    lse = torch.full((H, 500), 7.0, device="cuda")
    call(L, q, k, v, ql, kl, True, q_starts=qs, k_starts=ks, out=out, lse=lse)
    own = torch.zeros(500, dtype=torch.bool, device="cuda")
    for x, y, a, b in zip(ql, kl, qs, ks):
        want, wl = call(L, q[a:a + x], k[b:b + y], v[b:b + y], [x], [y], True)
        assert torch.equal(out[a:a + x], want) and torch.equal(lse[:, a:a + x], wl)
        own[a:a + x] = True
    assert (out[~own] == 3).all() and (lse[:, ~own] == 7).all()
    hm = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    room = hm(torch.full_like(q, 3.0))
    call(L, hm(q), hm(k), hm(v), ql, kl, True, q_starts=qs, k_starts=ks, out=room)
    assert torch.equal(room, out)
    y = q.clone()  # in place
    call(L, y, k, v, ql, kl, True, q_starts=qs, k_starts=ks, out=y)
    assert torch.equal(y[own], out[own]) and torch.equal(y[~own], q[~own])
    one = k[:1].expand(800, Hkv, d)[:1]
    o, _ = call(L, q[:3], one, v[:1], [3], [1], False)
    assert torch.equal(o, v[:1].repeat_interleave(H // Hkv, 1).expand(3, H, d))


def test_padded_layout_of_the_sparse_path(L):
    """[B, H, N_pad, d] tensors, addressed as rows of d with a start per batch: a dense
    step equals the construction step's output on every valid row, within two roundings
    of its values (both forms round their probabilities and outputs to bf16)."""
    B, H, N, d, C = 2, 3, 333, 128, 128
    n_pad = L.padded_len(N, C, C)
    q, k, v = (randn(B, H, n_pad, d, seed=s, dtype=BF).cuda() for s in (12, 13, 14))
    for t in (q, k, v):
        t[:, :, N:] = 0
    rows = ((B - 1) * H + 1) * n_pad
    flat = lambda t: t.as_strided((rows, H, d), (d, n_pad * d, 1))  # noqa: E731
    out = torch.zeros_like(q)
    starts = [b * H * n_pad for b in range(B)]
    plan = L.losa_packed_plan([N] * B, [N] * B, H, H, BF, q_starts=starts, k_starts=starts)
    L.losa_packed_attn_fwd(flat(q), flat(k), flat(v), plan, out=flat(out))
    o, _ = L.losa_construct(q, k, v, N, C, C)
    assert not out[:, :, N:].any()
    w = torch.softmax(q[:, :, :N].float() @ k[:, :, :N].float().transpose(2, 3).contiguous() / d ** 0.5, 3)
    size = w @ v[:, :, :N].float().abs().contiguous()
    err = (out.float() - o.float())[:, :, :N].abs()
    assert (err <= 2 * (2.0 ** -8 * (size + o.float()[:, :, :N].abs()) + 1e-3 * size)).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_does_not_reach_it(L, dtype, bad):
    """Values that are not finite in other sequences, behind the end, and at future keys."""
    d, H, Hkv = 128, 4, 2
    ql, kl = [150, 3, 200, 40, 1], [150, 1000, 260, 40, 700]
    k, v = (randn(sum(kl), Hkv, d, seed=s, dtype=dtype).cuda() for s in (15, 16))
    q = randn(sum(ql), H, d, seed=17, dtype=dtype).cuda()
    want, wl = call(L, q, k, v, ql, kl, True)
    ends_q = [sum(ql[:i]) for i in range(len(ql) + 1)]
    ends_k = [sum(kl[:i]) for i in range(len(kl) + 1)]
    for i in range(len(ql)):
        # everything outside sequence i
        k2, v2 = k.clone(), v.clone()
        for t in (k2, v2):
            t[:ends_k[i]] = bad
            t[ends_k[i + 1]:] = bad
        o, lse = call(L, q, k2, v2, ql, kl, True)
        s = slice(ends_q[i], ends_q[i + 1])
        assert torch.equal(o[s], want[s]) and torch.equal(lse[:, s], wl[:, s]), i
    # future keys: from key c on, rows that see none of them
    for i, cut in ((0, 5), (0, 100), (0, 149), (1, 998), (1, 999), (2, 70), (2, 259), (3, 33)):
        for which in range(3):
            k2, v2 = k.clone(), v.clone()
            if which != 1:
                v2[ends_k[i] + cut:ends_k[i + 1]] = bad
            if which != 0:
                k2[ends_k[i] + cut:ends_k[i + 1]] = bad
            o, lse = call(L, q, k2, v2, ql, kl, True)
            first = cut - (kl[i] - ql[i])  # the first row that sees key `cut`
            s = slice(ends_q[i], ends_q[i] + max(0, first))
            if dtype == F and which == 1:
                assert torch.equal(o[s], want[s])
            ref = reference(q[s.start:ends_q[i + 1]], k[ends_k[i]:ends_k[i + 1]],
                            v[ends_k[i]:ends_k[i + 1]], True, d ** -0.5)
            n = max(0, first)
            check(o[s], lse[:, s], tuple(x[:n] if x.dim() == 3 else x[:, :n] for x in ref), kl[i], d)
            if which == 0 and first < ql[i]:  # and rows that see one are not finite
                seen = o[ends_q[i] + max(0, first):ends_q[i + 1]]
                assert not torch.isfinite(seen).any()


@pytest.mark.parametrize("dtype", [BF, F])
def test_tiles_over_a_long_cache(L, dtype):
    """Rows of tiles whose keys are split: the same bits alone and packed, values that are
    not finite at keys that a row does not see."""
    d, ql, kl = 64, (90, 40, 300, 2600), (5000, 2500, 700, 2300)
    q = randn(sum(ql), 4, d, seed=70, dtype=dtype).cuda()
    k, v = (randn(sum(kl), 2, d, seed=s, dtype=dtype).cuda() for s in (71, 72))
    o, lse = call(L, q, k, v, ql, kl, True)
    a = b = 0
    for x, y in zip(ql, kl):
        o1, l1 = call(L, q[a:a + x], k[b:b + y], v[b:b + y], [x], [y], True)
        assert torch.equal(o1, o[a:a + x]) and torch.equal(l1, lse[:, a:a + x])
        a, b = a + x, b + y
    ref = reference(q[:90], k[:5000], v[:5000], True, d ** -0.5)
    check(o[:90], lse[:, :90], ref, 5000, d)
    for cut in (4915, 4950, 4999):
        v2 = v.clone()
        v2[cut:5000] = float("nan")
        k2 = k.clone()
        k2[cut:5000] = float("inf")
        n = cut - 4910  # rows that see no key from `cut` on
        o2, l2 = call(L, q, k2, v2, ql, kl, True)
        check(o2[:n], l2[:, :n], tuple(x[:n] if x.dim() == 3 else x[:, :n] for x in ref), 5000, d)
        assert not torch.isfinite(o2[n:90]).any() and torch.equal(o2[90:], o[90:])
    for keys in (2048, 130):  # the fewest that are split; rows that see nothing
        o, lse = call(L, q[:256], k[:keys], v[:keys], [256], [keys], True)
        check(o, lse, reference(q[:256], k[:keys], v[:keys], True, d ** -0.5), keys, d)


@pytest.mark.parametrize("dtype", [BF, F])
def test_no_key_at_all(L, dtype):
    """k and v without a row; rows that see nothing are 0, their lse -inf."""
    q = randn(40, 4, 64, seed=60, dtype=dtype).cuda()
    k = torch.empty(0, 2, 64, dtype=dtype, device="cuda")
    for causal in (False, True):
        for ql in ([40], [1, 39], [16, 24]):
            o, lse = call(L, q, k, k, ql, [0] * len(ql), causal, k_starts=[99] * len(ql),
                          out=torch.full_like(q, 2.0))
            assert not o.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_plan_that_is_none_writes_nothing(L, dtype):
    """Units and joins outside q, k and the workspace are passed over."""
    d, ql, kl = 128, [3, 200], [3000, 200]
    q = randn(sum(ql), 4, d, seed=61, dtype=dtype).cuda()
    k, v = (randn(sum(kl), 2, d, seed=s, dtype=dtype).cuda() for s in (62, 63))
    plan = L.losa_packed_plan(ql, kl, 4, 2, dtype, causal=True)
    good = plan.data.clone()
    ws = plan.workspace(d)
    for fill in (-1, 0x7f7f7f7f7f7f7f7f, 1 << 40):
        plan.data.fill_(fill)
        ws.zero_()
        out, lse = torch.full_like(q, 5.0), torch.full((4, sum(ql)), 6.0, device="cuda")
        L.losa_packed_attn_fwd(q, k, v, plan, want_lse=True, out=out, lse=lse, workspace=ws)
        assert (out == 5).all() and (lse == 6).all() and not ws.any(), fill
    plan.data.copy_(good)
    want, _ = call(L, q, k, v, ql, kl, True)
    assert torch.equal(L.losa_packed_attn_fwd(q, k, v, plan), want)


def test_infinite_value_of_one_channel(L):
    """One infinite value at one key: only that channel, only the rows that see it."""
    for dtype in (BF, F):
        q, k, v = (randn(170, 2, 64, seed=s, dtype=dtype).cuda() for s in (18, 19, 20))
        want, _ = call(L, q, k, v, [170], [170], True)
        v[77, 1, 13] = float("inf")
        o, _ = call(L, q, k, v, [170], [170], True)
        assert (o[77:, 1, 13] == float("inf")).all()
        bad = torch.zeros_like(o, dtype=torch.bool)
        bad[77:, 1, 13] = True
        assert torch.isfinite(o[~bad]).all()
        ref = reference(q, k, torch.where(torch.isinf(v), 0.0, v), True, 64 ** -0.5)
        keep = ~bad.cpu()
        bound = torch.finfo(dtype).eps / 2 * ref[0].abs() + ref[1] * (2.0 ** -8 if dtype == BF else 1e-4)
        assert ((o.double().cpu() - ref[0]).abs() <= bound + 1e-3 * ref[1])[keep].all()


def test_a_cache_beyond_32_bits_of_bytes(L):
    """A row stride that puts the end of the cache past 4 GiB: bitwise as a dense cache."""
    rows, d = 70_000, 64
    for dtype, ql in ((BF, [2, 70]), (F, [2])):
        wide = torch.empty(rows, 70_000 // torch.finfo(dtype).bits // 8 * 8 * 8, dtype=dtype, device="cuda")
        assert wide.nbytes > 1 << 32
        k, v = wide[:, 64:128].unsqueeze(1), wide[:, -64:].unsqueeze(1)
        k.copy_(randn(rows, 1, d, seed=21, dtype=dtype))
        v.copy_(randn(rows, 1, d, seed=22, dtype=dtype))
        q = randn(sum(ql), 2, d, seed=23, dtype=dtype).cuda()
        starts = [0] * len(ql)
        got = call(L, q, k, v, ql, [rows] * len(ql), True, k_starts=starts)
        want = call(L, q, k.contiguous(), v.contiguous(), ql, [rows] * len(ql), True, k_starts=starts)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [BF, F])
def test_streams_graphs_and_a_shared_workspace(L, dtype):
    """Two captured calls that share a workspace, replayed in turn with eager work between."""
    d = 128
    sets = []
    for i, (ql, kl) in enumerate((([1, 1, 40], [3000, 700, 40]), ([3, 260], [5000, 260]))):
        q = randn(sum(ql), 4, d, seed=30 + i, dtype=dtype).cuda()
        k, v = (randn(sum(kl), 2, d, seed=40 + 2 * i + j, dtype=dtype).cuda() for j in (0, 1))
        plan = L.losa_packed_plan(ql, kl, 4, 2, dtype, causal=True)
        sets.append((q, k, v, plan, torch.empty_like(q), torch.empty(4, sum(ql), device="cuda")))
    ws = torch.empty(max(s[3].workspace_bytes(d) for s in sets), dtype=torch.uint8, device="cuda")

    def run(s):
        L.losa_packed_attn_fwd(*s[:4], want_lse=True, out=s[4], lse=s[5], workspace=ws)

    for s in sets:
        run(s)
    torch.cuda.synchronize()
    ref = [(s[4].clone(), s[5].clone()) for s in sets]
    side = torch.cuda.Stream()
    graphs = []
    for s in sets:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(s)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(s)
        graphs.append(g)
    for rep in range(4):
        for s in sets:
            s[4].fill_(rep)
            s[5].fill_(rep)
        ws.fill_(255)
        torch.cuda.synchronize()
        for g in (graphs if rep % 2 else graphs[::-1]):
            g.replay()
        torch.cuda.synchronize()
        for s, (o, lse) in zip(sets, ref):
            assert torch.equal(s[4], o) and torch.equal(s[5], lse), rep


def test_a_layer_of_packed_clips(L):
    """Projections of two clips of different sizes and their prompts, as a layer runs them:
    norms and rotation into packed rows, self-attention of each clip, text attention, and
    the sparse path on one clip from the same projections."""
    H, d, grids, text = 4, 128, [(2, 6, 9), (1, 7, 11)], [13, 40]
    lens = [a * b * c for a, b, c in grids]
    total = sum(lens)
    x = randn(1, total, 3 * H, d, seed=50, dtype=BF).cuda()
    pos = torch.cat([torch.stack([g.flatten() for g in torch.meshgrid(
        *[torch.arange(s) for s in sizes], indexing="ij")]) for sizes in grids], 1).to(torch.int32).cuda()
    table = L.losa_rope_table((44, 42, 42), (2, 7, 11))
    packed = [torch.empty(1, total, H, d, dtype=BF, device="cuda") for _ in range(2)]
    w = (1 + 0.1 * torch.randn(d, generator=torch.Generator().manual_seed(51))).cuda()
    L.losa_qk_norm_rope(x[:, :, :H], x[:, :, H:2 * H], q_weight=w, k_weight=w, table=table, pos=pos,
                        q_out=packed[0].transpose(1, 2), k_out=packed[1].transpose(1, 2))
    q, k, v = packed[0][0], packed[1][0], x[0, :, 2 * H:]
    plan = L.losa_packed_plan(lens, None, H, H, BF)
    o = L.losa_packed_attn_fwd(q, k, v, plan)
    for i, n in enumerate(lens):
        s = slice(sum(lens[:i]), sum(lens[:i + 1]))
        check(o[s], None, reference(q[s], k[s], v[s], False, d ** -0.5), n, d)
    kt, vt = (randn(sum(text), H, d, seed=s, dtype=BF).cuda() for s in (52, 53))
    plan_t = L.losa_packed_plan(lens, text, H, H, BF)
    ot = L.losa_packed_attn_fwd(q, kt, vt, plan_t)
    for i, n in enumerate(lens):
        s, t = slice(sum(lens[:i]), sum(lens[:i + 1])), slice(sum(text[:i]), sum(text[:i + 1]))
        check(ot[s], None, reference(q[s], kt[t], vt[t], False, d ** -0.5), text[i], d)
    # clip 0 through the sparse path: the same rows, laid out and padded
    n, C = lens[0], 64
    n_pad = L.padded_len(n, C, C)
    ps = L.losa_qk_norm_rope(x[:, :n, :H], x[:, :n, H:2 * H], x[:, :n, 2 * H:], q_weight=w, k_weight=w,
                             table=table, pos=pos[:, :n].contiguous(), n_pad=n_pad)
    assert torch.equal(ps[0][0, :, :n].transpose(0, 1), q[:n])
    od, mass = L.losa_construct(*ps, n, C, C)
    check(od[0, :, :n].transpose(0, 1), None, reference(q[:n], k[:n], v[:n], False, d ** -0.5), n, d)


def test_device_argument_checks(L):
    q = torch.zeros(10, 4, 64, device="cuda", dtype=BF)
    k = torch.zeros(500, 2, 64, device="cuda", dtype=BF)
    p = L.losa_packed_plan([4, 6], [300, 200], 4, 2, BF)
    short = torch.empty(16, dtype=torch.uint8, device="cuda")
    cases = [
        (lambda: L.losa_packed_attn_fwd(q, k, k, None), TypeError, "PackedPlan"),
        (lambda: L.losa_packed_attn_fwd(q[0], k, k, p), ValueError, "rows, heads, d"),
        (lambda: L.losa_packed_attn_fwd(q.float(), k, k, p), TypeError, "q must be"),
        (lambda: L.losa_packed_attn_fwd(q[:, :2], k, k, p), ValueError, "q must have shape"),
        (lambda: L.losa_packed_attn_fwd(q, k[:, :1], k, p), ValueError, "k must have shape"),
        (lambda: L.losa_packed_attn_fwd(q, k, k[:, :, :32], p), ValueError, "v must have shape"),
        (lambda: L.losa_packed_attn_fwd(q, k, k[:499], p), ValueError, "v must have shape"),
        (lambda: L.losa_packed_attn_fwd(q, k[:499], k[:499], p), L.LosaError, "INVALID_SHAPE"),
        (lambda: L.losa_packed_attn_fwd(q[:9], k, k, p), L.LosaError, "INVALID_SHAPE"),
        (lambda: L.losa_packed_attn_fwd(q, k, k, p, out=q[:9].clone()), ValueError, "out must have"),
        (lambda: L.losa_packed_attn_fwd(q, k, k, p, workspace=short), ValueError, "workspace holds"),
        (lambda: L.losa_packed_attn_fwd(q, k, k, p, scale=-1.0), L.LosaError, "scale"),
        (lambda: L.losa_packed_attn_fwd(q, k, k, p, want_lse=True, lse=torch.empty(4, 9, device="cuda")),
         ValueError, "lse must have"),
        (lambda: L.losa_packed_attn_fwd(q.cpu(), k, k, p), ValueError, "must live on"),
    ]
    for fn, exc, msg in cases:
        with pytest.raises(exc, match=msg):
            fn()
    assert L.losa_packed_attn_fwd(q, k, k, p).shape == q.shape


@pytest.mark.parametrize("dtype", [BF, F])
def test_units_at_the_end_of_64_bits_write_nothing(L, dtype):
    """Rows of q or k next to 2^63 in a plan: outside whatever is added to them."""
    d, ql, kl = 128, [3, 200], [3000, 200]
    q = randn(sum(ql), 4, d, seed=64, dtype=dtype).cuda()
    k, v = (randn(sum(kl), 2, d, seed=s, dtype=dtype).cuda() for s in (65, 66))
    plan = L.losa_packed_plan(ql, kl, 4, 2, dtype, causal=True)
    good, ws = plan.data.clone(), plan.workspace(d)
    units = 5 * (plan.info.n_tiles + plan.info.n_few)  # 40 bytes each, q_row and k_row first
    for word in (0, 1):
        for far in (2 ** 63 - 1, 2 ** 63 - 2, 2 ** 63 - 30):
            print(f"[gpu-packed] unit word {word} = {far}", flush=True)
            plan.data.copy_(good)
            plan.data[word:units:5] = far
            plan.data[units::3] = 2 ** 63 - 1  # joins: 24 bytes, q_row first
            ws.zero_()
            out, lse = torch.full_like(q, 5.0), torch.full((4, sum(ql)), 6.0, device="cuda")
            L.losa_packed_attn_fwd(q, k, v, plan, want_lse=True, out=out, lse=lse, workspace=ws)
            assert (out == 5).all() and (lse == 6).all() and not ws.any(), (word, far)
