"""The operators around the sparse attention path, as cases that can be timed and compared.

A case is one call through the public binding `paper_2608_12032_amd.losa`.  `op` says which:

  rope    rotary positions with one to three axes: token-major x to the library's padded
          head-major layout
  qknorm  norms of queries and keys with the rotation in the same pass, values laid out beside them
  attn    attention over packed sequences of different lengths, with grouped heads

`run` computes each in its plain form, elementary torch operations in 32 bits, or, where `own` is
set, with the library's kernels.
"""
import math

import torch

own = False

ROPE = {"op": "rope", "dtype": "bf16", "B": 1, "T": 21, "Hg": 30, "Wg": 52, "text": 0, "H": 12,
        "d": 128, "axes": 3, "rot": 128, "pairing": "interleaved", "packed": 3, "pad": 128}
QKNORM = dict(ROPE, op="qknorm", Hkv=12, norm="rms", over="head", bias=False, rotate=True)
ATTN = {"op": "attn", "dtype": "bf16", "H": 12, "Hkv": 12, "d": 128, "q_lens": "", "k_lens": "",
        "causal": False, "lse": False}


def listed():
    def case(base, name, **kw):
        return dict(base, name=name, **kw)

    return [
        # one patch row of the tiny fp32 workload: the smallest call, where latency counts
        case(ROPE, "rope-patches-f32", dtype="f32", T=1, Hg=4, Wg=13, H=2, d=64, rot=64, pad=64),
        # queries of the Wan2.1-1.3B shape, 81 frames at 480p, out of a fused q, k, v projection
        case(ROPE, "rope-wan"),
        # a batch of stills, two axes, rotated halves, a quarter of each head left as it is
        case(ROPE, "rope-stills-halves", B=4, T=1, Hg=45, Wg=80, H=16, d=64, axes=2, rot=48,
             pairing="halves", packed=1),
        # one streamed token for each of eight requests, grouped heads, one axis
        case(QKNORM, "qknorm-token", B=8, T=1, Hg=1, Wg=1, H=16, Hkv=4, axes=1, pairing="halves",
             pad=1),
        # the Wan2.1-1.3B layer: norms over all heads together
        case(QKNORM, "qknorm-wan", over="all"),
        # text and video tokens in one sequence, layer norms with bias, 64-wide heads, ragged
        case(QKNORM, "qknorm-joint-layer", T=13, Wg=45, text=226, H=30, Hkv=30, d=64, rot=64,
             norm="layer", bias=True),
        # fp32, both guidance branches, odd grid
        case(QKNORM, "qknorm-clip-f32", dtype="f32", B=2, T=3, Hg=29, Wg=51, H=4, Hkv=4),
        # prompts of a text encoder, causal, grouped heads, from one token to a thousand
        case(ATTN, "attn-prompts", H=32, Hkv=8, q_lens="1 77 226 512 1024 300 19 768 129 640",
             causal=True),
        # a dense step before the construction step for clips of different sizes in one batch
        case(ATTN, "attn-clips", q_lens="32760 7800 1560"),
        # video queries over text keys, one ragged prompt per clip
        case(ATTN, "attn-text", H=30, Hkv=30, d=64, q_lens="17550 17550 5850", k_lens="226 77 512"),
        # one new token for each of sixteen requests over caches of a few keys to a long clip
        case(ATTN, "attn-token", H=32, Hkv=8, q_lens="1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1",
             k_lens="32760 7 1560 8193 4096 129 17550 1 31 2048 12000 640 5000 9999 255 20480",
             causal=True, lse=True),
        # fp32, causal, ragged, grouped
        case(ATTN, "attn-prompts-f32", dtype="f32", H=6, Hkv=2, d=64, q_lens="700 333 1 1027 64",
             causal=True, lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over the whole range, in proportion to their logarithm."""
    op = rng.choice(["rope", "qknorm", "qknorm", "attn", "attn", "attn"])
    c = dict({"rope": ROPE, "qknorm": QKNORM, "attn": ATTN}[op])
    c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c["d"] = rng.choice([64, 128])
    if op == "attn":
        c["Hkv"] = rng.choice([1, 2, 3, 4, 8, 12])
        c["H"] = c["Hkv"] * rng.choice([1, 1, 2, 3, 4, 8])
        c["causal"] = rng.choice([True, False])
        c["lse"] = rng.choice([True, False])
        kind = rng.choice(["self", "self", "cross", "rows"])
        # scores of the whole call
        most = 9.3 if c["dtype"] == "f32" else 10.0
        scores = 10 ** rng.uniform(4.0, 8.5 if kind == "rows" else most)
        n = rng.choice([1, 2, 3, 5, 8, 16])
        ql, kl = [], []
        for _ in range(n):
            each = scores / c["H"] / n * rng.uniform(0.2, 1.8)
            if kind == "self":
                q = min(32760, max(1, int(math.sqrt(each))))
                k = q
            elif kind == "cross":
                k = _log(rng, 1, 1024)
                q = max(1, int(min(32760 * rng.uniform(0.2, 1.0), each / k)))
                c["causal"] = False
            else:
                q = rng.choice([1, 1, 1, 2, 4, 7])
                k = _log(rng, 1, max(2, min(120000, 4 * each / q)))  # some shorter than q
            ql.append(q)
            kl.append(k)
        c["q_lens"] = " ".join(map(str, ql))
        c["k_lens"] = "" if kind == "self" else " ".join(map(str, kl))
        return c
    c["B"] = rng.choice([1, 1, 2, 4])
    c["H"] = rng.choice([1, 2, 3, 5, 8, 12, 16, 30, 40])
    c["axes"] = rng.choice([1, 2, 3, 3])
    c["pairing"] = rng.choice(["interleaved", "interleaved", "halves"])
    c["rot"] = rng.choice([c["d"], c["d"], c["d"] // 4 * 3, c["d"] // 2])
    c["packed"] = rng.choice([1, 3])
    c["text"] = rng.choice([0, 0, 77, 226])
    c["pad"] = rng.choice([1, 64, 128])
    n = _log(rng, 1, min(120000, 90e6 / (c["B"] * c["H"] * c["d"])))
    c["T"] = max(1, min(33, round(n ** 0.3 * rng.uniform(0.5, 1.5)))) if c["axes"] == 3 else 1
    c["Hg"] = max(1, round(math.sqrt(n / c["T"]) * rng.uniform(0.6, 1.0))) if c["axes"] > 1 else 1
    c["Wg"] = max(1, n // (c["T"] * c["Hg"]))
    if op == "qknorm":
        c["Hkv"] = rng.choice([h for h in (1, 2, 3, 4, 5, 8, 12, 16, 30, 40) if c["H"] % h == 0])
        c["norm"] = rng.choice(["rms", "rms", "layer"])
        c["over"] = rng.choice(["head", "head", "all"])
        c["bias"] = c["norm"] == "layer" and rng.choice([True, False])
        c["rotate"] = rng.choice([True, True, True, False])
    return c


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _tokens(c):
    n = c["text"] + c["T"] * c["Hg"] * c["Wg"]
    return n, -(-n // c["pad"]) * c["pad"]


def _axes(c):
    """Rotated dims of each axis, and the number of its positions."""
    dims = {1: [1.0], 2: [0.5], 3: [0.25, 0.375]}[c["axes"]]
    dims = [int(c["rot"] * x) // 2 * 2 for x in dims]
    if c["axes"] > 1:
        dims.append(c["rot"] - sum(dims))
    grid = [c["T"], c["Hg"], c["Wg"]]
    return dims, grid[3 - c["axes"]:]


def _positions(c):
    """int32 [axes, N]: text tokens come first and are not rotated (-1)."""
    grid = torch.meshgrid(*[torch.arange(x, device="cuda") for x in _axes(c)[1]], indexing="ij")
    video = torch.stack([g.flatten() for g in grid])
    text = torch.full((c["axes"], c["text"]), -1, device="cuda")
    return torch.cat([text, video], 1).to(torch.int32)


def _angles(c):
    """[N, rot / 2] in 64 bits."""
    pos, out = _positions(c).double(), []
    for a, dim in enumerate(_axes(c)[0]):
        freq = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
        out.append(pos[a].clamp(min=0)[:, None] * freq)
    return torch.cat(out, 1)


def _lens(c):
    q = [int(x) for x in c["q_lens"].split()]
    return q, [int(x) for x in c["k_lens"].split()] or q


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(7919 * seed + 17)

    def randn(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(scale)

    st = {"case": c}
    if c["op"] == "attn":
        # queries and keys as they leave a norm: unit variance, the heads' weights around one
        q_lens, k_lens = _lens(c)
        H, Hkv, d = c["H"], c["Hkv"], c["d"]
        st["q"] = (randn(sum(q_lens), H, d) * (1 + randn(H, 1, scale=0.2))).to(_type(c))
        if c["k_lens"]:  # keys and values of their own: one projection
            kv = torch.cat([randn(sum(k_lens), Hkv, d), randn(sum(k_lens), Hkv, d)], 1).to(_type(c))
            st["k"], st["v"] = kv[:, :Hkv], kv[:, Hkv:]
        else:  # self-attention: keys and values each in a tensor
            st["k"] = randn(sum(k_lens), Hkv, d).to(_type(c))
            st["v"] = randn(sum(k_lens), Hkv, d).to(_type(c))
        st["q_lens"], st["k_lens"] = q_lens, k_lens
        st["out"] = torch.empty_like(st["q"])
        if own:  # the batch's plan and workspace, which every layer and step of it uses
            from paper_2608_12032_amd import losa
            st["plan"] = losa.losa_packed_plan(q_lens, k_lens, H, Hkv, _type(c),
                                               causal=c["causal"])
            st["workspace"] = st["plan"].workspace(d)
        return st

    n, n_pad = _tokens(c)
    heads = [c["H"]] if c["op"] == "rope" else [c["H"], c["Hkv"], c["Hkv"]]
    scale = 1.0 + randn(1, 1, 1, c["d"], scale=0.3)  # projections: channels of uneven size
    if c["packed"] == 3:  # slices of one fused projection
        H = c["H"] * 3 if c["op"] == "rope" else sum(heads)
        whole = (randn(c["B"], n, H, c["d"]) * scale).to(_type(c))
        st["x"] = [whole[:, :, sum(heads[:i]):sum(heads[:i + 1])] for i in range(len(heads))]
    else:
        st["x"] = [(randn(c["B"], n, h, c["d"]) * scale).to(_type(c)) for h in heads]
    st["out"] = [torch.empty(c["B"], h, n_pad, c["d"], dtype=_type(c), device="cuda")
                 for h in heads]
    if c["op"] == "qknorm":
        span = [c["d"] if c["over"] == "head" else h * c["d"] for h in heads[:2]]
        st["weight"] = [1 + randn(s, scale=0.2) for s in span]
        st["bias"] = [randn(s, scale=0.1) if c["bias"] else None for s in span]
    # the position table of the grid, which every layer and step uses
    angle = _angles(c)
    rotated = (_positions(c)[:1] >= 0).t()
    st["cos"] = torch.where(rotated, angle.cos(), 1.0).float()[None, :, None, :]
    st["sin"] = torch.where(rotated, angle.sin(), 0.0).float()[None, :, None, :]
    if own:
        from paper_2608_12032_amd import losa
        dims, lens = _axes(c)
        st["table"] = losa.losa_rope_table(dims, lens, base=10000.0)
        st["pos"] = _positions(c)
    return st


def _rotate(c, x, cos, sin):
    """Rotation of x [B, N, H, d] in 32 bits."""
    r = c["rot"]
    head, tail = x[..., :r], x[..., r:]
    if c["pairing"] == "halves":
        a, b = head[..., :r // 2], head[..., r // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, tail], -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), tail], -1)


def _norm(c, x, weight, bias):
    """Norm of x [B, N, H, d] in 32 bits over each head or over all of them."""
    y = x if c["over"] == "head" else x.flatten(2)
    if c["norm"] == "layer":
        y = y - y.mean(-1, keepdim=True)
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight
    if bias is not None:
        y = y + bias
    return y.view(x.shape)


def _lay_out(c, y):
    """[B, N, H, d] to [B, H, N_pad, d], padding rows 0, rounded once."""
    n, n_pad = _tokens(c)
    out = torch.zeros(y.shape[0], y.shape[2], n_pad, c["d"], dtype=_type(c), device=y.device)
    out[:, :, :n] = y.transpose(1, 2)
    return out


def _attend(c, q, k, v):
    """Attention of one sequence in 32 bits -> o [Lq, H, d], lse [H, Lq]."""
    (lq, H, d), (lk, Hkv) = q.shape, k.shape[:2]
    if lk == 0:
        return torch.zeros_like(q), torch.full((H, lq), -math.inf, device=q.device)
    qg = q.float().view(lq, Hkv, H // Hkv, d).permute(1, 2, 0, 3).reshape(Hkv, -1, d)
    s = torch.matmul(qg / math.sqrt(d), k.float().permute(1, 2, 0).contiguous())
    s = s.view(Hkv, H // Hkv, lq, lk)
    if c["causal"]:
        i = torch.arange(lq, device=q.device)[:, None]
        j = torch.arange(lk, device=q.device)[None, :]
        s.masked_fill_(j > i + (lk - lq), -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    vg = v.float().permute(1, 0, 2).contiguous()
    o = torch.matmul(p.view(Hkv, -1, lk), vg).view(Hkv, H // Hkv, lq, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (m + total.log()).view(H, lq)
    return o.permute(2, 0, 1, 3).reshape(lq, H, d), lse


def run(state):
    st, c = state, state["case"]
    if own:
        from paper_2608_12032_amd import losa
        if c["op"] == "attn":
            got = losa.losa_packed_attn_fwd(st["q"], st["k"], st["v"], st["plan"],
                                            want_lse=c["lse"], out=st["out"],
                                            workspace=st["workspace"])
            return {"o": got[0], "lse": got[1]} if c["lse"] else {"o": got}
        n_pad = _tokens(c)[1]
        if c["op"] == "rope":
            return {"y": losa.losa_rope(st["x"][0], st["table"], st["pos"], n_pad=n_pad,
                                        pairing=c["pairing"], out=st["out"][0])}
        table, pos = (st["table"], st["pos"]) if c["rotate"] else (None, None)
        q, k, v = losa.losa_qk_norm_rope(
            *st["x"], norm=c["norm"], over=c["over"], q_weight=st["weight"][0],
            q_bias=st["bias"][0], k_weight=st["weight"][1], k_bias=st["bias"][1], eps=1e-6,
            table=table, pos=pos, pairing=c["pairing"], n_pad=n_pad, q_out=st["out"][0],
            k_out=st["out"][1], v_out=st["out"][2])
        return {"q": q, "k": k, "v": v}
    if c["op"] == "attn":
        parts = [_attend(c, *x) for x in zip(st["q"].split(st["q_lens"]),
                                             st["k"].split(st["k_lens"]),
                                             st["v"].split(st["k_lens"]))]
        out = {"o": torch.cat([o for o, _ in parts]).to(_type(c))}
        if c["lse"]:
            out["lse"] = torch.cat([lse for _, lse in parts], 1)
        return out
    if c["op"] == "rope":
        return {"y": _lay_out(c, _rotate(c, st["x"][0].float(), st["cos"], st["sin"]))}
    out = {"v": _lay_out(c, st["x"][2])}
    for name, x, w, b in zip("qk", st["x"], st["weight"], st["bias"]):
        y = _norm(c, x.float(), w, b)
        out[name] = _lay_out(c, _rotate(c, y, st["cos"], st["sin"]) if c["rotate"] else y)
    return out


def work(case):
    """Each input read once, each output written once; the products over the visible pairs."""
    c = case
    el = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "attn":
        q_lens, k_lens = _lens(c)
        pairs = 0
        for lq, lk in zip(q_lens, k_lens):
            if c["causal"]:  # row i sees lk - lq + 1 + i keys where that is above 0
                seen = min(lq, lk)
                pairs += seen * (lk - seen) + seen * (seen + 1) // 2
            else:
                pairs += lq * lk
        rows = 2 * sum(q_lens) * c["H"] + 2 * sum(k_lens) * c["Hkv"]
        return {"bytes": rows * c["d"] * el + (4 * sum(q_lens) * c["H"] if c["lse"] else 0),
                "flops": 4 * pairs * c["H"] * c["d"]}
    n, n_pad = _tokens(c)
    heads = c["H"] if c["op"] == "rope" else c["H"] + 2 * c["Hkv"]
    rotated = c["op"] == "rope" or c["rotate"]
    dims, lens = _axes(c)
    small = 4 * sum(a * b for a, b in zip(dims, lens)) + 4 * c["axes"] * n if rotated else 0
    flops = 3 * c["B"] * n * (heads if c["op"] == "rope" else c["H"] + c["Hkv"]) * c["d"]
    return {"bytes": c["B"] * heads * (n + n_pad) * c["d"] * el + small,
            "flops": flops if c["op"] == "rope" else 2 * flops}


def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    c, st = case, prepare(case, seed)
    if c["op"] == "attn":
        q_lens, k_lens = _lens(c)
        if sum(a * b for a, b in zip(q_lens, k_lens)) * c["H"] > 2e10:
            return None
        o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full((c["H"], sum(q_lens)), -math.inf, dtype=torch.float64, device="cuda")
        group, q0, k0 = c["H"] // c["Hkv"], 0, 0
        for lq, lk in zip(q_lens, k_lens):
            step = max(1, (1 << 28) // max(1, lk))
            for h in range(c["H"]):
                kh = st["k"][k0:k0 + lk, h // group].double()
                vh = st["v"][k0:k0 + lk, h // group].double()
                for i in range(0, lq if lk else 0, step):
                    e = min(lq, i + step)
                    s = st["q"][q0 + i:q0 + e, h].double() @ kh.t() * c["d"] ** -0.5
                    if c["causal"]:
                        s += torch.full_like(s, -math.inf).triu(i + lk - lq + 1)
                    total = torch.logsumexp(s, 1)
                    lse[h, q0 + i:q0 + e] = total
                    o[q0 + i:q0 + e, h] = torch.exp(s - total[:, None]).nan_to_num(0.0) @ vh
            q0, k0 = q0 + lq, k0 + lk
        return {"o": o, "lse": lse} if c["lse"] else {"o": o}

    n, n_pad = _tokens(c)
    turn = torch.polar(torch.ones_like(_angles(c)), _angles(c))
    turn[(_positions(c)[0] < 0)] = 1.0

    def rotated(x):
        r = c["rot"]
        y = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if c["pairing"] == "halves" \
            else x[..., :r].unflatten(-1, (r // 2, 2))
        y = torch.view_as_real(torch.view_as_complex(y.contiguous()) * turn[:, None, :])
        y = y.transpose(-1, -2) if c["pairing"] == "halves" else y
        return torch.cat([y.flatten(-2), x[..., r:]], -1)

    def padded(y):
        return torch.nn.functional.pad(y.transpose(1, 2), (0, 0, 0, n_pad - n))

    if c["op"] == "rope":
        return {"y": padded(rotated(st["x"][0].double()))}
    out = {"v": padded(st["x"][2].double())}
    for i, name in enumerate("qk"):
        x = st["x"][i].double()
        dims = (3,) if c["over"] == "head" else (2, 3)
        mean = x.mean(dims, keepdim=True) if c["norm"] == "layer" else 0.0
        var = ((x - mean) ** 2).mean(dims, keepdim=True)
        shape = (1, c["d"]) if c["over"] == "head" else x.shape[2:]
        y = (x - mean) / torch.sqrt(var + 1e-6) * st["weight"][i].double().view(shape)
        if st["bias"][i] is not None:
            y = y + st["bias"][i].double().view(shape)
        out[name] = padded(rotated(y) if c["rotate"] else y)
    return out
