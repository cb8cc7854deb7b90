"""Performance cases of the operators between a layer shard's GEMMs: the norms of a block with its gate and residual, the paged key / value
cache, and the attention of one new token over it.  Sizes are those of the layer shapes in perf/cases.py, from one token to a training batch.

A case is a dict of plain values; its "kind" names the operator:
  join     norm after a block, gate, scaled residual, norm before the next block: forward
  join_bwd its gradient
  append   rotation of the query and key heads, keys and values appended to the paged cache
  decode   attention of one new token per sequence over the paged cache

`run` computes them in elementary torch operations, or where `own` is true with the entry points of paper_2504_06095_amd.
"""
import math

import torch

own = False

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
EPS = 1.0e-5
THETA = 500000.0


def listed():
    return [
        # 16 sequences' new tokens between two blocks of a hidden-8192 layer: latency
        dict(name="join_token", kind="join", tokens=16, hidden=8192, norm="rms", post=False, pre=True, gate="none", residual="bf16", bias=False, a=1.0, b=1.0),
        # GPT-3-175B-shape layer, one 2048-token sequence: residual addition and the next layer norm
        dict(name="join_gpt3", kind="join", tokens=2048, hidden=12288, norm="layer", post=False, pre=True, gate="none", residual="bf16", bias=True, a=1.0, b=1.0),
        # 405B-shape hidden size, norms on both sides of the block, a gate per channel, scaled branch
        dict(name="join_405b", kind="join", tokens=8192, hidden=16384, norm="rms", post=True, pre=True, gate="channel", residual="bf16", bias=False, a=1.0, b=0.25),
        # gradient of join_gpt3
        dict(name="join_bwd_gpt3", kind="join_bwd", tokens=2048, hidden=12288, norm="layer", post=False, pre=True, gate="none", residual="bf16", bias=True, a=1.0, b=1.0),
        # hidden 6144, an odd number of tokens, both norms, gate per channel, residual stream kept in fp32
        dict(name="join_bwd_6144", kind="join_bwd", tokens=4099, hidden=6144, norm="rms", post=True, pre=True, gate="channel", residual="fp32", bias=False, a=1.0, b=0.5),
        # one new token of 64 sequences, three query heads over one KV head (TP 32 -> 30)
        dict(name="append_token", kind="append", tokens=64, q=3, kv=1, dim=128, rotary=128, pairs=False, page=16, longest=131072, prompt=False, padded=0),
        # a prompt batch of the GPT-3-175B-shape shard at TP 7, the rotated keys also kept for the core
        dict(name="append_prompt", kind="append", tokens=8192, q=14, kv=14, dim=128, rotary=128, pairs=False, page=64, longest=2048, prompt=True, padded=0),
        # heads of 64, half of a head rotated in neighbouring pairs, a ragged batch padded to its size
        dict(name="append_d64", kind="append", tokens=1021, q=11, kv=4, dim=64, rotary=32, pairs=True, page=32, longest=8192, prompt=True, padded=37),
        # one sequence, three query heads over one KV head: latency
        dict(name="decode_one", kind="decode", n_seq=1, longest=1021, ragged=False, q=3, kv=1, q_off=0, kv_off=0, group=8, dim=128, page=16),
        # a serving batch of the GPT-3-175B-shape shard at TP 7 (no grouped heads), lengths up to 8192
        dict(name="decode_batch", kind="decode", n_seq=64, longest=8192, ragged=True, q=14, kv=14, q_off=0, kv_off=0, group=1, dim=128, page=64),
        # two long sequences, two KV heads of 16 query heads each
        dict(name="decode_long", kind="decode", n_seq=2, longest=131072, ragged=False, q=32, kv=2, q_off=0, kv_off=0, group=16, dim=128, page=256),
        # 32 heads of 64 over 8 KV heads at TP 3, the middle rank: its first and last KV heads are read by a part of their group
        dict(name="decode_d64", kind="decode", n_seq=48, longest=4096, ragged=True, q=11, kv=4, q_off=11, kv_off=2, group=4, dim=64, page=32),
    ]


MAX_BYTES = 1.6e9  # a drawn case moves no more than this (join_405b moves 1.1e9, decode_batch about 1.9e9)


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw(rng, kind):
    if kind in ("join", "join_bwd"):
        post = rng.random() < 0.5
        return dict(kind=kind, tokens=max(1, round(_log(rng, 1, 16384))), hidden=8 * round(_log(rng, 512, 16384) / 8), norm=rng.choice(("rms", "layer")), post=post,
                    pre=rng.random() < 0.85 or not post, gate=rng.choice(("none", "channel", "channel", "token")), residual=rng.choice(("bf16", "bf16", "fp32")),
                    bias=rng.random() < 0.5, a=rng.choice((1.0, 1.0, 1.5)), b=rng.choice((1.0, 0.25, 0.5)))
    if kind == "append":
        dim = rng.choice((64, 128, 128))
        kv = rng.choice((1, 1, 2, 4, 8, 14))
        tokens = max(1, round(_log(rng, 1, 16384)))
        return dict(kind=kind, tokens=tokens, q=kv * rng.choice((1, 2, 4)) + rng.choice((0, 0, 1)), kv=kv, dim=dim, rotary=rng.choice((dim, dim, dim // 2, 0)),
                    pairs=rng.random() < 0.3, page=rng.choice((16, 32, 64, 256)), longest=round(_log(rng, 512, 131072)), prompt=rng.random() < 0.5,
                    padded=rng.choice((0, 0, tokens // 9)))
    group = rng.choice((1, 1, 2, 4, 8, 16))
    kv = rng.choice((1, 1, 2, 4, 8, 14))
    # some query heads of the first and of the last group may live on other ranks
    first, last = rng.randrange(group), rng.randrange(group)
    q = kv * group - first - last if kv > 1 else group - min(first, last)
    return dict(kind="decode", n_seq=max(1, round(_log(rng, 1, 256))), longest=max(1, round(_log(rng, 1, 131072))), ragged=rng.random() < 0.7, q=q, kv=kv,
                q_off=3 * group + (first if kv > 1 else min(first, last)), kv_off=3, group=group, dim=rng.choice((64, 128, 128)), page=rng.choice((16, 32, 64, 256)))


def draw(rng):
    kind = rng.choice(("join", "join_bwd", "append", "decode", "decode"))
    while True:
        case = _draw(rng, kind)
        if work(case)["bytes"] <= MAX_BYTES:
            return case


def _lengths(case, seed):
    """Tokens in the cache per sequence, the new one included."""
    if not case["ragged"]:
        return [case["longest"]] * case["n_seq"]
    import random
    rng = random.Random(1000003 * seed + case["longest"])
    return [case["longest"]] + [rng.randint(1, case["longest"]) for _ in range(case["n_seq"] - 1)]


def work(case):
    k = case["kind"]
    if k in ("join", "join_bwd"):
        n, rt = case["tokens"] * case["hidden"], 4 if case["residual"] == "fp32" else 2
        vec = 2 * case["hidden"] * (case["post"] * (1 + case["bias"]) + case["pre"] * (1 + case["bias"]) + (case["gate"] == "channel"))
        token_gate = 2 * n if case["gate"] == "token" else 0
        stats = 8 * case["tokens"] * (case["post"] + case["pre"])
        if k == "join":  # X, Z in, X' and Y out
            return dict(bytes=n * (2 * rt + 2 + (2 if case["pre"] else 0)) + token_gate + vec + stats, flops=16 * n)
        # dX', dY, X', Z in (Z where the norm behind the block or a gate needs it), dX, dZ out; fp32 gradients of the vectors
        need_z = case["post"] or case["gate"] != "none"
        return dict(bytes=n * (2 * rt + 2 + (2 + rt if case["pre"] else 0) + (2 if need_z else 0)) + 2 * token_gate + 3 * vec + stats, flops=30 * n)
    d = case["dim"]
    if k == "append":
        m = case["tokens"]
        out = case["q"] + (case["kv"] if case["prompt"] else 0)
        return dict(bytes=2 * m * d * (case["q"] + 2 * case["kv"] + out) + 2 * (m - case["padded"]) * d * 2 * case["kv"] + 12 * m, flops=3 * m * case["rotary"] * (case["q"] + case["kv"]))
    # the mean of the ragged lengths is just above half of the longest; each key and value of a KV head once
    keys = case["longest"] + (case["n_seq"] - 1) * (0.5 * (case["longest"] + 1) if case["ragged"] else case["longest"])
    return dict(bytes=4 * d * keys * case["kv"] + 4 * d * case["n_seq"] * case["q"] + 4 * keys / case["page"], flops=4 * d * keys * case["q"])


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, std=1.0, dtype=BF):
    return torch.randn(*shape, device="cuda", generator=g, dtype=F32).mul_(std).to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    s = _PREPARE[case["kind"]](case, seed, g)
    s["case"] = case
    if own:
        import paper_2504_06095_amd as N
        s["N"], s["handle"] = N, N.ntp_create()
        _PLAN[case["kind"]](N, s)
    return s


def _workspace(N, s, call):
    """The workspace that a serving or training loop gives its handle once."""
    n = N.ntp_workspace_bytes(call, s["shape"], handle=s["handle"])
    if n > 0:
        N.ntp_set_workspace(torch.empty(n, dtype=torch.uint8, device="cuda"), handle=s["handle"])


# ---- norms, gate and residual -------------------------------------------------------
def _vectors(case, g):
    h = case["hidden"]
    v = {}
    for at in ("post", "pre"):
        if case[at]:
            v[at + "_gamma"] = (1.0 + _randn(g, h, std=0.1, dtype=F32)).to(BF)
            if case["bias"]:
                v[at + "_beta"] = _randn(g, h, std=0.1)
    if case["gate"] == "channel":
        v["gate"] = (0.5 + _randn(g, h, std=0.2, dtype=F32)).to(BF)
    if case["gate"] == "token":
        v["gate"] = torch.sigmoid(_randn(g, case["tokens"], h, dtype=F32)).to(BF)
    return v


def _stream(case, g, std):
    """Rows of the residual stream: a few channels are far larger than the others."""
    x = torch.randn(case["tokens"], case["hidden"], device="cuda", generator=g, dtype=F32).mul_(std)
    x[:, :: max(1, case["hidden"] // 4)] *= 12.0
    return x.to(F32 if case["residual"] == "fp32" else BF)


def _prepare_join(case, seed, g):
    m, h = case["tokens"], case["hidden"]
    X = _stream(case, g, 2.0)
    s = dict(X=X, Z=_randn(g, m, h), **_vectors(case, g))
    s.update(Xout=torch.empty_like(X), Y=torch.empty(m, h, dtype=BF, device="cuda") if case["pre"] else None, Stats=torch.zeros(4, m, dtype=F32, device="cuda"))
    return s


def _row_stats(x, layer):
    x = x.to(F64)
    mean = x.mean(1) if layer else torch.zeros_like(x[:, 0])
    return mean, torch.rsqrt(((x - mean[:, None]) ** 2).mean(1) + EPS)


def _prepare_join_bwd(case, seed, g):
    m, h = case["tokens"], case["hidden"]
    Xout, Z = _stream(case, g, 2.0), _randn(g, m, h)
    s = dict(Xout=Xout, Z=Z, **_vectors(case, g))
    # what the forward call kept of its rows
    s["Stats"] = torch.zeros(4, m, dtype=F32, device="cuda")
    for at, t, i in (("post", Z, 0), ("pre", Xout, 2)):
        if case[at]:
            for lo in range(0, m, 1024):
                mean, rstd = _row_stats(t[lo:lo + 1024], case["norm"] == "layer")
                s["Stats"][i, lo:lo + 1024], s["Stats"][i + 1, lo:lo + 1024] = mean.to(F32), rstd.to(F32)
    s.update(dXout=_randn(g, m, h, std=1e-2, dtype=Xout.dtype), dY=_randn(g, m, h, std=1e-2) if case["pre"] else None)
    s.update(dX=torch.empty_like(Xout), dZ=torch.empty_like(Z))
    for n in ("post_gamma", "post_beta", "pre_gamma", "pre_beta"):
        if n in s:
            s["d_" + n] = torch.empty(h, dtype=F32, device="cuda")
    if "gate" in s:
        s["d_gate"] = torch.empty(h, dtype=F32, device="cuda") if case["gate"] == "channel" else torch.empty_like(s["gate"])
    return s


def _plan_join(N, s):
    c = s["case"]
    s["shape"] = N.block_norm_shape(c["tokens"], c["hidden"], norm=N.binding.NTP_NORM_LAYER if c["norm"] == "layer" else N.binding.NTP_NORM_RMS,
                                    gate={"none": N.binding.NTP_GATE_NONE, "channel": N.binding.NTP_GATE_CHANNEL, "token": N.binding.NTP_GATE_TOKEN}[c["gate"]],
                                    residual_fp32=c["residual"] == "fp32", eps=EPS, residual_scale=c["a"], branch_scale=c["b"])
    _workspace(N, s, N.binding.NTP_CALL_BLOCK_NORM)


def _f32(t):
    return None if t is None else t.to(F32)


def _norm32(x, layer, gamma, beta):
    """Normalised and scaled rows, and their mean and reciprocal deviation."""
    mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    y = c * rstd * gamma.to(F32)
    if beta is not None:
        y = y + beta.to(F32)
    return y, mean[:, 0], rstd[:, 0]


def _run_join(s):
    c = s["case"]
    get = s.get
    if own:
        s["N"].ntp_block_norm_fwd(s["shape"], s["X"], s["Z"], s["Xout"], s["Y"], s["Stats"], post_gamma=get("post_gamma"), post_beta=get("post_beta"), gate=get("gate"),
                                  pre_gamma=get("pre_gamma"), pre_beta=get("pre_beta"), handle=s["handle"])
        out = dict(Xout=s["Xout"], Stats=s["Stats"])
        return dict(out, Y=s["Y"]) if c["pre"] else out
    layer = c["norm"] == "layer"
    x, r = _f32(s["X"]), _f32(s["Z"])
    stats = torch.zeros_like(s["Stats"])
    if c["post"]:
        r, stats[0], stats[1] = _norm32(r, layer, s["post_gamma"], get("post_beta"))
    if c["gate"] != "none":
        r = r * _f32(s["gate"])
    x = c["a"] * x + c["b"] * r
    out = dict(Xout=x.to(s["X"].dtype), Stats=stats)
    if c["pre"]:
        y, stats[2], stats[3] = _norm32(x, layer, s["pre_gamma"], get("pre_beta"))
        out["Y"] = y.to(BF)
    return out


def _colsum(t):
    return t.sum(0, dtype=F64).to(F32)


def _run_join_bwd(s):
    c = s["case"]
    get = s.get
    if own:
        s["N"].ntp_block_norm_bwd(s["shape"], s["dXout"], s["dY"], s["Xout"], s["Z"], s["Stats"], s["dX"], s["dZ"], post_gamma=get("post_gamma"), post_beta=get("post_beta"),
                                  gate=get("gate"), pre_gamma=get("pre_gamma"), pre_beta=get("pre_beta"), d_post_gamma=get("d_post_gamma"), d_post_beta=get("d_post_beta"),
                                  d_gate=get("d_gate"), d_pre_gamma=get("d_pre_gamma"), d_pre_beta=get("d_pre_beta"), handle=s["handle"])
        return {k: s[k] for k in ("dX", "dZ", "d_post_gamma", "d_post_beta", "d_gate", "d_pre_gamma", "d_pre_beta") if k in s}
    layer = c["norm"] == "layer"
    G, st, out = _f32(s["dXout"]), s["Stats"], {}
    if c["pre"]:
        dy = _f32(s["dY"])
        xh = (_f32(s["Xout"]) - st[2][:, None]) * st[3][:, None]
        out["d_pre_gamma"] = _colsum(dy * xh)
        if c["bias"]:
            out["d_pre_beta"] = _colsum(dy)
        u = dy * _f32(s["pre_gamma"])
        d = u - xh * (u * xh).mean(1, keepdim=True)
        if layer:
            d = d - u.mean(1, keepdim=True)
        G = G + d * st[3][:, None]
    out["dX"] = (c["a"] * G).to(s["dX"].dtype)
    dr = c["b"] * G
    r = z = _f32(s["Z"])
    if c["post"]:
        z = (z - st[0][:, None]) * st[1][:, None]
        r = z * _f32(s["post_gamma"])
        if c["bias"]:
            r = r + _f32(s["post_beta"])
    if c["gate"] != "none":
        dg = dr * r
        out["d_gate"] = _colsum(dg) if c["gate"] == "channel" else dg.to(BF)
        dr = dr * _f32(s["gate"])
    if c["post"]:
        out["d_post_gamma"] = _colsum(dr * z)
        if c["bias"]:
            out["d_post_beta"] = _colsum(dr)
        v = dr * _f32(s["post_gamma"])
        d = v - z * (v * z).mean(1, keepdim=True)
        if layer:
            d = d - v.mean(1, keepdim=True)
        dr = d * st[1][:, None]
    out["dZ"] = dr.to(BF)
    return {k: out[k] for k in ("dX", "dZ", "d_post_gamma", "d_post_beta", "d_gate", "d_pre_gamma", "d_pre_beta") if k in out}


# ---- paged cache ----------------------------------------------------------------------
def _inv_freq(rotary):
    return torch.tensor([THETA ** (-2.0 * i / rotary) for i in range(rotary // 2)], dtype=F64, device="cuda") if rotary else None


def _prepare_append(case, seed, g):
    import random
    m, q, kv, d, page = (case[k] for k in ("tokens", "q", "kv", "dim", "page"))
    rng = random.Random(7919 * seed + m)
    rows = m - case["padded"]
    if case["prompt"]:  # consecutive positions of a few prompts, each into pages of its own
        pos, slots, at = [], [], 0
        while len(pos) < rows:
            n = min(case["longest"], rows - len(pos), rng.randint(1, case["longest"]) if pos else case["longest"])
            pos += range(n)
            slots += range(at * page, at * page + n)
            at += (n + page - 1) // page
        n_pages = at
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
        slot = torch.tensor(slots, dtype=torch.int64)
        slot = order[slot // page] * page + slot % page
    else:  # one new token of every sequence, each in a page of its own
        pos = [rng.randrange(case["longest"]) for _ in range(rows)]
        n_pages = rows
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
        slot = order * page + torch.tensor(pos, dtype=torch.int64) % page
    pad = [0] * case["padded"]
    s = dict(QKV=_randn(g, m, (q + 2 * kv) * d), positions=torch.tensor(pos + pad, dtype=torch.int32).cuda(),
             slots=torch.cat([slot, torch.full((len(pad),), -1, dtype=torch.int64)]).cuda(), inv_freq=_inv_freq(case["rotary"]))
    s["K"], s["V"] = torch.zeros(n_pages, kv, page, d, dtype=BF, device="cuda"), torch.zeros(n_pages, kv, page, d, dtype=BF, device="cuda")
    s["Qout"] = torch.empty(m, q * d, dtype=BF, device="cuda")
    s["Kout"] = torch.empty(m, kv * d, dtype=BF, device="cuda") if case["prompt"] else None
    return s


def _plan_append(N, s):
    c = s["case"]
    s["shape"] = N.kv_append_shape(c["tokens"], dict(q_cnt=c["q"], kv_cnt=c["kv"], head_dim=c["dim"]), rotary_dim=c["rotary"], interleaved=c["pairs"])
    s["cache"] = N.kv_cache(s["K"], s["V"])


def _run_append(s):
    c = s["case"]
    m, q, kv, d, page, rd = (c[k] for k in ("tokens", "q", "kv", "dim", "page", "rotary"))
    if own:
        s["N"].ntp_kv_append_shard(s["shape"], s["cache"], s["QKV"], s["positions"], s["slots"], s["inv_freq"], s["Qout"], s["Kout"], handle=s["handle"])
        out = dict(Q=s["Qout"], K=s["K"], V=s["V"])
        return dict(out, Kout=s["Kout"]) if c["prompt"] else out
    x = s["QKV"].view(m, q + 2 * kv, d)
    rot = x[:, :q + kv].to(F32)
    if rd:
        angle = s["positions"].to(F64)[:, None] * s["inv_freq"]
        cs, sn = angle.cos().to(F32)[:, None], angle.sin().to(F32)[:, None]
        a, b = (rot[..., 0:rd:2], rot[..., 1:rd:2]) if c["pairs"] else (rot[..., :rd // 2], rot[..., rd // 2:rd])
        ra, rb = a * cs - b * sn, b * cs + a * sn
        both = torch.stack((ra, rb), -1).flatten(-2) if c["pairs"] else torch.cat((ra, rb), -1)
        rot = torch.cat((both, rot[..., rd:]), -1)
    rot = rot.to(BF)
    rows = torch.nonzero(s["slots"] >= 0)[:, 0]
    slot = s["slots"][rows]
    s["K"][slot // page, :, slot % page] = rot[rows, q:]
    s["V"][slot // page, :, slot % page] = x[rows, q + kv:]
    out = dict(Q=rot[:, :q].reshape(m, q * d), K=s["K"], V=s["V"])
    return dict(out, Kout=rot[:, q:].reshape(m, kv * d)) if c["prompt"] else out


# ---- attention of one new token ---------------------------------------------------------
def _prepare_decode(case, seed, g):
    n, q, kv, d, page = (case[k] for k in ("n_seq", "q", "kv", "dim", "page"))
    lengths = _lengths(case, seed)
    need = [(x + page - 1) // page for x in lengths]
    n_pages, cols = sum(need) + 3, max(need)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table, at = torch.zeros(n, cols, dtype=torch.int32), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    s = dict(lengths=torch.tensor(lengths, dtype=torch.int32).cuda(), table=table.cuda(), host_lengths=lengths)
    s["Q"] = _randn(g, n, q * d, std=1.5)
    s["K"], s["V"] = (torch.empty(n_pages, kv, page, d, dtype=BF, device="cuda").normal_(generator=g) for _ in range(2))
    s["C"], s["LSE"] = torch.empty(n, q * d, dtype=BF, device="cuda"), torch.empty(q, n, dtype=F32, device="cuda")
    return s


def _plan_decode(N, s):
    c = s["case"]
    plan = dict(q_cnt=c["q"], kv_cnt=c["kv"], q_off=c["q_off"], kv_off=c["kv_off"], head_dim=c["dim"])
    s["shape"] = N.attn_decode_shape(c["n_seq"], c["longest"], plan, c["group"])
    s["cache"] = N.kv_cache(s["K"], s["V"])
    _workspace(N, s, N.binding.NTP_CALL_ATTN_DECODE_SHARD)


def _kv_of(c):
    return [(c["q_off"] + j) // c["group"] - c["kv_off"] for j in range(c["q"])]


def _run_decode(s):
    c = s["case"]
    if own:
        s["N"].ntp_attn_decode_shard(s["shape"], s["cache"], s["Q"], s["table"], s["lengths"], s["C"], s["LSE"], handle=s["handle"])
        return dict(C=s["C"], LSE=s["LSE"])
    n, q, kv, d, page = (c[k] for k in ("n_seq", "q", "kv", "dim", "page"))
    C, LSE = torch.empty(n, q, d, dtype=BF, device="cuda"), torch.empty(q, n, dtype=F32, device="cuda")
    heads = _kv_of(c)
    for i, length in enumerate(s["host_lengths"]):
        pages = s["table"][i, :(length + page - 1) // page].long()
        k, v = (t[pages].transpose(0, 1).reshape(kv, -1, d)[:, :length].to(F32) for t in (s["K"], s["V"]))
        x = s["Q"][i].view(q, d).to(F32)
        for g in sorted(set(heads)):
            lo, hi = heads.index(g), len(heads) - heads[::-1].index(g)
            score = (x[lo:hi] @ k[g].t()) * (1.0 / math.sqrt(d))
            top = score.max(1, keepdim=True).values
            p = torch.exp(score - top)
            total = p.sum(1, keepdim=True)
            C[i, lo:hi] = ((p @ v[g]) / total).to(BF)
            LSE[lo:hi, i] = (top + torch.log(total))[:, 0]
    return dict(C=C.view(n, q * d), LSE=LSE)


def run(state):
    return _RUN[state["case"]["kind"]](state)


# ---- the definitions in 64 bits -----------------------------------------------------------
def exact(case, seed):
    return _EXACT[case["kind"]](case, _PREPARE[case["kind"]](case, seed, _gen(seed)))


def _blocks(m, h):
    step = max(1, (1 << 24) // h)
    return [slice(lo, min(m, lo + step)) for lo in range(0, m, step)]


def _d(t, rows=None):
    return t.double() if rows is None else t[rows].double()


def _exact_join(c, s):
    m, h = c["tokens"], c["hidden"]
    xo, y, st = torch.empty(m, h, dtype=F64, device="cuda"), torch.empty(m, h, dtype=F64, device="cuda"), torch.zeros(4, m, dtype=F64, device="cuda")

    def normed(t, at, i, rows):
        mu = t.sum(1) / h if c["norm"] == "layer" else torch.zeros(t.shape[0], dtype=F64, device="cuda")
        dev = t - mu.unsqueeze(1)
        rs = 1.0 / torch.sqrt((dev ** 2).sum(1) / h + EPS)
        st[i, rows], st[i + 1, rows] = mu, rs
        w = dev * rs.unsqueeze(1) * _d(s[at + "_gamma"])
        return w + _d(s[at + "_beta"]) if c["bias"] else w

    for rows in _blocks(m, h):
        branch = _d(s["Z"], rows)
        if c["post"]:
            branch = normed(branch, "post", 0, rows)
        if c["gate"] == "channel":
            branch = branch * _d(s["gate"])
        elif c["gate"] == "token":
            branch = branch * _d(s["gate"], rows)
        xo[rows] = c["a"] * _d(s["X"], rows) + c["b"] * branch
        if c["pre"]:
            y[rows] = normed(xo[rows], "pre", 2, rows)
    out = dict(Xout=xo, Stats=st)
    return dict(out, Y=y) if c["pre"] else out


def _exact_join_bwd(c, s):
    m, h = c["tokens"], c["hidden"]
    out = dict(dX=torch.empty(m, h, dtype=F64, device="cuda"), dZ=torch.empty(m, h, dtype=F64, device="cuda"))
    for n in ("post_gamma", "post_beta", "gate", "pre_gamma", "pre_beta"):
        if n in s:
            out["d_" + n] = torch.zeros(s[n].shape, dtype=F64, device="cuda")
    st = s["Stats"].double()

    def through(up, hat, rs):  # gradient of a normalised row, up = gradient of the normalised values
        lost = hat * ((up * hat).sum(1, keepdim=True) / h)
        if c["norm"] == "layer":
            lost = lost + up.sum(1, keepdim=True) / h
        return (up - lost) * rs.unsqueeze(1)

    for rows in _blocks(m, h):
        grad = _d(s["dXout"], rows)
        if c["pre"]:
            dy = _d(s["dY"], rows)
            hat = (_d(s["Xout"], rows) - st[2, rows].unsqueeze(1)) * st[3, rows].unsqueeze(1)
            out["d_pre_gamma"] += (dy * hat).sum(0)
            if c["bias"]:
                out["d_pre_beta"] += dy.sum(0)
            grad = grad + through(dy * _d(s["pre_gamma"]), hat, st[3, rows])
        out["dX"][rows] = c["a"] * grad
        branch = value = _d(s["Z"], rows)
        if c["post"]:
            branch = (branch - st[0, rows].unsqueeze(1)) * st[1, rows].unsqueeze(1)
            value = branch * _d(s["post_gamma"]) + (_d(s["post_beta"]) if c["bias"] else 0.0)
        grad = grad * c["b"]
        if c["gate"] == "channel":
            out["d_gate"] += (grad * value).sum(0)
            grad = grad * _d(s["gate"])
        elif c["gate"] == "token":
            out["d_gate"][rows] = grad * value
            grad = grad * _d(s["gate"], rows)
        if c["post"]:
            out["d_post_gamma"] += (grad * branch).sum(0)
            if c["bias"]:
                out["d_post_beta"] += grad.sum(0)
            grad = through(grad * _d(s["post_gamma"]), branch, st[1, rows])
        out["dZ"][rows] = grad
    return {k: out[k] for k in ("dX", "dZ", "d_post_gamma", "d_post_beta", "d_gate", "d_pre_gamma", "d_pre_beta") if k in out}


def _exact_append(c, s):
    m, q, kv, d, page, rd = (c[k] for k in ("tokens", "q", "kv", "dim", "page", "rotary"))
    x = s["QKV"].double().view(m, q + 2 * kv, d).clone()
    if rd:
        z = torch.polar(torch.ones(m, rd // 2, dtype=F64, device="cuda"), s["positions"].double().unsqueeze(1) * s["inv_freq"].unsqueeze(0)).unsqueeze(1)
        even, odd = (slice(0, rd, 2), slice(1, rd, 2)) if c["pairs"] else (slice(0, rd // 2), slice(rd // 2, rd))
        w = torch.complex(x[:, :q + kv, even], x[:, :q + kv, odd]) * z
        x[:, :q + kv, even], x[:, :q + kv, odd] = w.real, w.imag
    K, V = s["K"].double(), s["V"].double()
    for t, first in ((K, q), (V, q + kv)):
        flat = t.transpose(1, 2).reshape(-1, kv, d).clone()
        keep = s["slots"] >= 0
        flat[s["slots"][keep]] = x[keep, first:first + kv]
        t.copy_(flat.view(-1, page, kv, d).transpose(1, 2))
    out = dict(Q=x[:, :q].reshape(m, q * d), K=K, V=V)
    return dict(out, Kout=x[:, q:q + kv].reshape(m, kv * d)) if c["prompt"] else out


def _exact_decode(c, s):
    n, q, kv, d, page = (c[k] for k in ("n_seq", "q", "kv", "dim", "page"))
    C, LSE = torch.zeros(n, q, d, dtype=F64, device="cuda"), torch.zeros(q, n, dtype=F64, device="cuda")
    for i in range(n):
        length = s["host_lengths"][i]
        at = torch.arange(length, device="cuda")
        page_of, row_of = s["table"][i].long()[at // page], at % page
        for g in range(kv):
            mine = [j for j in range(q) if (c["q_off"] + j) // c["group"] == c["kv_off"] + g]
            if not mine:
                continue
            k, v = s["K"][page_of, g, row_of].double(), s["V"][page_of, g, row_of].double()
            x = s["Q"][i].double().view(q, d)[mine]
            score = (x @ k.t()) / math.sqrt(d)
            LSE[mine, i] = torch.logsumexp(score, 1)
            C[i, mine] = torch.softmax(score, 1) @ v
    return dict(C=C.view(n, q * d), LSE=LSE)


_PREPARE = dict(join=_prepare_join, join_bwd=_prepare_join_bwd, append=_prepare_append, decode=_prepare_decode)
_PLAN = dict(join=_plan_join, join_bwd=_plan_join, append=_plan_append, decode=_plan_decode)
_RUN = dict(join=_run_join, join_bwd=_run_join_bwd, append=_run_append, decode=_run_decode)
_EXACT = dict(join=_exact_join, join_bwd=_exact_join_bwd, append=_exact_append, decode=_exact_decode)
