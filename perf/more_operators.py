"""Performance cases of serving a layer shard from its paged cache, past one bf16 token at a time: the norms of query and key heads with the
rotation in the same pass (forward with the append, and backward), the cache held in 8 bits, and the attention of chunks of new tokens over either cache.
Sizes are those of the layer shapes in perf/cases.py, from one token to a prompt batch.

A case is a dict of plain values; its "kind" names the operator:
  norm_append  norm of every query and key head, rotation, keys and values appended to the paged cache (bf16, or e4m3 with a power of two per token and head)
  norm_bwd     gradient of the norms and the rotation: of the projections' output and of the norms' weights
  chunk        attention of each sequence's new tokens (one to thousands) over its pages

`run` computes them in elementary torch operations, or where `own` is true with the entry points of paper_2504_06095_amd.
"""
import math
import random

import torch

own = False

BF, F32, F64, E4M3, U8 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn, torch.uint8
EPS = 1.0e-6
THETA = 500000.0


def listed():
    return [
        # one new token of 64 sequences, three query heads over one KV head (TP 32 -> 30), 8-bit cache: latency
        dict(name="norm_append8_token", kind="norm_append", tokens=64, q=3, kv=1, dim=128, rotary=128, pairs=False, page=16, bits=8, longest=131072, prompt=False, padded=0),
        # a prompt batch of the GPT-3-175B-shape shard at TP 7 into an 8-bit cache
        dict(name="norm_append8_prompt", kind="norm_append", tokens=8192, q=14, kv=14, dim=128, rotary=128, pairs=False, page=64, bits=8, longest=2048, prompt=True, padded=0),
        # heads of 64, half of a head rotated in neighbouring pairs, a ragged batch padded to its size, bf16 cache
        dict(name="norm_append_d64", kind="norm_append", tokens=1021, q=11, kv=4, dim=64, rotary=32, pairs=True, page=32, bits=16, longest=8192, prompt=True, padded=37),
        # training, GPT-3-175B-shape shard at TP 7, one 2048-token sequence
        dict(name="norm_bwd_gpt3", kind="norm_bwd", tokens=2048, q=14, kv=14, dim=128, rotary=128, pairs=False, longest=2048),
        # training, 405B-shape shard at TP 7 (19 query heads that read two KV heads), an odd number of tokens
        dict(name="norm_bwd_405b", kind="norm_bwd", tokens=8191, q=19, kv=2, dim=128, rotary=128, pairs=False, longest=8191),
        # one new token of one sequence over the 8-bit cache: latency
        dict(name="one_token8", kind="chunk", bits=8, n_seq=1, new=1, context=1020, ragged=False, ones=0, short=False, q=3, kv=1, q_off=0, kv_off=0, group=8, dim=128, page=16, padded=0),
        # a serving batch's new tokens over the 8-bit cache, GPT-3-175B-shape shard at TP 7, lengths up to 8192
        dict(name="batch8", kind="chunk", bits=8, n_seq=64, new=1, context=8191, ragged=True, ones=0, short=False, q=14, kv=14, q_off=0, kv_off=0, group=1, dim=128, page=64, padded=0),
        # four proposed tokens of 32 sequences checked at once, eight query heads over one KV head
        dict(name="verify", kind="chunk", bits=16, n_seq=32, new=4, context=4096, ragged=True, ones=0, short=False, q=8, kv=1, q_off=8, kv_off=1, group=8, dim=128, page=16, padded=0),
        # packed prompts of different lengths with nothing before them, padded to the batch's rows, GPT-3-175B-shape shard at TP 7
        dict(name="prompts", kind="chunk", bits=16, n_seq=8, new=2048, context=0, ragged=True, ones=0, short=False, q=14, kv=14, q_off=0, kv_off=0, group=1, dim=128, page=64, padded=37),
        # the last chunk of a long prompt, 16 query heads over one KV head, 8-bit cache
        dict(name="long8", kind="chunk", bits=8, n_seq=1, new=512, context=130560, ragged=False, ones=0, short=False, q=16, kv=1, q_off=0, kv_off=0, group=16, dim=128, page=256, padded=0),
        # one prompt's chunk beside the new tokens of 32 other sequences, 8-bit cache
        dict(name="mixed8", kind="chunk", bits=8, n_seq=33, new=2048, context=16384, ragged=True, ones=32, short=False, q=16, kv=2, q_off=0, kv_off=0, group=8, dim=128, page=64, padded=0),
        # 32 heads of 64 over 8 KV heads at TP 3, the middle rank: its first and last KV heads are read by a part of their group
        dict(name="chunks_d64", kind="chunk", bits=16, n_seq=5, new=777, context=3001, ragged=True, ones=1, short=True, q=11, kv=4, q_off=11, kv_off=2, group=4, dim=64, page=32, padded=5),
    ]


MAX_BYTES, MAX_FLOPS = 1.0e9, 5.0e11  # a drawn case costs no more than this (batch8 reads 0.95e9 bytes, long8 takes 5.5e11 operations)


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw(rng, kind):
    if kind != "chunk":
        dim, kv = rng.choice((64, 128, 128)), rng.choice((1, 1, 2, 4, 8, 14))
        case = dict(kind=kind, tokens=_log(rng, 1, 16384), q=kv * rng.choice((1, 2, 4)) + rng.choice((0, 0, 1)), kv=kv, dim=dim, rotary=rng.choice((dim, dim, dim // 2, 0)),
                    pairs=rng.random() < 0.3, longest=_log(rng, 512, 131072))
        if kind == "norm_append":
            case.update(page=rng.choice((16, 32, 64, 256)), bits=rng.choice((8, 8, 16)), prompt=rng.random() < 0.5, padded=rng.choice((0, 0, case["tokens"] // 9)))
        return case
    group, kv = rng.choice((1, 1, 2, 4, 8, 16)), rng.choice((1, 1, 2, 4, 8, 14))
    # some query heads of the first and of the last group may live on other ranks
    first, last = rng.randrange(group), rng.randrange(group)
    q = kv * group - first - last if kv > 1 else group - min(first, last)
    new = rng.choice((1, 1, _log(rng, 2, 16), _log(rng, 16, 4096), _log(rng, 16, 4096)))
    n_seq = _log(rng, 1, 128)
    return dict(kind=kind, bits=rng.choice((8, 16)), n_seq=n_seq, new=new, context=rng.choice((0, _log(rng, 1, 65536), _log(rng, 1, 65536))), ragged=rng.random() < 0.7,
                ones=rng.choice((0, 0, n_seq // 2)), short=rng.random() < 0.15, q=q, kv=kv, q_off=3 * group + (first if kv > 1 else min(first, last)), kv_off=3, group=group,
                dim=rng.choice((64, 128, 128)), page=rng.choice((16, 32, 64, 256)), padded=rng.choice((0, 0, 7)))


def draw(rng):
    kind = rng.choice(("norm_append", "norm_bwd", "chunk", "chunk", "chunk"))
    while True:
        case = _draw(rng, kind)
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
            return case


def _batch(case, seed):
    """New tokens of every sequence, the case's own, and its tokens in the cache (the new ones included)."""
    rng, own_rng = random.Random(1000003 * seed + case["context"]), random.Random(8191 * case["new"] + case["n_seq"])
    news, lens = [], []
    for i in range(case["n_seq"]):
        first = i == 0 or not case["ragged"]
        n = 1 if i >= case["n_seq"] - case["ones"] and i > 0 else case["new"] if first else own_rng.randint((case["new"] + 3) // 4, case["new"])
        news.append(n)
        lens.append(n + (case["context"] if first else rng.randint(0, case["context"])))
    if case["short"]:  # a sequence that was cut: its first rows have nothing to look at
        lens[-1] = news[-1] // 2
    return news, lens


def work(case):
    d, q, kv = case["dim"], case["q"], case["kv"]
    if case["kind"] == "norm_append":
        m, b = case["tokens"], case["bits"] // 8
        cache = (m - case["padded"]) * 2 * kv * (d * b + (b == 1))
        return dict(bytes=2 * m * d * (2 * q + 2 * kv + (kv if case["prompt"] else 0)) + cache + 12 * m, flops=m * (q + kv) * (6 * d + 3 * case["rotary"]))
    if case["kind"] == "norm_bwd":  # the projections' query and key columns, their gradients in and out
        m = case["tokens"]
        return dict(bytes=2 * m * d * 3 * (q + kv) + 4 * m + 12 * d, flops=m * (q + kv) * (14 * d + 3 * case["rotary"]))
    news, lens = _batch(case, 0)
    per_key = 2 * kv * (2 * d if case["bits"] == 16 else d + 1) + 4 / case["page"]
    pairs = sum(sum(max(0, x - n + i + 1) for i in range(n)) for n, x in zip(news, lens))
    return dict(bytes=per_key * sum(lens) + 4 * d * q * sum(news) + 4 * q * sum(news), flops=4 * d * q * pairs)


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
        N.ntp_set_workspace(torch.empty(n, dtype=U8, device="cuda"), handle=s["handle"])


# ---- the cache in 8 bits: e4m3 values and the power of two that they are multiplied by, one for each token and head ----
def _exponents(x):
    """The smallest e with |x| <= 448 * 2^e for every value of a head (the last axis), as int32, at least -111; 0 for zeros."""
    top = x.abs().amax(-1)
    part, e = torch.frexp(top)  # top = part * 2^e, 0.5 <= part < 1; 448 = 0.875 * 2^9
    e = e - 9 + (part > 0.875).to(torch.int32)
    return torch.where(top == 0, torch.zeros_like(e), e.clamp(min=-111))


def _two_to(e):
    """Powers of two in fp32 of int32 exponents -126 .. 127."""
    return ((e + 127) << 23).view(F32)


def _to_8_bits(x):
    """e4m3 values and exponent bytes (127 more than the exponent) of fp32 heads."""
    e = _exponents(x)
    return (x * _two_to(-e)[..., None]).to(E4M3), (e + 127).to(U8)


# ---- norms of query and key heads, rotation, append -----------------------------------------------------------
def _inv_freq(rotary):
    return torch.tensor([THETA ** (-2.0 * i / rotary) for i in range(rotary // 2)], dtype=F64, device="cuda") if rotary else None


def _projections(case, g):
    """Heads of the projections' output: sizes differ by head, a few channels are far larger than the others."""
    m, n, d = case["tokens"], case["q"] + 2 * case["kv"], case["dim"]
    x = torch.randn(m, n, d, device="cuda", generator=g, dtype=F32)
    x *= torch.exp(0.5 * torch.randn(1, n, 1, device="cuda", generator=g, dtype=F32))
    x[:, :, 5::d // 2] *= 6.0
    return x.to(BF).view(m, n * d)


def _gammas(case, g):
    return {k: (1.0 + _randn(g, case["dim"], std=0.2, dtype=F32)).to(BF) for k in ("q_gamma", "k_gamma")}


def _prepare_append(case, seed, g):
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
        n_pages = max(1, at)
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
        slot = torch.tensor(slots, dtype=torch.int64)
        slot = order[slot // page] * page + slot % page
    else:  # one new token of every sequence, each in a page of its own
        pos = [rng.randrange(case["longest"]) for _ in range(rows)]
        n_pages = max(1, rows)
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
        slot = order[:rows] * page + torch.tensor(pos, dtype=torch.int64) % page
    pad = [0] * case["padded"]
    s = dict(QKV=_projections(case, g), positions=torch.tensor(pos + pad, dtype=torch.int32).cuda(),
             slots=torch.cat([slot, torch.full((len(pad),), -1, dtype=torch.int64)]).cuda(), inv_freq=_inv_freq(case["rotary"]), **_gammas(case, g))
    for n in ("K", "V"):
        if case["bits"] == 16:
            s[n] = torch.zeros(n_pages, kv, page, d, dtype=BF, device="cuda")
        else:
            s[n] = torch.zeros(n_pages, kv, page, d, dtype=U8, device="cuda").view(E4M3)
            s[n + "_exp"] = torch.full((n_pages, kv, page), 127, dtype=U8, device="cuda").view(torch.float8_e8m0fnu)
    s["Qout"] = torch.empty(m, q * d, dtype=BF, device="cuda")
    s["Kout"] = torch.empty(m, kv * d, dtype=BF, device="cuda") if case["prompt"] else None
    return s


def _plan_append(N, s):
    c = s["case"]
    s["shape"] = N.kv_append_shape(c["tokens"], dict(q_cnt=c["q"], kv_cnt=c["kv"], head_dim=c["dim"]), rotary_dim=c["rotary"], interleaved=c["pairs"])
    s["norm"] = N.qk_norm(s["q_gamma"], s["k_gamma"], eps=EPS)
    s["pages"] = N.kv_pages(s["K"], s["V"], s.get("K_exp"), s.get("V_exp"))


def _halves(c, t):
    rd = c["rotary"]
    return (t[..., 0:rd:2], t[..., 1:rd:2]) if c["pairs"] else (t[..., :rd // 2], t[..., rd // 2:rd])


def _turned(c, t, positions, inv_freq, sign):
    """fp32 heads [M, heads, d] rotated to their positions (sign 1) or back (-1)."""
    if not c["rotary"]:
        return t
    angle = positions.to(F64)[:, None] * inv_freq
    cs, sn = angle.cos().to(F32)[:, None], sign * angle.sin().to(F32)[:, None]
    a, b = _halves(c, t)
    ra, rb = a * cs - b * sn, b * cs + a * sn
    both = torch.stack((ra, rb), -1).flatten(-2) if c["pairs"] else torch.cat((ra, rb), -1)
    return torch.cat((both, t[..., c["rotary"]:]), -1)


def _weights(c, s):
    """The norms' weights by head: [q + kv, d]."""
    return torch.cat((s["q_gamma"].to(F32).expand(c["q"], -1), s["k_gamma"].to(F32).expand(c["kv"], -1)))


def _run_append(s):
    c = s["case"]
    m, q, kv, d, page = (c[k] for k in ("tokens", "q", "kv", "dim", "page"))
    names = ("K", "V") if c["bits"] == 16 else ("K", "K_exp", "V", "V_exp")
    if own:
        s["N"].ntp_qk_norm_append_shard(s["shape"], s["norm"], s["pages"], s["QKV"], s["positions"], s["slots"], s["inv_freq"], s["Qout"], s["Kout"], handle=s["handle"])
        out = dict(Q=s["Qout"], **{k: s[k] for k in names})
        return dict(out, Kout=s["Kout"]) if c["prompt"] else out
    x = s["QKV"].view(m, q + 2 * kv, d)
    h = x[:, :q + kv].to(F32)
    h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * _weights(c, s)
    h = _turned(c, h, s["positions"], s["inv_freq"], 1.0)
    rows = torch.nonzero(s["slots"] >= 0)[:, 0]
    slot = s["slots"][rows]
    for n, t in (("K", h[rows, q:]), ("V", x[rows, q + kv:])):
        if c["bits"] == 16:
            s[n][slot // page, :, slot % page] = t.to(BF)
        else:
            values, exps = _to_8_bits(t.to(F32))
            s[n].view(U8)[slot // page, :, slot % page] = values.view(U8)
            s[n + "_exp"].view(U8)[slot // page, :, slot % page] = exps
    h = h.to(BF)
    out = dict(Q=h[:, :q].reshape(m, q * d), **{k: s[k] for k in names})
    return dict(out, Kout=h[:, q:].reshape(m, kv * d)) if c["prompt"] else out


# ---- gradient of the norms and the rotation --------------------------------------------------------------------
def _prepare_bwd(case, seed, g):
    m, q, kv, d = (case[k] for k in ("tokens", "q", "kv", "dim"))
    s = dict(QKV=_projections(case, g), positions=(torch.arange(m, dtype=torch.int32) % case["longest"]).cuda(), inv_freq=_inv_freq(case["rotary"]), **_gammas(case, g))
    s.update(dQ=_randn(g, m, q * d, std=1e-2), dK=_randn(g, m, kv * d, std=1e-2))
    # the value columns of the gradient are the attention's already
    s["dQKV"] = _randn(g, m, (q + 2 * kv) * d, std=1e-2)
    s.update(d_q_gamma=torch.empty(d, dtype=F32, device="cuda"), d_k_gamma=torch.empty(d, dtype=F32, device="cuda"))
    return s


def _plan_bwd(N, s):
    c = s["case"]
    s["shape"] = N.kv_append_shape(c["tokens"], dict(q_cnt=c["q"], kv_cnt=c["kv"], head_dim=c["dim"]), rotary_dim=c["rotary"], interleaved=c["pairs"])
    s["norm"] = N.qk_norm(s["q_gamma"], s["k_gamma"], eps=EPS)
    _workspace(N, s, N.binding.NTP_CALL_QK_NORM)


def _run_bwd(s):
    c = s["case"]
    m, q, kv, d = (c[k] for k in ("tokens", "q", "kv", "dim"))
    if own:
        s["N"].ntp_qk_norm_shard_bwd(s["shape"], s["norm"], s["QKV"], s["dQ"], s["dK"], s["positions"], s["inv_freq"], s["dQKV"], s["d_q_gamma"], s["d_k_gamma"], handle=s["handle"])
        return {k: s[k] for k in ("dQKV", "d_q_gamma", "d_k_gamma")}
    x = s["QKV"].view(m, q + 2 * kv, d)[:, :q + kv].to(F32)
    up = torch.cat((s["dQ"].view(m, q, d), s["dK"].view(m, kv, d)), 1).to(F32)
    up = _turned(c, up, s["positions"], s["inv_freq"], -1.0)
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    hat = x * rstd
    parts = up * hat
    dq, dk = (t.sum((0, 1), dtype=F64).to(F32) for t in (parts[:, :q], parts[:, q:]))
    w = up * _weights(c, s)
    dx = (w - hat * (w * hat).mean(-1, keepdim=True)) * rstd
    out = s["dQKV"].clone()
    out[:, :(q + kv) * d] = dx.to(BF).view(m, -1)
    return dict(dQKV=out, d_q_gamma=dq, d_k_gamma=dk)


# ---- attention of chunks of new tokens over the pages ------------------------------------------------------------
def _cache(case, g, n_pages):
    """Keys and values whose size differs by token and head."""
    kv, d, page = case["kv"], case["dim"], case["page"]
    out = {}
    for n in ("K", "V"):
        t = torch.empty(n_pages, kv, page, d, dtype=BF if case["bits"] == 16 else U8, device="cuda")
        e = torch.empty(n_pages, kv, page, dtype=U8, device="cuda")
        step = max(1, (1 << 26) // (kv * page * d))
        for lo in range(0, n_pages, step):
            x = torch.randn(min(step, n_pages - lo), kv, page, d, device="cuda", generator=g, dtype=F32)
            x *= torch.exp(0.2 * torch.randn(*x.shape[:3], 1, device="cuda", generator=g, dtype=F32))
            if case["bits"] == 16:
                t[lo:lo + step] = x.to(BF)
            else:
                values, e[lo:lo + step] = _to_8_bits(x)
                t[lo:lo + step] = values.view(U8)
        out[n] = t if case["bits"] == 16 else t.view(E4M3)
        if case["bits"] == 8:
            out[n + "_exp"] = e.view(torch.float8_e8m0fnu)
    return out


def _prepare_chunk(case, seed, g):
    q, d, page = case["q"], case["dim"], case["page"]
    news, lens = _batch(case, seed)
    need = [(x + page - 1) // page for x in lens]
    most = case["context"] + case["new"]
    n_pages, cols = sum(need) + 3, (most + page - 1) // page
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table, at = torch.zeros(len(need), cols, dtype=torch.int32), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    m = starts[-1] + case["padded"]
    s = dict(news=news, lens=lens, most=most, rows=m, lengths=torch.tensor(lens, dtype=torch.int32).cuda(), table=table.cuda())
    s["starts"] = torch.tensor(starts, dtype=torch.int32).cuda() if case["new"] > 1 or case["padded"] else None
    s["Q"] = _randn(g, m, q * d, std=1.5)
    s.update(_cache(case, g, n_pages))
    # the rows of the padding stay as they are
    s["C"], s["LSE"] = torch.zeros(m, q * d, dtype=BF, device="cuda"), torch.zeros(q, m, dtype=F32, device="cuda")
    return s


def _plan_chunk(N, s):
    c = s["case"]
    plan = dict(q_cnt=c["q"], kv_cnt=c["kv"], q_off=c["q_off"], kv_off=c["kv_off"], head_dim=c["dim"])
    s["shape"] = N.attn_chunk_shape(s["rows"], c["n_seq"], c["new"], s["most"], plan, c["group"])
    s["pages"] = N.kv_pages(s["K"], s["V"], s.get("K_exp"), s.get("V_exp"))
    _workspace(N, s, N.binding.NTP_CALL_ATTN_CHUNK_SHARD)


def _run_chunk(s):
    c = s["case"]
    if own:
        s["N"].ntp_attn_chunk_shard(s["shape"], s["pages"], s["Q"], s["starts"], s["table"], s["lengths"], s["C"], s["LSE"], handle=s["handle"])
        return dict(C=s["C"], LSE=s["LSE"])
    q, kv, d, page = (c[k] for k in ("q", "kv", "dim", "page"))
    C, LSE = torch.zeros_like(s["C"]), torch.zeros_like(s["LSE"])
    head = [(c["q_off"] + j) // c["group"] - c["kv_off"] for j in range(q)]
    row = 0
    for i, (n, length) in enumerate(zip(s["news"], s["lens"])):
        pages = s["table"][i, :(length + page - 1) // page].long()

        def tokens(name):
            t = s[name].view(BF if c["bits"] == 16 else U8)[pages]
            if c["bits"] == 8:
                t = t.view(E4M3).to(F32) * _two_to(s[name + "_exp"].view(U8)[pages].to(torch.int32) - 127)[..., None]
            return t.to(F32).transpose(0, 1).reshape(kv, -1, d)[head, :length]

        k, v = tokens("K"), tokens("V")
        x = s["Q"][row:row + n].view(n, q, d).transpose(0, 1).to(F32)
        score = torch.matmul(x, k.transpose(1, 2)) * (1.0 / math.sqrt(d))
        seen = torch.arange(length, device="cuda") < torch.arange(length - n + 1, length + 1, device="cuda")[:, None]
        score = score.masked_fill(~seen, -math.inf)
        top = score.amax(2, keepdim=True) if length else torch.full((q, n, 1), -math.inf, device="cuda")
        base = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = torch.exp(score - base)
        total = p.sum(2, keepdim=True)
        C[row:row + n] = (torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)).transpose(0, 1).reshape(n, q * d).to(BF)
        LSE[:, row:row + n] = (base + torch.log(total))[:, :, 0]
        row += n
    return dict(C=C, LSE=LSE)


def run(state):
    return _RUN[state["case"]["kind"]](state)


# ---- the definitions in 64 bits -----------------------------------------------------------
def exact(case, seed):
    return _EXACT[case["kind"]](case, _PREPARE[case["kind"]](case, seed, _gen(seed)))


def _rotation(c, s, rows):
    """The rows' rotations as complex numbers [M, 1, rotary / 2]."""
    a = s["positions"][rows].double().unsqueeze(1) * s["inv_freq"].unsqueeze(0)
    return torch.complex(torch.cos(a), torch.sin(a)).unsqueeze(1)


def _apply(c, x, z):
    rd = c["rotary"]
    even, odd = (slice(0, rd, 2), slice(1, rd, 2)) if c["pairs"] else (slice(0, rd // 2), slice(rd // 2, rd))
    w = torch.complex(x[..., even].contiguous(), x[..., odd].contiguous()) * z
    x = x.clone()
    x[..., even], x[..., odd] = w.real, w.imag
    return x


def _grid8(x):
    """A head's values in units of its power of two, each taken to the nearest e4m3 number (ties to the even one), and that power."""
    def power_of_two(e):
        return ((e.long() + 1023) << 52).view(F64)

    top = x.abs().max(-1).values
    power = power_of_two(torch.frexp(top).exponent - 9)  # (top / power in 256 .. 512)
    power = torch.where(top > 448.0 * power, 2.0 * power, power).clamp(min=2.0 ** -111)
    power = torch.where(top > 0, power, torch.ones_like(power))
    u = x / power.unsqueeze(-1)
    step = power_of_two(torch.frexp(u.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return torch.round(u / step) * step, power


def _exact_append(c, s):
    m, q, kv, d, page = (c[k] for k in ("tokens", "q", "kv", "dim", "page"))
    gq, gk = s["q_gamma"].double(), s["k_gamma"].double()
    x = s["QKV"].double().view(m, q + 2 * kv, d)
    size = torch.sqrt((x[:, :q + kv] ** 2).sum(2) / d + EPS).unsqueeze(2)
    heads = x[:, :q + kv] / size
    heads = torch.cat([heads[:, :q] * gq, heads[:, q:] * gk], 1)
    if c["rotary"]:
        heads = _apply(c, heads, _rotation(c, s, slice(None)))
    keep = s["slots"] >= 0
    out = dict(Q=heads[:, :q].reshape(m, q * d))

    def put(into, rows):  # into: [pages, kv, page, ...]
        flat = into.transpose(1, 2).reshape(-1, kv, *into.shape[3:]).clone()
        flat[s["slots"][keep]] = rows[keep]
        return flat.view(into.shape[0], page, kv, *into.shape[3:]).transpose(1, 2)

    for n, t in (("K", heads[:, q:]), ("V", x[:, q + kv:])):
        if c["bits"] == 8:
            t, power = _grid8(t)
            out[n + "_exp"] = put(torch.ones(s[n].shape[:3], dtype=F64, device="cuda"), power)
        out[n] = put(torch.zeros(s[n].shape, dtype=F64, device="cuda"), t)
    return dict(out, Kout=heads[:, q:].reshape(m, kv * d)) if c["prompt"] else out


def _exact_bwd(c, s):
    m, q, kv, d = (c[k] for k in ("tokens", "q", "kv", "dim"))
    out = s["dQKV"].double().clone()
    sums = {"q": torch.zeros(d, dtype=F64, device="cuda"), "k": torch.zeros(d, dtype=F64, device="cuda")}
    for lo in range(0, m, 4096):
        rows = slice(lo, min(m, lo + 4096))
        for which, n, first in (("q", q, 0), ("k", kv, q)):
            t = s["QKV"][rows].double().view(-1, q + 2 * kv, d)[:, first:first + n]
            grad = s["d" + which.upper()][rows].double().view(-1, n, d)
            if c["rotary"]:
                grad = _apply(c, grad, _rotation(c, s, rows).conj())
            size = torch.sqrt((t ** 2).sum(2, keepdim=True) / d + EPS)
            unit = t / size
            sums[which] += (grad * unit).sum((0, 1))
            grad = grad * s[which + "_gamma"].double()
            grad = (grad - unit * ((grad * unit).sum(2, keepdim=True) / d)) / size
            out[rows, first * d:(first + n) * d] = grad.reshape(-1, n * d)
    return dict(dQKV=out, d_q_gamma=sums["q"], d_k_gamma=sums["k"])


def _exact_chunk(c, s):
    q, kv, d, page = (c[k] for k in ("q", "kv", "dim", "page"))
    C, LSE = torch.zeros(s["rows"], q, d, dtype=F64, device="cuda"), torch.zeros(q, s["rows"], dtype=F64, device="cuda")
    start = 0
    for i in range(c["n_seq"]):
        n, length = s["news"][i], s["lens"][i]
        LSE[:, start:start + n] = -math.inf
        at = torch.arange(length, device="cuda")
        page_of, row_of = s["table"][i].long()[at // page], at % page
        for g in range(kv):
            mine = [j for j in range(q) if (c["q_off"] + j) // c["group"] == c["kv_off"] + g]
            if not mine:
                continue
            k, v = (s[t].view(BF if c["bits"] == 16 else U8)[page_of, g, row_of] for t in ("K", "V"))
            if c["bits"] == 8:
                k, v = (t.view(E4M3).double() * torch.pow(2.0, s[e].view(U8)[page_of, g, row_of].double() - 127.0).unsqueeze(1) for t, e in ((k, "K_exp"), (v, "V_exp")))
            k, v = k.double(), v.double()
            step = max(1, (1 << 27) // (max(length, 1) * len(mine)))
            for lo in range(max(0, n - length), n, step):  # (rows before have nothing to look at)
                hi = min(n, lo + step)
                x = s["Q"][start + lo:start + hi].double().view(-1, q, d)[:, mine].permute(1, 0, 2).reshape(-1, d)
                score = (x @ k.t()).view(len(mine), hi - lo, length) / math.sqrt(d)
                last = length - n + torch.arange(lo, hi, device="cuda")
                score.masked_fill_(at.unsqueeze(0) > last.unsqueeze(1), -math.inf)
                total = torch.logsumexp(score, 2)
                w = torch.exp(score - total.unsqueeze(2)).view(-1, length) @ v
                for a, j in enumerate(mine):
                    C[start + lo:start + hi, j] = w.view(len(mine), hi - lo, d)[a]
                    LSE[j, start + lo:start + hi] = total[a]
        start += n
    return dict(C=C.view(-1, q * d), LSE=LSE)


_PREPARE = dict(norm_append=_prepare_append, norm_bwd=_prepare_bwd, chunk=_prepare_chunk)
_PLAN = dict(norm_append=_plan_append, norm_bwd=_plan_bwd, chunk=_plan_chunk)
_RUN = dict(norm_append=_run_append, norm_bwd=_run_bwd, chunk=_run_chunk)
_EXACT = dict(norm_append=_exact_append, norm_bwd=_exact_bwd, chunk=_exact_chunk)
