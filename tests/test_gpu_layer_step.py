"""The norms, the paged cache and the attention of one new token together with the layer calls, as a user runs them, on a real MI355X: a prompt, then new
tokens one by one from a captured graph; and the gradient of a norm - MLP - residual chain.  One rank's shard stands for the layer (its partial sums are
taken as the all-reduced ones), and the oracle computes the same in float64 without rounding anything.

Tolerance: on any path from a layer's input to its output lie at most eight roundings to bf16, each half a step, 2^-8, of a value that is no larger
than the largest of the matrix: 8 * 2^-8 of the largest output."""
import sys

import numpy as np
import pytest

from oracle import block_oracle as B
from oracle import ntp_oracle as O

pytestmark = pytest.mark.gpu
TOL = 8 * 2.0 ** -8
EPS = 1e-5


def _say(msg):
    print(f"[gpu-case] {msg}", file=sys.stderr, flush=True)


def f64(t):
    return t.double().cpu().numpy()


def _close(got, want, what):
    err = np.abs(f64(got) - want).max() / np.abs(want).max()
    assert err <= TOL, f"{what}: {err}"


class Layer:
    """Weights of one rank's shard of a layer, and its calls."""

    def __init__(self, H, ffn, n_q, n_kv, d, tp, rank, seed=0):
        import torch
        import paper_2504_06095_amd as N
        self.torch, self.N, self.H, self.d = torch, N, H, d
        self.plan, self.group = N.ntp_attn_shard_plan(n_q, n_kv, d, tp, rank), n_q // n_kv
        self.n_r = N.ntp_shard_plan(ffn, tp, rank)[1]
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        p = self.plan
        self.Wqkv, self.Wo = self.rand(p["w_qkv"], H, std=H ** -0.5), self.rand(p["w_o"], H, std=p["w_o"] ** -0.5)
        self.A, self.Bw = self.rand(self.n_r, H, std=H ** -0.5), self.rand(self.n_r, H, std=self.n_r ** -0.5)
        v = lambda base: (base + 0.2 * torch.randn(H, device="cuda", generator=self.g)).to(torch.bfloat16)
        self.n1, self.post1, self.gate1, self.n2 = v(1.0), v(1.0), v(0.5), v(1.0)
        self.inv_freq = torch.tensor([10000.0 ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float64, device="cuda")
        self.h = N.ntp_create()
        N.ntp_set_workspace(torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), handle=self.h)

    def rand(self, r, c, std=1.0):
        return (self.torch.randn(r, c, device="cuda", generator=self.g) * std).to(self.torch.bfloat16)

    def buffers(self, M):
        e = lambda w: self.torch.zeros(M, w, dtype=self.torch.bfloat16, device="cuda")
        pad = (self.n_r + 7) // 8 * 8
        return dict(X=e(self.H), Y=e(self.H), QKV=e(self.plan["w_qkv"]), C=e(self.plan["w_o"]), Z=e(self.H), X1=e(self.H), Y1=e(self.H), P=e(pad), G=e(pad), Z2=e(self.H), X2=e(self.H),
                    Q=e(self.plan["w_o"]))

    def before_attention(self, b, M):
        N, p = self.N, self.plan
        N.ntp_block_norm_fwd(N.block_norm_shape(M, self.H, eps=EPS), b["X"], Y=b["Y"], pre_gamma=self.n1, handle=self.h)
        N.ntp_attn_proj_shard_fwd(M, self.H, p["w_qkv"], p["w_o"], b["Y"], self.Wqkv, b["QKV"], handle=self.h)

    def after_attention(self, b, M):
        N, p = self.N, self.plan
        N.ntp_attn_proj_shard_fwd(M, self.H, p["w_qkv"], p["w_o"], C_=b["C"], Wo=self.Wo, Zpart=b["Z"], handle=self.h)
        N.ntp_block_norm_fwd(N.block_norm_shape(M, self.H, gate=N.binding.NTP_GATE_CHANNEL, eps=EPS), b["X"], b["Z"], b["X1"], b["Y1"], post_gamma=self.post1, gate=self.gate1,
                             pre_gamma=self.n2, handle=self.h)
        N.ntp_mlp_shard_fwd(b["Y1"], self.A, self.Bw, b["P"][:, :self.n_r], b["G"][:, :self.n_r], b["Z2"], self.n_r, handle=self.h)
        N.ntp_block_norm_fwd(N.block_norm_shape(M, self.H, branch_scale=0.5, eps=EPS), b["X1"], b["Z2"], b["X2"], handle=self.h)

    def oracle(self, X, n_seq):
        """The layer's output for whole sequences, X [n_seq * S, H] in float64."""
        p, d, S = self.plan, self.d, X.shape[0] // n_seq
        q, kv = p["q_cnt"], p["kv_cnt"]
        _, y, _ = B.block_norm_fwd(X, None, {"pre_gamma": f64(self.n1)}, B.RMS, EPS)
        QKV = y @ f64(self.Wqkv).T
        pos = np.tile(np.arange(S), n_seq)
        x = QKV.reshape(-1, q + 2 * kv, d).copy()
        x[:, :q + kv] = B.rotate(x[:, :q + kv], pos, f64(self.inv_freq), False)
        C = O.attn_core_shard_fwd(x.reshape(QKV.shape), p, self.group, d, n_seq, True)
        Z = C @ f64(self.Wo)
        X1, Y1, _ = B.block_norm_fwd(X, Z, dict(post_gamma=f64(self.post1), gate=f64(self.gate1), pre_gamma=f64(self.n2)), B.RMS, EPS)
        _, _, Z2 = O.mlp_shard_fwd(Y1, f64(self.A).T, f64(self.Bw))
        return X1 + 0.5 * Z2


@pytest.mark.parametrize("H,ffn,n_q,n_kv,d,tp,rank,n_seq,S,page", [
    (1024, 4096, 16, 4, 64, 3, 1, 3, 37, 16),     # a rank in the middle: its KV heads are read by parts of their groups
    (2048, 4096, 16, 16, 128, 7, 0, 1, 300, 64),  # no grouped heads, the uneven shard of TP 8 -> 7
    (1024, 2816, 16, 2, 128, 8, 7, 2, 129, 32),
])
def test_a_prompt_and_then_token_by_token(H, ffn, n_q, n_kv, d, tp, rank, n_seq, S, page):
    import torch
    import paper_2504_06095_amd as N
    _say(f"layer step, hidden {H}, heads {n_q} / {n_kv} of {d} at TP {tp} rank {rank}, {n_seq} sequences of {S} tokens and 5 new ones")
    L = Layer(H, ffn, n_q, n_kv, d, tp, rank)
    p, new = L.plan, 5
    T = S + new
    X = L.rand(n_seq * T, H)
    want = L.oracle(f64(X), n_seq).reshape(n_seq, T, H)
    X = X.view(n_seq, T, H)
    per_seq = (T + page - 1) // page
    cache_t = [torch.full((n_seq * per_seq + 3, p["kv_cnt"], page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = N.kv_cache(*cache_t)
    table = torch.randperm(n_seq * per_seq + 3, generator=torch.Generator().manual_seed(1))[:n_seq * per_seq].view(n_seq, per_seq)
    slot = lambda s, t: int(table[s, t // page]) * page + t % page
    table_d = table.to(torch.int32).cuda()
    # the prompt: queries and keys are rotated inside QKV, which the attention core then reads
    M = n_seq * S
    b = L.buffers(M)
    b["X"].copy_(X[:, :S].reshape(M, H))
    L.before_attention(b, M)
    wq, wk = p["w_o"], p["kv_cnt"] * d
    pos = torch.arange(S, dtype=torch.int32, device="cuda").repeat(n_seq)
    slots = torch.tensor([slot(s, t) for s in range(n_seq) for t in range(S)], device="cuda")
    N.ntp_kv_append_shard(N.kv_append_shape(M, p), cache, b["QKV"], pos, slots, L.inv_freq, b["QKV"][:, :wq], b["QKV"][:, wq:wq + wk], handle=L.h)
    N.ntp_attn_core_shard_fwd(N.attn_core_shape(n_seq, S, p, L.group, True), b["QKV"], b["C"], handle=L.h)
    L.after_attention(b, M)
    torch.cuda.synchronize()
    _close(b["X2"], want[:, :S].reshape(M, H), "prompt")
    # new tokens: one captured step, replayed with the positions, slots and lengths of each token
    b = L.buffers(n_seq)
    pos, slots, lengths = (torch.zeros(n_seq, dtype=t, device="cuda") for t in (torch.int32, torch.int64, torch.int32))

    def step():
        L.before_attention(b, n_seq)
        N.ntp_kv_append_shard(N.kv_append_shape(n_seq, p), cache, b["QKV"], pos, slots, L.inv_freq, b["Q"], handle=L.h)
        N.ntp_attn_decode_shard(N.attn_decode_shape(n_seq, per_seq * page, p, L.group), cache, b["Q"], table_d, lengths, b["C"], handle=L.h)
        L.after_attention(b, n_seq)

    def inputs(t):
        b["X"].copy_(X[:, t])
        pos.fill_(t)
        slots.copy_(torch.tensor([slot(s, t) for s in range(n_seq)]))
        lengths.fill_(t + 1)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    inputs(S)
    step()  # eagerly: the first new token
    torch.cuda.synchronize()
    first = b["X2"].clone()
    _close(first, want[:, S], "first new token")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for t in range(S, T):
        inputs(t)
        b["X2"].fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _close(b["X2"], want[:, t], f"token {t} replayed")
        if t == S:
            assert torch.equal(b["X2"], first)
    N.ntp_destroy(L.h)


@pytest.mark.parametrize("norm", [B.RMS, B.LAYER])
@pytest.mark.parametrize("fp32", [False, True], ids=["bf16 residual", "fp32 residual"])
def test_gradient_of_a_residual_block(norm, fp32):
    """X' = X + gate * post(MLP(pre(X))), forward and backward, two micro-batches whose weight gradients add up."""
    import torch
    import paper_2504_06095_amd as N
    M, H = 200, 1024
    L = Layer(H, 4096, 16, 4, 64, 7, 2, seed=3)
    rt = torch.float32 if fp32 else torch.bfloat16
    first = N.block_norm_shape(M, H, norm, eps=EPS, residual_fp32=fp32)
    last = N.block_norm_shape(M, H, norm, N.binding.NTP_GATE_CHANNEL, fp32, EPS)
    e = lambda w=H, dt=torch.bfloat16: torch.zeros(M, w, dtype=dt, device="cuda")
    pad = (L.n_r + 7) // 8 * 8
    vec = lambda: torch.zeros(H, device="cuda")
    grads = dict(n1=vec(), post=vec(), gate=vec(), A=torch.zeros(L.n_r, H, device="cuda"), B=torch.zeros(L.n_r, H, device="cuda"))
    sums = {}
    for micro in range(2):
        X, dOut = L.rand(M, H).to(rt), L.rand(M, H, std=0.1).to(rt)
        Y, P, G, Z, Xo = e(), e(pad), e(pad), e(), e(dt=rt)
        st1, st2 = torch.zeros(4, M, device="cuda"), torch.zeros(4, M, device="cuda")
        N.ntp_block_norm_fwd(first, X, Y=Y, Stats=st1, pre_gamma=L.n1, handle=L.h)
        N.ntp_mlp_shard_fwd(Y, L.A, L.Bw, P[:, :L.n_r], G[:, :L.n_r], Z, L.n_r, handle=L.h)
        N.ntp_block_norm_fwd(last, X, Z, Xo, None, st2, post_gamma=L.post1, gate=L.gate1, handle=L.h)
        dRes, dZ, dP, dY, dX = e(dt=rt), e(), e(pad), e(), e(dt=rt)
        N.ntp_block_norm_bwd(last, dOut, None, None, Z, st2, dRes, dZ, post_gamma=L.post1, gate=L.gate1, d_post_gamma=grads["post"], d_gate=grads["gate"], accumulate=micro > 0,
                             handle=L.h)
        N.ntp_mlp_shard_bwd(dZ, Y, L.A, L.Bw, P[:, :L.n_r], G[:, :L.n_r], dP[:, :L.n_r], dY, grads["A"], grads["B"], L.n_r, accumulate=micro > 0, handle=L.h)
        N.ntp_block_norm_bwd(first, dRes, dY, X, None, st1, dX, None, pre_gamma=L.n1, d_pre_gamma=grads["n1"], accumulate=micro > 0, handle=L.h)
        torch.cuda.synchronize()
        # the same in float64
        x, d, w = f64(X), f64(dOut), dict(post_gamma=f64(L.post1), gate=f64(L.gate1))
        _, y, s1 = B.block_norm_fwd(x, None, {"pre_gamma": f64(L.n1)}, norm, EPS)
        _, _, z = O.mlp_shard_fwd(y, f64(L.A).T, f64(L.Bw))
        xo, _, s2 = B.block_norm_fwd(x, z, w, norm, EPS)
        up = B.block_norm_bwd(d, None, xo, z, s2, w, norm)
        dp, dy, dA, dB = O.mlp_shard_bwd(up["dZ"], y, f64(L.A).T, f64(L.Bw))
        down = B.block_norm_bwd(up["dX"], dy, x, None, s1, {"pre_gamma": f64(L.n1)}, norm, branch=False)
        _close(Xo, xo, "forward")
        _close(dX, down["dX"], "dX")
        for k, v in dict(n1=down["pre_gamma"], post=up["post_gamma"], gate=up["gate"], A=dA.T, B=dB).items():
            sums[k] = sums.get(k, 0.0) + v
    for k, v in sums.items():
        _close(grads[k], v, k)
    N.ntp_destroy(L.h)


@pytest.mark.parametrize("H,ffn,n_q,n_kv,d,tp,rank,n_seq,S,page", [
    (1024, 4096, 16, 4, 64, 3, 1, 2, 1300, 16),
    (1024, 2816, 16, 16, 128, 7, 0, 1, 600, 64),
])
def test_steps_whose_attention_is_cut(H, ffn, n_q, n_kv, d, tp, rank, n_seq, S, page):
    """The same at lengths that the call of one new token shares out among the workgroups and joins."""
    import paper_2504_06095_amd as N
    plan = N.ntp_attn_shard_plan(n_q, n_kv, d, tp, rank)
    assert N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_DECODE_SHARD, N.attn_decode_shape(n_seq, S, plan, n_q // n_kv)) > 0
    test_a_prompt_and_then_token_by_token(H, ffn, n_q, n_kv, d, tp, rank, n_seq, S, page)
