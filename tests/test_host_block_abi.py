"""What the norm, cache and decode calls refuse, and their workspace sizes; nothing is launched here: every refused call is refused by its argument
checks, and calls with nothing to do return at once."""
import ctypes as C

import pytest

import paper_2504_06095_amd as N
from paper_2504_06095_amd import binding as Bd

P = 0x10000000  # an aligned address that nothing dereferences
INV, ALIGN, UNSUP = Bd.NTP_ERR_INVALID_ARG, Bd.NTP_ERR_ALIGNMENT, Bd.NTP_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def h():
    handle = N.ntp_create()
    yield handle.ptr
    N.ntp_destroy(handle)


def _has_gpu():
    import torch
    return torch.cuda.is_available()


def _norm_fwd(h, shape=None, w=None, **k):
    s = dict(M=4, H=64, norm=0, gate=0, residual_fp32=0, eps=1e-5, residual_scale=1.0, branch_scale=1.0)
    s.update(shape or {})
    v = dict(post_gamma=None, post_beta=None, gate=None, pre_gamma=P, pre_beta=None, ldgate=0)
    v.update(w or {})
    a = dict(X=P, ldx=64, Z=2 * P, ldz=64, Xout=3 * P, ldxo=64, Y=4 * P, ldy=64, Stats=5 * P)
    a.update(k)
    return Bd.lib().ntp_block_norm_fwd(h, C.byref(Bd.BlockNormShape(**s)), C.byref(Bd.BlockNormWeights(**v)), a["X"], a["ldx"], a["Z"], a["ldz"], a["Xout"], a["ldxo"],
                                       a["Y"], a["ldy"], a["Stats"], None)


def test_block_norm_forward_refuses(h):
    for shape in (dict(M=-1), dict(H=-8), dict(norm=2), dict(gate=3), dict(gate=-1), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")),
                  dict(residual_scale=float("nan")), dict(branch_scale=float("inf"))):
        assert _norm_fwd(h, shape) == INV, shape
    assert _norm_fwd(h, dict(H=60)) == ALIGN
    assert _norm_fwd(h, dict(H=32776)) == UNSUP and _norm_fwd(h, dict(M=1 << 31)) == UNSUP
    for w in (dict(post_beta=P), dict(pre_gamma=None, pre_beta=P), dict(gate=P), dict(pre_gamma=None)):
        assert _norm_fwd(h, None, w) == INV, w
    assert _norm_fwd(h, dict(gate=1)) == INV                              # a gate is announced and not given
    assert _norm_fwd(h, dict(gate=2), dict(gate=P, ldgate=56)) == INV      # rows of the gate overlap
    assert _norm_fwd(h, dict(gate=2), dict(gate=P, ldgate=68)) == ALIGN
    assert _norm_fwd(h, None, dict(post_gamma=P), Z=None, Xout=None) == INV  # a norm behind a block that is not there
    for k in (dict(X=None), dict(Y=None), dict(Z=None), dict(ldx=56), dict(ldz=56), dict(ldxo=56), dict(ldy=56), dict(Xout=P, ldxo=72)):
        assert _norm_fwd(h, **k) == INV, k
    assert _norm_fwd(h, None, dict(pre_gamma=None), Y=None, Xout=None) == INV  # nothing to write
    for k in (dict(X=P + 8), dict(Z=P + 2), dict(Xout=P + 8), dict(Y=P + 8), dict(Stats=P + 2), dict(ldx=68), dict(ldz=68), dict(ldxo=68), dict(ldy=68)):
        assert _norm_fwd(h, **k) == ALIGN, k
    assert _norm_fwd(h, dict(residual_fp32=1), ldx=66) == ALIGN
    assert _norm_fwd(h, None, dict(pre_gamma=P + 4)) == ALIGN
    assert _norm_fwd(None) == INV
    assert Bd.lib().ntp_block_norm_fwd(h, None, None, *[None, 0] * 4, None, None) == INV
    assert _norm_fwd(h, dict(M=0), X=None, Z=None, Xout=None, Y=None, Stats=None) == 0
    assert _norm_fwd(h, dict(H=0)) == 0


def _norm_bwd(h, shape=None, w=None, g=None, **k):
    s = dict(M=4, H=64, norm=0, gate=0, residual_fp32=0, eps=1e-5, residual_scale=1.0, branch_scale=1.0)
    s.update(shape or {})
    v = dict(post_gamma=P, post_beta=None, gate=None, pre_gamma=P, pre_beta=None, ldgate=0)
    v.update(w or {})
    gr = dict(post_gamma=P, post_beta=None, gate=None, pre_gamma=P, pre_beta=None, ldgate=0)
    gr.update(g or {})
    a = dict(dXout=P, lddxo=64, dY=2 * P, lddy=64, Xout=3 * P, ldxo=64, Z=4 * P, ldz=64, Stats=5 * P, dX=6 * P, lddx=64, dZ=7 * P, lddz=64)
    a.update(k)
    return Bd.lib().ntp_block_norm_bwd(h, C.byref(Bd.BlockNormShape(**s)), C.byref(Bd.BlockNormWeights(**v)), a["dXout"], a["lddxo"], a["dY"], a["lddy"], a["Xout"], a["ldxo"],
                                       a["Z"], a["ldz"], a["Stats"], a["dX"], a["lddx"], a["dZ"], a["lddz"], C.byref(Bd.BlockNormGrads(**gr)), 0, None)


def test_block_norm_backward_refuses(h):
    for shape in (dict(M=-1), dict(norm=2), dict(eps=-1.0), dict(gate=1)):
        assert _norm_bwd(h, shape) == INV, shape
    assert _norm_bwd(h, dict(H=60)) == ALIGN and _norm_bwd(h, dict(H=32776)) == UNSUP
    for k in (dict(dY=None), dict(Xout=None), dict(Z=None), dict(Stats=None), dict(dX=None), dict(dZ=None), dict(lddxo=56), dict(lddy=56), dict(ldxo=56), dict(ldz=56),
              dict(lddx=56), dict(lddz=56), dict(dX=P, lddx=72)):
        assert _norm_bwd(h, **k) == INV, k
    for g in (dict(post_beta=P), dict(pre_beta=P), dict(gate=P)):
        assert _norm_bwd(h, None, None, g) == INV, g  # gradients of what there is not
    assert _norm_bwd(h, None, dict(pre_gamma=None)) == INV
    assert _norm_bwd(h, dict(gate=2), dict(gate=P, ldgate=64), dict(gate=P, ldgate=56)) == INV
    for k in (dict(dXout=P + 8), dict(dY=P + 8), dict(Xout=P + 8), dict(Z=P + 8), dict(Stats=P + 1), dict(dX=P + 8), dict(dZ=P + 8), dict(lddx=68), dict(lddz=68),
              dict(lddy=68), dict(ldz=68)):
        assert _norm_bwd(h, **k) == ALIGN, k
    assert _norm_bwd(h, None, None, dict(pre_gamma=P + 4)) == ALIGN
    assert _norm_bwd(None) == INV


def _append(h, s=None, c=None, **k):
    v = dict(M=4, q_cnt=3, kv_cnt=1, head_dim=64, rotary_dim=64, interleaved=0)
    v.update(s or {})
    cc = dict(K=P, V=2 * P, n_pages=4, page_stride=1024, page_size=16)
    cc.update(c or {})
    a = dict(QKV=3 * P, ldqkv=320, positions=4 * P, slots=5 * P, inv_freq=6 * P, Qout=7 * P, ldq=192, Kout=8 * P, ldk=64, cache=True)
    a.update(k)
    return Bd.lib().ntp_kv_append_shard(h, C.byref(Bd.KvAppendShape(**v)), C.byref(Bd.KvCache(**cc)) if a["cache"] else None, a["QKV"], a["ldqkv"], a["positions"], a["slots"],
                                        a["inv_freq"], a["Qout"], a["ldq"], a["Kout"], a["ldk"], None)


BAD_CACHE = [(dict(K=None), INV), (dict(V=None), INV), (dict(n_pages=-1), INV), (dict(page_stride=1016), INV), (dict(page_stride=-8), INV), (dict(page_size=8), UNSUP),
             (dict(page_size=48), UNSUP), (dict(page_size=0), UNSUP), (dict(page_size=1 << 17), UNSUP), (dict(n_pages=1 << 31), UNSUP), (dict(page_stride=1028), ALIGN),
             (dict(K=P + 8), ALIGN), (dict(V=P + 2), ALIGN)]


def test_append_refuses(h):
    for s in (dict(M=-1), dict(q_cnt=-1), dict(kv_cnt=-1), dict(rotary_dim=-16), dict(rotary_dim=72), dict(rotary_dim=80), dict(rotary_dim=8)):
        assert _append(h, s) == INV, s
    for s in (dict(head_dim=96), dict(M=1 << 31), dict(q_cnt=1 << 22)):
        assert _append(h, s) == UNSUP, s
    for c, want in BAD_CACHE:
        assert _append(h, None, c) == want, c
    for k in (dict(QKV=None), dict(positions=None), dict(inv_freq=None), dict(slots=None), dict(cache=False), dict(ldqkv=312), dict(ldq=184), dict(ldk=56)):
        assert _append(h, **k) == INV, k
    for k in (dict(QKV=P + 8), dict(Qout=P + 8), dict(Kout=P + 8), dict(ldqkv=324), dict(ldq=196), dict(ldk=68), dict(positions=P + 2), dict(slots=P + 4), dict(inv_freq=P + 4)):
        assert _append(h, **k) == ALIGN, k
    # memory shared with QKV other than by the same columns
    for k in (dict(Qout=3 * P, ldq=192), dict(Qout=3 * P + 128, ldq=320), dict(Kout=3 * P, ldk=320), dict(Kout=3 * P + 384, ldk=64), dict(Qout=3 * P + 640, ldq=192)):
        assert _append(h, **k) == INV, k
    assert _append(None) == INV
    assert Bd.lib().ntp_kv_append_shard(h, None, None, None, 0, None, None, None, None, 0, None, 0, None) == INV
    # nothing to do
    assert _append(h, dict(M=0), QKV=None, positions=None, slots=None, inv_freq=None, Qout=None, Kout=None) == 0
    assert _append(h, slots=None, cache=False, Qout=None, Kout=None) == 0


def _decode(h, s=None, c=None, **k):
    v = dict(n_seq=2, max_len=40, q_cnt=3, kv_cnt=1, q_off=0, kv_off=0, group=4, head_dim=64)
    v.update(s or {})
    cc = dict(K=P, V=2 * P, n_pages=4, page_stride=1024, page_size=16)
    cc.update(c or {})
    a = dict(Q=3 * P, ldq=192, table=4 * P, ldt=3, lengths=5 * P, C=6 * P, ldc=192, LSE=7 * P, cache=True)
    a.update(k)
    return Bd.lib().ntp_attn_decode_shard(h, C.byref(Bd.AttnDecodeShape(**v)), C.byref(Bd.KvCache(**cc)) if a["cache"] else None, a["Q"], a["ldq"], a["table"], a["ldt"],
                                          a["lengths"], a["C"], a["ldc"], a["LSE"], None)


def test_decode_refuses(h):
    for s in (dict(n_seq=-1), dict(max_len=-1), dict(q_cnt=-1), dict(q_off=-1), dict(kv_off=-1), dict(group=0), dict(q_off=2), dict(kv_off=1), dict(group=2), dict(kv_cnt=0)):
        assert _decode(h, s) == INV, s
    assert _decode(h, dict(head_dim=32)) == UNSUP
    for c, want in BAD_CACHE:
        assert _decode(h, None, c) == want, c
    for k in (dict(Q=None), dict(table=None), dict(lengths=None), dict(C=None), dict(ldq=184), dict(ldc=184), dict(ldt=2), dict(cache=False)):
        assert _decode(h, **k) == INV, k
    for k in (dict(Q=P + 8), dict(C=P + 2), dict(ldq=196), dict(ldc=196), dict(table=P + 2), dict(lengths=P + 1), dict(LSE=P + 2)):
        assert _decode(h, **k) == ALIGN, k
    assert _decode(None) == INV
    assert _decode(h, dict(n_seq=0)) == 0 and _decode(h, dict(q_cnt=0)) == 0


def test_launches_that_count_more_than_32_bits_of_threads_are_refused(h):
    for H, M in ((64, 1 << 26), (2048, 1 << 26), (32768, 1 << 22)):
        wide = {k: H for k in ("ldx", "ldz", "ldxo", "ldy")}
        assert _norm_fwd(h, dict(M=M, H=H), **wide) == UNSUP, (H, M)
        if not _has_gpu():  # (with one, the call would run)
            assert _norm_fwd(h, dict(M=M - 4, H=H), **wide) == Bd.NTP_ERR_NO_DEVICE
    far = dict(Qout=1 << 45, Kout=1 << 46)  # (not inside QKV's rows)
    assert _append(h, dict(M=(1 << 31) - 1), **far) == UNSUP
    assert _decode(h, dict(n_seq=1 << 24, q_cnt=1)) == UNSUP and _decode(h, dict(n_seq=(1 << 24) // 3 + 1)) == UNSUP


def test_workspace_sizes(h):
    L, n = Bd.lib(), C.c_int64()
    ask = lambda call, s: (L.ntp_workspace_bytes(h, call, C.byref(s), C.byref(n)), n.value)
    # the sums over the tokens: nothing for one row, at most one set of five vectors per compute unit
    assert ask(3, N.block_norm_shape(1, 1024)) == (0, 0)
    st, need = ask(3, N.block_norm_shape(4096, 1024))
    assert st == 0 and 0 < need and need % (5 * 1024 * 4) == 0
    assert ask(3, N.block_norm_shape(4, 60))[0] == INV
    plan = N.ntp_attn_shard_plan(64, 8, 128, 30, 0)
    assert ask(4, N.attn_decode_shape(4, 0, plan, 8))[0] == 0
    assert ask(4, N.attn_decode_shape(-1, 5, plan, 8))[0] == INV


def test_the_binding_checks_its_tensors():
    import torch
    bf = torch.bfloat16
    t = lambda *s, dt=bf: torch.zeros(*s, dtype=dt)
    with pytest.raises(ValueError):  # not on the device
        N.ntp_block_norm_fwd(N.block_norm_shape(2, 8), t(2, 8), Y=t(2, 8), pre_gamma=t(8))
    with pytest.raises(TypeError):
        N.ntp_block_norm_fwd(N.block_norm_shape(2, 8), t(2, 8), Y=t(2, 8), pre_gamma=t(8, dt=torch.float32))
    with pytest.raises(ValueError):
        N.ntp_block_norm_fwd(N.block_norm_shape(2, 8), t(3, 8), Y=t(2, 8))
    with pytest.raises(ValueError):
        N.kv_cache(t(2, 1, 16, 64), t(2, 1, 16, 64))
    with pytest.raises(TypeError):
        N.kv_cache(t(2, 1, 16, 64, dt=torch.float16), t(2, 1, 16, 64, dt=torch.float16))


def test_append_compares_columns_where_leading_dimensions_agree(h):
    """Columns of one wide matrix beside QKV's share no element with it; two outputs may not share one either."""
    if not _has_gpu():  # (with one, the calls would run)
        wide = dict(ldqkv=576, ldq=576, ldk=576)  # 320 columns of QKV, 192 and 64 beside them
        for k in (dict(Qout=3 * P + 2 * 320, Kout=3 * P + 2 * 512), dict(QKV=3 * P + 2 * 256, Qout=3 * P, Kout=3 * P + 2 * 192), dict(Qout=3 * P, Kout=3 * P + 2 * 192),
                  # the rows of one matrix behind the other's, in the same columns
                  dict(Qout=3 * P + 2 * 4 * 576, Kout=3 * P - 2 * 4 * 576)):
            assert _append(h, **{**wide, **k}) == Bd.NTP_ERR_NO_DEVICE, k
        assert _append(h, dict(M=1), Qout=3 * P, ldq=192, Kout=3 * P + 2 * 192, ldk=64) == Bd.NTP_ERR_NO_DEVICE  # one row: in place whatever the leading dimension says
    for k in (dict(Qout=3 * P + 2 * 312, Kout=3 * P + 2 * 512), dict(Qout=3 * P + 2 * 392), dict(Qout=3 * P - 2 * 576 + 2 * 312), dict(Kout=3 * P + 2 * 3 * 576 + 2 * 312)):
        k = {**dict(Qout=9 * P, Kout=10 * P), **k}
        assert _append(h, ldqkv=576, ldq=576, ldk=576, **k) == INV, k
    # queries and keys in the same place
    for k in (dict(Qout=7 * P, Kout=7 * P, ldq=192, ldk=64), dict(Qout=7 * P, Kout=7 * P + 2 * 128, ldq=256, ldk=256), dict(Qout=7 * P, Kout=7 * P + 2 * 3 * 192 + 2 * 64, ldq=192, ldk=64)):
        assert _append(h, **k) == INV, k
