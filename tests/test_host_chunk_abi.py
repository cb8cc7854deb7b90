"""What the calls of the head norms, the 8-bit pages and the chunk attention refuse; nothing is launched here: every refused call is refused by its argument checks, and calls
with nothing to do return at once."""
import ctypes as C

import pytest

import paper_2504_06095_amd as N
from paper_2504_06095_amd import binding as Bd
from tests.test_host_block_abi import BAD_CACHE, P, _has_gpu, h  # noqa: F401

INV, ALIGN, UNSUP, NODEV = Bd.NTP_ERR_INVALID_ARG, Bd.NTP_ERR_ALIGNMENT, Bd.NTP_ERR_UNSUPPORTED, Bd.NTP_ERR_NO_DEVICE
BAD_PAGES = BAD_CACHE + [(dict(format=2), INV), (dict(format=-1), INV)]
BAD_PAGES8 = BAD_PAGES + [(dict(K_exp=None), INV), (dict(V_exp=None), INV), (dict(exp_stride=0), INV), (dict(exp_stride=24), ALIGN), (dict(K_exp=P + 4), ALIGN),
                          (dict(V_exp=P + 8), ALIGN), (dict(page_stride=1032), ALIGN)]


def _pages(c, fp8):
    v = dict(K=P, V=2 * P, K_exp=20 * P, V_exp=21 * P, n_pages=4, page_stride=1024, exp_stride=16, page_size=16, format=1)
    if not fp8:
        v.update(K_exp=None, V_exp=None, exp_stride=0, format=0)
    v.update(c or {})
    return Bd.KvPages(**v)


def _append(h, s=None, c=None, n=None, fp8=True, **k):
    v = dict(M=4, q_cnt=3, kv_cnt=1, head_dim=64, rotary_dim=64, interleaved=0)
    v.update(s or {})
    nn = dict(q_gamma=P, k_gamma=P, eps=1e-6)
    nn.update(n or {})
    a = dict(QKV=3 * P, ldqkv=320, positions=4 * P, slots=5 * P, inv_freq=6 * P, Qout=7 * P, ldq=192, Kout=8 * P, ldk=64, pages=True, norm=True)
    a.update(k)
    return Bd.lib().ntp_qk_norm_append_shard(h, C.byref(Bd.KvAppendShape(**v)), C.byref(Bd.QkNorm(**nn)) if a["norm"] else None, C.byref(_pages(c, fp8)) if a["pages"] else None,
                                             a["QKV"], a["ldqkv"], a["positions"], a["slots"], a["inv_freq"], a["Qout"], a["ldq"], a["Kout"], a["ldk"], None)


def test_append_refuses(h):  # noqa: F811
    for s in (dict(M=-1), dict(q_cnt=-1), dict(kv_cnt=-1), dict(rotary_dim=-16), dict(rotary_dim=72), dict(rotary_dim=80), dict(rotary_dim=8)):
        assert _append(h, s) == INV, s
    for s in (dict(head_dim=96), dict(M=1 << 31), dict(q_cnt=1 << 22), dict(kv_cnt=(1 << 31) - 1, q_cnt=(1 << 31) - 1)):
        assert _append(h, s) == UNSUP, s
    for fp8, bad in ((False, BAD_PAGES), (True, BAD_PAGES8)):
        for c, want in bad:
            assert _append(h, None, c, fp8=fp8) == want, (fp8, c)
    for n in (dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert _append(h, n=n) == INV, n
    for n in (dict(q_gamma=P + 8), dict(k_gamma=P + 2)):
        assert _append(h, n=n) == ALIGN, n
    for k in (dict(QKV=None), dict(positions=None), dict(inv_freq=None), dict(slots=None), dict(pages=False), dict(ldqkv=312), dict(ldq=184), dict(ldk=56)):
        assert _append(h, **k) == INV, k
    for k in (dict(QKV=P + 8), dict(Qout=P + 8), dict(Kout=P + 8), dict(ldqkv=324), dict(ldq=196), dict(ldk=68), dict(positions=P + 2), dict(slots=P + 4), dict(inv_freq=P + 4)):
        assert _append(h, **k) == ALIGN, k
    for k in (dict(Qout=3 * P, ldq=192), dict(Qout=3 * P + 128, ldq=320), dict(Kout=3 * P, ldk=320), dict(Kout=3 * P + 384, ldk=64), dict(Qout=7 * P, Kout=7 * P, ldq=192, ldk=64)):
        assert _append(h, **k) == INV, k
    assert _append(None) == INV
    # nothing to do; eps does not count without a norm
    assert _append(h, dict(M=0), QKV=None, positions=None, slots=None, inv_freq=None, Qout=None, Kout=None) == 0
    assert _append(h, n=dict(q_gamma=None, k_gamma=None, eps=0.0), slots=None, pages=False, Qout=None, Kout=None) == 0
    if not _has_gpu():  # (with one, the calls would run)
        assert _append(h) == NODEV and _append(h, norm=False) == NODEV and _append(h, fp8=False) == NODEV
        assert _append(h, n=dict(q_gamma=None, k_gamma=None, eps=0.0)) == NODEV


def _bwd(h, s=None, n=None, **k):
    v = dict(M=4, q_cnt=3, kv_cnt=1, head_dim=64, rotary_dim=64, interleaved=0)
    v.update(s or {})
    nn = dict(q_gamma=P, k_gamma=P, eps=1e-6)
    nn.update(n or {})
    a = dict(QKV=3 * P, ldqkv=320, dQ=4 * P, lddq=192, dK=5 * P, lddk=64, positions=6 * P, inv_freq=7 * P, dQKV=8 * P, lddqkv=320, da=9 * P, db=10 * P)
    a.update(k)
    return Bd.lib().ntp_qk_norm_shard_bwd(h, C.byref(Bd.KvAppendShape(**v)), C.byref(Bd.QkNorm(**nn)), a["QKV"], a["ldqkv"], a["dQ"], a["lddq"], a["dK"], a["lddk"], a["positions"],
                                          a["inv_freq"], a["dQKV"], a["lddqkv"], a["da"], a["db"], 0, None)


def test_gradient_refuses(h):  # noqa: F811
    for s in (dict(M=-1), dict(q_cnt=-1), dict(rotary_dim=8)):
        assert _bwd(h, s) == INV, s
    for s in (dict(head_dim=32), dict(M=1 << 31)):
        assert _bwd(h, s) == UNSUP, s
    for n in (dict(eps=0.0), dict(q_gamma=None), dict(k_gamma=None)):  # (gradients of gammas that there are not)
        assert _bwd(h, n=n) == INV, n
    for k in (dict(QKV=None), dict(dQ=None), dict(dK=None), dict(positions=None), dict(inv_freq=None), dict(dQKV=None), dict(ldqkv=312), dict(lddq=184), dict(lddk=56), dict(lddqkv=312)):
        assert _bwd(h, **k) == INV, k
    for k in (dict(QKV=P + 8), dict(dQ=P + 8), dict(dK=P + 8), dict(dQKV=P + 8), dict(ldqkv=324), dict(lddq=196), dict(lddk=68), dict(lddqkv=324), dict(positions=P + 2),
              dict(inv_freq=P + 4), dict(da=P + 2), dict(db=P + 1)):
        assert _bwd(h, **k) == ALIGN, k
    # over what is read, but for the gradients in their own columns
    for k in (dict(dQKV=3 * P), dict(dQKV=4 * P), dict(dQKV=5 * P), dict(dQ=8 * P + 128, lddq=320), dict(dK=8 * P, lddk=320), dict(dK=8 * P + 2 * 192, lddk=64)):
        assert _bwd(h, **k) == INV, k
    assert _bwd(None) == INV
    assert _bwd(h, dict(M=0), da=None, db=None, dQ=None, dK=None, QKV=None, dQKV=None) == 0
    if not _has_gpu():
        assert _bwd(h, dQ=8 * P, lddq=320, dK=8 * P + 2 * 192, lddk=320) == NODEV
        assert _bwd(h, dQ=8 * P + 2 * 256, lddq=320, lddqkv=320, dK=5 * P) == INV  # (the columns behind the keys and the next row's first)


def _chunk(h, s=None, c=None, fp8=True, **k):
    v = dict(M=6, n_seq=2, max_new=4, max_len=40, q_cnt=3, kv_cnt=1, q_off=0, kv_off=0, group=4, head_dim=64)
    v.update(s or {})
    a = dict(Q=3 * P, ldq=192, starts=9 * P, table=4 * P, ldt=3, lengths=5 * P, C=6 * P, ldc=192, LSE=7 * P, pages=True)
    a.update(k)
    return Bd.lib().ntp_attn_chunk_shard(h, C.byref(Bd.AttnChunkShape(**v)), C.byref(_pages(c, fp8)) if a["pages"] else None, a["Q"], a["ldq"], a["starts"], a["table"], a["ldt"],
                                         a["lengths"], a["C"], a["ldc"], a["LSE"], None)


def test_chunk_refuses(h):  # noqa: F811
    for s in (dict(M=-1), dict(n_seq=-1), dict(max_new=-1), dict(max_len=-1), dict(q_cnt=-1), dict(q_off=-1), dict(kv_off=-1), dict(group=0), dict(q_off=2), dict(kv_off=1),
              dict(group=2), dict(kv_cnt=0)):
        assert _chunk(h, s) == INV, s
    for s in (dict(head_dim=32), dict(M=1 << 31), dict(M=1 << 30), dict(max_len=(1 << 30) + 1), dict(n_seq=1 << 26, max_len=1 << 20)):
        assert _chunk(h, s) == UNSUP, s
    assert _chunk(h, dict(n_seq=(1 << 24) + 1, M=(1 << 24) + 1, max_new=1, max_len=0, q_cnt=1), starts=None, ldt=0) == UNSUP  # (more than a launch has room for)
    assert _chunk(h, dict(n_seq=1 << 17, M=1 << 21, max_new=1 << 21, max_len=0, q_cnt=6), ldt=0) == UNSUP  # (row tiles past 2^31, were every sequence as long)
    assert _chunk(h, dict(q_cnt=(1 << 20) + 8, group=1 << 21, M=1, n_seq=1, max_new=1), ldq=1 << 30, ldc=1 << 30) == UNSUP
    for fp8, bad in ((False, BAD_PAGES), (True, BAD_PAGES8)):
        for c, want in bad:
            assert _chunk(h, None, c, fp8=fp8) == want, (fp8, c)
    for k in (dict(Q=None), dict(table=None), dict(lengths=None), dict(C=None), dict(ldq=184), dict(ldc=184), dict(ldt=2), dict(pages=False), dict(starts=None)):
        assert _chunk(h, **k) == INV, k
    for k in (dict(Q=P + 8), dict(C=P + 2), dict(ldq=196), dict(ldc=196), dict(starts=P + 1), dict(table=P + 2), dict(lengths=P + 1), dict(LSE=P + 2)):
        assert _chunk(h, **k) == ALIGN, k
    assert _chunk(None) == INV
    for s in (dict(M=0), dict(n_seq=0), dict(q_cnt=0), dict(max_new=0)):
        assert _chunk(h, s) == 0, s
    if not _has_gpu():
        assert _chunk(h) == NODEV and _chunk(h, dict(M=2), starts=None) == NODEV and _chunk(h, LSE=None, fp8=False) == NODEV


def test_workspace_sizes(h):  # noqa: F811
    L, n = Bd.lib(), C.c_int64()
    ask = lambda call, s: (L.ntp_workspace_bytes(h, call, C.byref(s), C.byref(n)), n.value)  # noqa: E731
    plan = dict(q_cnt=3, kv_cnt=1, q_off=0, kv_off=0, head_dim=128)
    st, need = ask(Bd.NTP_CALL_QK_NORM, N.kv_append_shape(4096, plan))
    assert st == 0 and 0 < need <= 4 * 256 * 2 * 128 * 4 and ask(Bd.NTP_CALL_QK_NORM, N.kv_append_shape(0, plan)) == (0, 0)
    assert ask(Bd.NTP_CALL_QK_NORM, N.kv_append_shape(-1, plan))[0] == INV
    assert ask(Bd.NTP_CALL_ATTN_CHUNK_SHARD, N.attn_chunk_shape(4, 4, 1, 0, plan, 3))[0] == 0
    assert ask(Bd.NTP_CALL_ATTN_CHUNK_SHARD, N.attn_chunk_shape(-1, 4, 1, 0, plan, 3))[0] == INV


def test_the_binding_checks_its_tensors():
    import torch
    t = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    with pytest.raises(ValueError):  # not on the device
        N.kv_pages(t(2, 1, 16, 64), t(2, 1, 16, 64))
    with pytest.raises(TypeError):
        N.kv_pages(t(2, 1, 16, 64, dt=torch.float16), t(2, 1, 16, 64, dt=torch.float16))
    e = t(2, 1, 16, 64, dt=torch.uint8).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError):  # 8 bits without their powers of two
        N.kv_pages(e, e)
    with pytest.raises(TypeError):
        N.kv_pages(e, t(2, 1, 16, 64))
    with pytest.raises(ValueError):
        N.kv_pages(t(2, 1, 16, 64), t(2, 1, 16, 64), t(2, 1, 16, dt=torch.uint8), t(2, 1, 16, dt=torch.uint8))
    with pytest.raises(TypeError):
        N.qk_norm(t(64, dt=torch.float32))
