"""Refusals of the rotary, page-table and 4-bit-cache entry points: every one is
decided on the host before anything is launched (no GPU)."""
import ctypes
import math

import pytest

import paper_2603_22300_amd as sfa

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below fails validation
ODD = ctypes.c_void_p(0x1001)


@pytest.fixture(scope="module")
def L():
    return sfa.lib()


def _plan(d=128, sections=(64,), **kw):
    return sfa.sfa_rope_plan(d, sections, **kw)


def test_plan_refusals():
    for kw in (dict(d=128, sections=()), dict(d=128, sections=(1,) * 5), dict(d=128, sections=(65,)),
               dict(d=128, sections=(64, 0)), dict(d=128, sections=(-1,)), dict(d=1, sections=(1,)),
               dict(d=128, sections=(32, 33)), dict(theta=0.5), dict(theta=math.inf), dict(theta=math.nan)):
        with pytest.raises(sfa.SfaError) as e:
            _plan(**kw)
        assert e.value.status == sfa.SFA_EINVAL
    with pytest.raises(sfa.SfaError) as e:
        _plan(d=258, sections=(64,))
    assert e.value.status == sfa.SFA_ENOTSUP
    for kw in (dict(pairing="pairs"), dict(order="rows")):
        with pytest.raises(ValueError):
            _plan(**kw)


def _st(*s):
    return (ctypes.c_int64 * len(s))(*s)


def _rope(L, **kw):
    a = dict(x=FAKE, xs=None, pos=FAKE, pa=0, pb=0, plan=_plan().ref, B=2, H=3, n=5, inverse=0, x_t=2, y_t=3,
             y=FAKE, ys=None, stream=None)
    a.update(kw)
    return L.sfa_rope(*a.values())


def _enc(L, **kw):
    a = dict(x=FAKE, xs=None, pos=FAKE, pa=0, pb=0, plan=_plan().ref, B=2, H=3, n=5, k=16, x_t=2, idx=FAKE,
             idx_t=0, val=FAKE, val_t=2, stream=None)
    a.update(kw)
    return L.sfa_rope_encode(*a.values())


def _bwd(L, **kw):
    a = dict(idx=FAKE, idx_t=0, dval=FAKE, pos=FAKE, pa=0, pb=0, plan=_plan().ref, B=2, H=3, n=5, k=16, dx_t=2,
             dx=FAKE, ds=None, stream=None)
    a.update(kw)
    return L.sfa_rope_encode_bwd(*a.values())


def test_rope_refusals(L):
    for f in (_rope, _enc, _bwd):
        assert f(L, pos=None) == 1 and f(L, plan=None) == 1
        assert f(L, B=0) == 1 and f(L, H=0) == 1 and f(L, n=-1) == 1
        assert f(L, pa=-1) == 1 and f(L, pb=-1) == 1
        assert f(L, B=1 << 16, n=1 << 15) == 1                     # tokens past 2^31 - 1
        assert f(L, n=0, pos=None) == 0                            # empty: no-op
        bad = _plan()
        bad._c.rot = 130
        assert f(L, plan=bad.ref) == 1
        bad = _plan()
        bad._c.axis[3] = 1                                         # an axis that pos does not have
        assert f(L, plan=bad.ref) == 1
    assert _rope(L, x=None) == 1 and _rope(L, y=None) == 1 and _rope(L, x_t=5) == 1 and _rope(L, y_t=0) == 1
    assert _rope(L, xs=_st(-1, 1, 1)) == 1
    assert _rope(L, ys=_st(0, 128 * 5, 128)) == 1                  # written rows may not overlap
    assert _rope(L, ys=_st(3 * 5 * 128, 5 * 128, 64)) == 1
    assert _rope(L, x=ODD) == 1 and _rope(L, y=ODD) == 1
    assert _enc(L, k=0) == 1 and _enc(L, k=129) == 1 and _enc(L, idx=None) == 1 and _enc(L, val=None) == 1
    assert _enc(L, idx_t=2) == 1 and _enc(L, val_t=0) == 1 and _enc(L, x_t=0) == 1
    assert _bwd(L, k=0) == 1 and _bwd(L, dval=None) == 1 and _bwd(L, dx=None) == 1 and _bwd(L, dx_t=5) == 1
    assert _bwd(L, ds=_st(0, 0, 0)) == 1 and _bwd(L, idx_t=3) == 1


def _tables(L, **kw):
    a = dict(old=FAKE, new=ctypes.c_void_p(0x2000), B=4, table=FAKE, max_pages=8, P=16, free=FAKE, num=64, fin=FAKE,
             fout=FAKE, got=ctypes.c_void_p(0x3000), starts=None, slots=None, pos=None, rows=0, ws=FAKE,
             ws_bytes=ctypes.c_size_t(0), stream=None)
    a.update(kw)
    return L.sfa_page_tables(*a.values())


def test_page_tables_refusals(L):
    need = L.sfa_page_tables_workspace(4)
    assert need > 0 and L.sfa_page_tables_workspace(0) == 0 and L.sfa_page_tables_workspace((1 << 20) + 1) == 0
    assert _tables(L) == 4 and _tables(L, ws_bytes=ctypes.c_size_t(need - 1)) == 4
    ok = dict(ws_bytes=ctypes.c_size_t(need))
    for name in ("new", "table", "free", "fin", "fout", "got", "ws"):
        assert _tables(L, **{name: None}, **ok) == 1, name
    assert _tables(L, B=0, **ok) == 1 and _tables(L, max_pages=0, **ok) == 1 and _tables(L, num=0, **ok) == 1
    assert _tables(L, P=24, **ok) == 1 and _tables(L, P=0, **ok) == 1 and _tables(L, rows=-1, **ok) == 1
    assert _tables(L, max_pages=1 << 27, **ok) == 1                # capacity beyond 2^30
    assert _tables(L, num=1 << 27, **ok) == 1                      # slots beyond int32
    assert _tables(L, got=FAKE, **ok) == 1                         # got_len over old_len
    assert _tables(L, got=ctypes.c_void_p(0x2000), **ok) == 1      # over new_len
    assert _tables(L, ws=ODD, **ok) == 1


def _app(L, **kw):
    a = dict(k_new=FAKE, v_new=FAKE, st=None, slots=None, n_new=None, seq_len=FAKE, B=2, Hkv=2, T=3, d=128, k=16,
             table=None, max_pages=0, P=100, num=2, ci=FAKE, cv=FAKE, cs=FAKE, vc=FAKE, vs=FAKE, k_idx=None,
             k_val=None, v_out=None, kt=2, vt=3, stream=None)
    a.update(kw)
    return L.sfa_kv_append_q4(*a.values())


def test_append_q4_refusals(L):
    for name in ("k_new", "v_new", "seq_len", "ci", "cv", "cs", "vc", "vs"):
        assert _app(L, **{name: None}) == 1, name
    assert _app(L, slots=FAKE) == 1                                # slots and seq_len
    assert _app(L, slots=FAKE, seq_len=None, table=FAKE) == 1
    assert _app(L, slots=FAKE, seq_len=None, n_new=FAKE) == 1
    assert _app(L, k_idx=FAKE) == 1 and _app(L, k_val=FAKE) == 1   # together or not at all
    assert _app(L, table=FAKE, max_pages=4) == 1                   # page size not a power of two
    assert _app(L, table=FAKE, max_pages=0, P=64) == 1
    assert _app(L, table=FAKE, max_pages=1 << 25, P=64) == 1
    assert _app(L, num=3) == 1                                     # contiguous: B sequences
    assert _app(L, num=1 << 27, P=64, slots=FAKE, seq_len=None) == 1
    assert _app(L, k=0) == 1 and _app(L, k=129) == 1 and _app(L, T=-1) == 1 and _app(L, P=0) == 1
    assert _app(L, kt=5) == 1 and _app(L, vt=1) == 1
    assert _app(L, st=_st(0, 0, -1, 0, 0, 0)) == 1
    assert _app(L, ci=ODD) == 1 and _app(L, vs=ODD) == 1 and _app(L, k_new=ODD) == 1
    assert _app(L, d=80, k=8) == 2 and _app(L, k=12) == 2 and _app(L, d=288) == 2
    assert _app(L, B=1 << 12, num=1 << 12, T=1 << 19) == 2


def _dec(L, **kw):
    a = dict(q=FAKE, qi=None, qv=None, ci=FAKE, cv=FAKE, cs=FAKE, vc=FAKE, vs=FAKE, table=FAKE, max_pages=4, P=64,
             num=16, seq_len=None, B=2, Hq=8, Hkv=2, d=128, k=16, scale=0.1, window=0, n_global=0, qit=0, qvt=2,
             o_t=2, o=FAKE, lse=None, ws=FAKE, ws_bytes=ctypes.c_size_t(1), stream=None)
    a.update(kw)
    return L.sfa_attn_decode_q4(*a.values())


def test_decode_q4_refusals(L):
    need = L.sfa_attn_decode_q4_workspace(2, 8, 256, 128)
    assert need > 0 and _dec(L) == 4 and _dec(L, ws_bytes=ctypes.c_size_t(need - 1)) == 4
    for a in ((0, 8, 256, 128), (2, 0, 256, 128), (2, 8, 0, 128), (2, 8, 256, 0), (2, 8, 256, 257)):
        assert L.sfa_attn_decode_q4_workspace(*a) == 0
    ok = dict(ws_bytes=ctypes.c_size_t(need))
    for name in ("q", "ci", "cv", "cs", "vc", "vs", "o", "ws"):
        assert _dec(L, **{name: None}, **ok) == 1, name
    assert _dec(L, qi=FAKE, qv=FAKE, **ok) == 1                    # dense query and codes
    assert _dec(L, q=None, qi=FAKE, **ok) == 1
    assert _dec(L, P=8, **ok) == 1 and _dec(L, P=48, **ok) == 1 and _dec(L, max_pages=0, **ok) == 1
    assert _dec(L, window=-1, **ok) == 1 and _dec(L, n_global=-1, **ok) == 1
    assert _dec(L, Hq=7, **ok) == 1 and _dec(L, scale=float("nan"), **ok) == 1 and _dec(L, o_t=5, **ok) == 1
    assert _dec(L, ci=ODD, **ok) == 1 and _dec(L, vc=ctypes.c_void_p(0x1008), **ok) == 1
    assert _dec(L, Hq=18, **ok) == 2 and _dec(L, d=80, k=8, **ok) == 2 and _dec(L, k=20, **ok) == 2
    assert _dec(L, d=288, **ok) == 2 and _dec(L, B=40000, Hq=2, **ok) == 2
    assert _dec(L, table=None, P=(1 << 30) + 1, **ok) == 2


def test_python_refuses_cpu_tensors():
    import torch
    plan = _plan()
    x, pos = torch.zeros(1, 1, 4, 128), torch.zeros(4, dtype=torch.int32)
    for f in (lambda: sfa.sfa_rope(x, pos, plan), lambda: sfa.sfa_rope_encode(x, pos, plan, 8),
              lambda: sfa.sfa_rope_encode_bwd(torch.zeros(1, 1, 4, 8, dtype=torch.int32), torch.zeros(1, 1, 4, 8), pos, plan),
              lambda: sfa.sfa_page_tables(None, pos, torch.zeros(4, 2, dtype=torch.int32), pos, pos[:1], 16),
              lambda: sfa.sfa_kv_append_q4(x, x, pos[:1], *[torch.zeros(1)] * 5, k=8)):
        with pytest.raises(ValueError):
            f()
