"""The 4-bit cache and eviction entry points turn bad arguments into status codes before anything is launched; no GPU needed."""
import ctypes as C

import numpy as np
import pytest

from tests import kv4_ref

ONE = C.c_void_p(4096)
ODD = C.c_void_p(4096 + 8)


@pytest.fixture(scope="module")
def ic():
    import paper_2603_12201_amd as m
    m.lib()
    return m


def _kd(ic, **kw):
    d = dict(B=2, Tn=3, Lk=100, reserved=0, pos0=0, pool_rows=200)
    d.update(kw)
    return ic.Kv4Desc(**d)


def _ad(ic, **kw):
    d = dict(B=2, Tq=1, Lk=100, H_q=32, d_qk=576, d_v=512, v_off=0, row_elems=576, k_sel=64, sm_scale=0.04)
    d.update(kw)
    return ic.AttnDesc(**d)


def _pc(ic, page=64, max_pages=2, table=4096, lens=None):
    return ic.PagedCache(page, max_pages, table, lens)


@pytest.mark.parametrize("fn", ["ic_kv4_write", "ic_kv4_read"])
def test_rows_are_checked(ic, fn):
    L, S = ic.lib(), ic.Status

    def call(d, a=ONE, b=ONE, pc=None):
        return getattr(L, fn)(C.byref(d) if d else None, C.byref(pc) if pc else None, a, b, None)

    assert call(None) == S.ERR_NULL
    assert call(_kd(ic), None) == S.ERR_NULL and call(_kd(ic), ONE, None) == S.ERR_NULL
    for bad in (dict(B=0), dict(Tn=0), dict(Lk=-1), dict(pool_rows=0), dict(pool_rows=199), dict(pool_rows=1 << 31), dict(pos0=1 << 41),
                dict(pos0=-(1 << 41)), dict(B=1 << 16, Tn=1 << 16, pool_rows=(1 << 31) - 1)):
        assert call(_kd(ic, **bad)) == S.ERR_SHAPE, bad
    assert call(_kd(ic, reserved=1)) == S.ERR_UNSUPPORTED
    assert call(_kd(ic), ODD) == S.ERR_SHAPE and call(_kd(ic), ONE, ODD) == S.ERR_SHAPE
    assert call(_kd(ic), pc=_pc(ic, table=None)) == S.ERR_NULL                   # neither lengths nor a table
    assert call(_kd(ic), pc=_pc(ic, page=48)) == S.ERR_SHAPE and call(_kd(ic), pc=_pc(ic, max_pages=1)) == S.ERR_SHAPE
    assert call(_kd(ic, pool_rows=199), pc=_pc(ic, table=None, lens=4096)) == S.ERR_SHAPE   # ragged but dense
    assert b"rows" in L.ic_last_error()


def test_attention_is_checked(ic):
    L, S = ic.lib(), ic.Status
    ws = ic.lib().ic_sparse_attn_kv4_workspace(C.byref(_ad(ic, k_sel=2048)))
    assert ws > 0 and ws % 256 == 0
    assert L.ic_sparse_attn_kv4_workspace(C.byref(_ad(ic, B=1, Tq=4096, Lk=5000))) == 0
    assert L.ic_sparse_attn_kv4_workspace(None) == 0 and L.ic_sparse_attn_kv4_workspace(C.byref(_ad(ic, H_q=33))) == 0
    assert L.ic_sparse_attn_kv4_workspace(C.byref(_ad(ic, d_qk=64, d_v=64, v_off=64, row_elems=128))) == 0

    def attn(d, pool=200, Q=ONE, kv=ONE, idx=ONE, O=ONE, w=ONE, n=1 << 40, pc=None):
        return L.ic_sparse_attn_kv4(C.byref(d) if d else None, C.byref(pc) if pc else None, pool, Q, kv, idx, O, None, w, n, None)

    def probs(d, pool=200, Q=ONE, kv=ONE, idx=ONE, lse=ONE, p=ONE, pc=None):
        return L.ic_attn_probs_kv4(C.byref(d) if d else None, C.byref(pc) if pc else None, pool, Q, kv, idx, lse, p, None)

    for f in (attn, probs):
        assert f(None) == S.ERR_NULL
        for k in ("Q", "kv", "idx"):
            assert f(_ad(ic), **{k: None}) == S.ERR_NULL
        assert f(_ad(ic), Q=ODD) == S.ERR_SHAPE and f(_ad(ic), kv=ODD) == S.ERR_SHAPE
        assert f(_ad(ic), pool=199) == S.ERR_SHAPE and f(_ad(ic), pool=1 << 31) == S.ERR_SHAPE
        assert f(_ad(ic, d_qk=64, d_v=64, v_off=64, row_elems=128)) == S.ERR_UNSUPPORTED
        assert f(_ad(ic, row_elems=640)) == S.ERR_UNSUPPORTED and f(_ad(ic, H_q=33)) == S.ERR_UNSUPPORTED
        assert f(_ad(ic, sm_scale=0.0)) == S.ERR_SHAPE and f(_ad(ic, k_sel=0)) == S.ERR_SHAPE
        assert f(_ad(ic), pc=_pc(ic, table=None)) == S.ERR_NULL and f(_ad(ic), pc=_pc(ic, page=32)) == S.ERR_SHAPE
    assert attn(_ad(ic), O=None) == S.ERR_NULL and attn(_ad(ic), O=ODD) == S.ERR_SHAPE
    assert probs(_ad(ic), lse=None) == S.ERR_NULL and probs(_ad(ic), p=None) == S.ERR_NULL
    big = _ad(ic, k_sel=2048)
    assert attn(big, w=None) == S.ERR_WORKSPACE and attn(big, w=ODD) == S.ERR_WORKSPACE and attn(big, n=ws - 1) == S.ERR_WORKSPACE


def test_weights_and_eviction_are_checked(ic):
    L, S = ic.lib(), ic.Status
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (2, 1 << 30, 4, 10), (1 << 12, 1, 4, 1 << 20)):
        assert L.ic_attn_weight_add(*bad, ONE, ONE, None, ONE, ONE, 1 << 40, None) == S.ERR_SHAPE
        assert L.ic_attn_weight_add_workspace(*bad) == 0
    assert L.ic_attn_weight_add(1 << 16, 1, 1, 1, ONE, ONE, None, ONE, ONE, 1 << 40, None) == S.ERR_UNSUPPORTED
    for a in ((None, ONE, ONE), (ONE, None, ONE), (ONE, ONE, None)):
        assert L.ic_attn_weight_add(1, 1, 8, 64, a[0], a[1], None, a[2], None, 0, None) == S.ERR_NULL
    need = L.ic_attn_weight_add_workspace(1, 4096, 2048, 4096)
    assert need > 0 and L.ic_attn_weight_add_workspace(32, 1, 2048, 65536) == 0
    assert L.ic_attn_weight_add(1, 4096, 2048, 4096, ONE, ONE, None, ONE, None, 0, None) == S.ERR_WORKSPACE
    assert L.ic_attn_weight_add(1, 4096, 2048, 4096, ONE, ONE, None, ONE, ONE, need - 1, None) == S.ERR_WORKSPACE

    def keep(B=1, Lk=100, n=50, first=0, recent=0, w=ONE, k=ONE, lens=ONE):
        return L.ic_evict_keep(B, Lk, w, None, n, first, recent, k, lens, None, ONE, 1 << 40, None)

    for bad in (dict(B=0), dict(Lk=0), dict(n=0), dict(n=101), dict(first=-1), dict(recent=-1), dict(first=30, recent=21), dict(B=1 << 12, Lk=1 << 20)):
        assert keep(**bad) == S.ERR_SHAPE, bad
    assert keep(w=None) == S.ERR_NULL and keep(k=None) == S.ERR_NULL and keep(lens=None) == S.ERR_NULL
    ws = L.ic_evict_keep_workspace(1, 1 << 20)
    if ws:
        assert L.ic_evict_keep(1, 1 << 20, ONE, None, 50, 0, 0, ONE, ONE, None, ONE, ws - 1, None) == S.ERR_WORKSPACE

    far = 4096 + (1 << 20)

    def move(n=1, B=1, Lk=100, nk=50, keep=ONE, src=4096, dst=far, sr=100, dr=50, rb=16, res=0, sp=None, dp=None):
        m = (ic.CacheMove * 17)()
        for i in range(17):
            m[i].src, m[i].dst, m[i].src_rows, m[i].dst_rows, m[i].row_bytes, m[i].reserved = src, dst, sr, dr, rb, res
        return L.ic_cache_compact(m if n != -7 else None, abs(n), B, Lk, nk, keep, C.byref(sp) if sp else None, C.byref(dp) if dp else None, None)

    assert move(n=-7) == S.ERR_NULL and move(keep=None) == S.ERR_NULL and move(src=None) == S.ERR_NULL and move(dst=None) == S.ERR_NULL
    for bad in (dict(n=0), dict(n=17), dict(B=0), dict(nk=101), dict(nk=0), dict(rb=6), dict(rb=0), dict(sr=99), dict(dr=49), dict(src=4098),
                dict(dst=4096 + 160), dict(dst=4096), dict(sp=_pc(ic, page=32)), dict(dp=_pc(ic, max_pages=0))):
        assert move(**bad) == S.ERR_SHAPE, bad
    assert move(res=1) == S.ERR_UNSUPPORTED
    same = _pc(ic)
    assert move(src=4096, dst=4096, sp=same, dp=same) == S.ERR_SHAPE             # rows onto themselves


def test_caches_of_one_call_must_not_write_over_each_other(ic):
    """Two moves of 100 rows to 50 of 400 bytes each, at addresses that nothing reads before the refusal."""
    S, L = ic.Status, ic.lib()
    far = 1 << 20

    def move(src0, dst0, src1, dst1):
        m = (ic.CacheMove * 2)()
        for c, (src, dst) in zip(m, ((src0, dst0), (src1, dst1))):
            c.src, c.dst, c.src_rows, c.dst_rows, c.row_bytes, c.reserved = src, dst, 100, 50, 400, 0
        return L.ic_cache_compact(m, 2, 1, 100, 50, C.c_void_p(4096), None, None, None)

    assert move(far, 2 * far, 3 * far, 2 * far) == S.ERR_SHAPE                   # one destination twice
    assert move(far, 2 * far, 3 * far, 2 * far + 19996) == S.ERR_SHAPE           # its last row
    assert move(far, 2 * far, 3 * far, far + 4000) == S.ERR_SHAPE                # the second writes what the first reads
    assert move(far, 2 * far, 2 * far + 8000, 4 * far) == S.ERR_SHAPE            # the second reads what the first writes


def test_binding_refuses_what_it_can_see(ic):
    import torch
    t = torch.zeros((1, 4, 576), dtype=torch.bfloat16)
    with pytest.raises(ic.IcError):
        ic.kv4_write(t, torch.zeros((1, 8, 400), dtype=torch.uint8))             # host tensors
    with pytest.raises(ic.IcError):
        ic.evict_keep(torch.zeros((1, 8)), 4)
    assert ic.KV4_ROW_BYTES == 400
    assert C.sizeof(ic.Kv4Desc) == 32 and C.sizeof(ic.CacheMove) == 40


def test_the_reference_row_by_hand():
    """The tests' own packing on values whose codes can be read off."""
    bits = np.zeros((1, 576), dtype=np.uint16)
    f = np.zeros(576, dtype=np.float32)
    f[:8] = [6.0, -6.0, 0.25, 0.75, 1.25, 2.5, 5.0, -0.2]                        # scale 2^0: ties to the even code
    f[128:130] = [6.5, 1.0]                                                      # over 6: scale 2^1
    f[512] = 3.0
    bits[0] = (f.view(np.uint32) >> 16).astype(np.uint16)
    p = kv4_ref.pack(bits)[0]
    codes = [7, 15, 0, 2, 2, 4, 6, 8]
    assert p[:4].tolist() == [codes[2 * i] | codes[2 * i + 1] << 4 for i in range(4)]
    assert p[64] == (5 | 1 << 4) and p[384:388].tolist() == [127, 128, 27, 27] and not p[388:].any()
    u = kv4_ref.unpack(p[None])[0]
    assert u[:8].tolist() == [6.0, -6.0, 0.0, 1.0, 1.0, 2.0, 4.0, 0.0] and u[128:130].tolist() == [6.0, 1.0] and u[512] == 3.0
    f[5] = np.inf
    bits[0] = (f.view(np.uint32) >> 16).astype(np.uint16)
    assert kv4_ref.pack(bits)[0, 384] == 255 and np.isnan(kv4_ref.unpack(kv4_ref.pack(bits))[0, :128]).all()


def test_a_layout_that_the_call_refuses_needs_no_workspace(ic):
    """With 2048 rows, which are split and need one otherwise."""
    L, S = ic.lib(), ic.Status
    assert L.ic_sparse_attn_kv4_workspace(C.byref(_ad(ic, k_sel=2048))) > 0
    for bad in (dict(k_sel=2048, d_qk=64, d_v=64, v_off=64, row_elems=128), dict(k_sel=2048, row_elems=640), dict(k_sel=(1 << 24) + 1),
                dict(k_sel=2048, sm_scale=-1.0)):
        d = _ad(ic, **bad)
        assert L.ic_sparse_attn_kv4_workspace(C.byref(d)) == 0, bad
        assert L.ic_sparse_attn_kv4(C.byref(d), None, 200, ONE, ONE, ONE, ONE, None, ONE, 1 << 40, None) in (S.ERR_UNSUPPORTED, S.ERR_SHAPE)
