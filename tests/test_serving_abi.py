"""The serving calls (block tables, slot-mapped writes, selected pages, four-bit pages): what they refuse, on the host.  Dummy
pointers: every refusal comes before a launch, so no GPU is touched."""
import ctypes as C

import pytest
import torch

A = 0x10000  # sixteen-byte aligned, never read


@pytest.fixture(scope="module")
def b():
    from paper_2506_11418_b200 import binding
    return binding


def resize(b, **kw):
    a = dict(lens=A, new_lens=2 * A, Bz=2, page=64, tables=3 * A, row=8, ring=4 * A, n_pages=16, state=5 * A, slots=6 * A, n_slots=4, begin=7 * A,
             lens_out=8 * A, state_out=9 * A, status=10 * A, views=None)
    a.update(kw)
    return b.lib.ckv_pages_resize(a["lens"], a["new_lens"], a["Bz"], a["page"], a["tables"], a["row"], a["ring"], a["n_pages"], a["state"], a["slots"],
                                  a["n_slots"], a["begin"], a["lens_out"], a["state_out"], a["status"], a["views"], None)


@pytest.mark.parametrize("status,kw", [
    (1, dict(lens=None)), (1, dict(new_lens=None)), (1, dict(tables=None)), (1, dict(ring=None)), (1, dict(state=None)), (1, dict(slots=None)),
    (1, dict(begin=None)), (1, dict(lens_out=None)), (1, dict(state_out=None)), (1, dict(status=None)), (1, dict(Bz=0)), (1, dict(row=0)),
    (1, dict(n_pages=0)), (1, dict(n_slots=-1)), (1, dict(lens_out=A)), (1, dict(lens_out=2 * A + 8)), (1, dict(state_out=5 * A)),
    (6, dict(page=48)), (6, dict(page=16)), (6, dict(Bz=8193)), (6, dict(n_pages=1 << 31)), (6, dict(n_slots=1 << 31))])
def test_resize_refusals(b, status, kw):
    assert resize(b, **kw) == status


def rows(b, **kw):
    a = dict(k=A, v=2 * A, deg=None, kt=1024, kh=128, vt=2048, vh=256, dt=0, dh=0, H=8, D=128, dtype=b.BF16)
    a.update(kw)
    return b.CkvTokenRows(*a.values())


def pool(b, **kw):
    a = dict(k_codes=A, v_codes=2 * A, k_scales=3 * A, v_scales=4 * A, deg_pages=None, logdeg_pages=None)
    a.update(kw)
    return b.CkvQuantPool(*a.values())


@pytest.mark.parametrize("status,kw", [
    (1, dict(k=None)), (1, dict(v=None)), (1, dict(H=0)), (1, dict(dtype=7)), (1, dict(kt=-1024)), (1, dict(kh=-128)), (1, dict(vt=-8)), (1, dict(vh=-8)), (1, dict(dt=-1)),
    (2, dict(k=A + 8)), (2, dict(v=A + 4)), (2, dict(kt=1028)), (2, dict(kh=132)), (2, dict(vt=1028)), (2, dict(vh=132)), (6, dict(D=64)), (6, dict(H=65536))])
def test_token_rows_refusals(b, status, kw):
    r = rows(b, **kw)
    assert b.lib.ckv_pages_write(C.byref(r), 5 * A, 3, 6 * A, 7 * A, None, None, 4, 64, None) == status
    p = pool(b)
    assert b.lib.ckv_pages_quantize(C.byref(r), 5 * A, 3, C.byref(p), 4, 64, None) == status


def test_write_and_quantize_refusals(b):
    r, p = rows(b), pool(b)
    w = lambda slots=5 * A, n=3, k=6 * A, v=7 * A, n_pages=4, page=64: b.lib.ckv_pages_write(C.byref(r), slots, n, k, v, None, None, n_pages, page, None)  # noqa: E731
    assert w(slots=None) == 1 and w(n=-1) == 1 and w(k=None) == 1 and w(v=None) == 1 and w(n_pages=0) == 1
    assert w(k=6 * A + 8) == 2 and w(page=96) == 6 and w(n=1 << 31) == 6
    assert w(n_pages=1 << 22) == 6                                       # 2^22 pages x 8 heads x 64 rows pass 31 bits
    assert b.lib.ckv_pages_quantize(C.byref(r), 5 * A, 3, C.byref(p), 1 << 22, 64, None) == 6
    assert w(n=0) == 0 and w(n=0, slots=None) == 0                       # nothing to write: nothing is launched
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        for value, status in ((None, 1), (A + 8, 2)):
            bad = pool(b, **{name: value})
            assert b.lib.ckv_pages_quantize(C.byref(r), 5 * A, 3, C.byref(bad), 4, 64, None) == status
            assert b.lib.ckv_pages_dequantize(A, 3, C.byref(bad), 64, 8, 128, b.BF16, 2 * A, 3 * A, None, None, 3, None) == status
            assert b.lib.ckv_decode_attn_quantized(A, C.byref(bad), 64, 1, 8, 4, 128, b.BF16, 2 * A, 3 * A, 0.1, 10, 4 * A, 1 << 20, None) == status
    assert b.lib.ckv_pages_quantize(C.byref(r), 5 * A, 0, C.byref(p), 4, 64, None) == 0


def test_dequantize_refusals(b):
    p = pool(b)
    d = lambda table=A, n=3, page=64, H=8, D=128, dt=b.BF16, k=2 * A, v=3 * A, cap=3: b.lib.ckv_pages_dequantize(  # noqa: E731
        table, n, C.byref(p), page, H, D, dt, k, v, None, None, cap, None)
    assert d(table=None) == 1 and d(k=None) == 1 and d(v=None) == 1 and d(n=-1) == 1 and d(cap=2) == 1 and d(H=0) == 1 and d(dt=9) == 1
    assert d(page=33) == 6 and d(D=96) == 6 and d(H=65536) == 6 and d(k=2 * A + 8) == 2 and d(n=0, cap=0) == 0


def test_summarize_and_select_refusals(b):
    s = lambda views=A, Bz=2, k=2 * A, page=64, H=8, D=128, dt=b.BF16, most=4, c=3 * A, cl=4 * A: b.lib.ckv_pages_summarize(  # noqa: E731
        views, None, Bz, k, None, page, H, D, dt, most, c, cl, None)
    assert s(views=None) == 1 and s(Bz=0) == 1 and s(k=None) == 1 and s(c=None) == 1 and s(cl=None) == 1 and s(most=-1) == 1 and s(dt=5) == 1
    assert s(dt=b.F32) == 6 and s(page=31) == 6 and s(D=64) == 6 and s(Bz=65536) == 6 and s(k=2 * A + 4) == 2 and s(most=0) == 0
    s = lambda views=A, c=2 * A, page=64, Bz=2, H=8, G=4, D=128, dt=b.BF16, q=3 * A, n=1000, first=1, last=2, sel=8, out=4 * A: b.lib.ckv_pages_select(  # noqa: E731
        views, c, None, page, Bz, H, G, D, dt, q, 0.1, n, first, last, sel, out, None)
    assert s(views=None) == 1 and s(c=None) == 1 and s(q=None) == 1 and s(out=None) == 1 and s(G=0) == 1 and s(n=-1) == 1 and s(sel=0) == 1
    assert s(first=-1) == 1 and s(last=-1) == 1 and s(first=4, last=5) == 1 and s(dt=3) == 1
    assert s(dt=b.F32) == 6 and s(G=9) == 6 and s(page=100) == 6 and s(n=64 * 24576 + 1) == 6 and s(q=3 * A + 2) == 2


def test_bounds_of_launches(b):
    v = lambda n: b.lib.ckv_pages_summarize(A, None, 2, 2 * A, None, 64, 8, 128, b.BF16, n, 3 * A, 4 * A, None)  # noqa: E731
    assert v(2**31) == 6 and v(2**63 - 1) == 6 and v(0) == 0 and v(-1) == 1


def test_attention_refusals(b):
    s = lambda views=A, k=2 * A, v=3 * A, page=64, sel=4 * A, n=8, Bz=2, H=8, G=4, D=128, dt=b.BF16, q=5 * A, out=6 * A: b.lib.ckv_decode_attn_selected(  # noqa: E731
        views, k, v, None, page, sel, n, Bz, H, G, D, dt, q, out, 0.1, None)
    assert s(views=None) == 1 and s(k=None) == 1 and s(v=None) == 1 and s(sel=None) == 1 and s(n=0) == 1 and s(q=None) == 1 and s(out=None) == 1
    assert s(dt=b.F32) == 6 and s(G=9) == 6 and s(D=64) == 6 and s(page=8) == 6 and s(k=2 * A + 8) == 2 and s(out=6 * A + 8) == 2
    p = pool(b)
    need = b.decode_quantized_workspace_bytes(2, 8, 4, 128, 1000)
    assert need > 0 and b.decode_quantized_workspace_bytes(0, 8, 4, 128, 1000) == 0
    s = lambda views=A, page=64, Bz=2, H=8, G=4, D=128, dt=b.BF16, q=5 * A, out=6 * A, n=1000, ws=7 * A, nb=need: b.lib.ckv_decode_attn_quantized(  # noqa: E731
        views, C.byref(p), page, Bz, H, G, D, dt, q, out, 0.1, n, ws, nb, None)
    assert s(views=None) == 1 and s(q=None) == 1 and s(out=None) == 1 and s(Bz=0) == 1 and s(n=-1) == 1 and s(dt=4) == 1
    assert s(Bz=60000, H=60000) == 6
    big = dict(Bz=1024, H=64, n=2**20 - 31)                              # 1024 * 64 * (max_len + 32) = 2^36 + 2^16
    assert s(**big, nb=1 << 50) == 6 and s(n=2**63 - 1, nb=1 << 50) == 6
    assert 0 < b.decode_quantized_workspace_bytes(2, 8, 4, 128, 2**63 - 1) == b.decode_quantized_workspace_bytes(2, 8, 4, 128, 1 << 20)
    assert s(dt=b.F32) == 6 and s(G=9) == 6 and s(page=24) == 6 and s(ws=None) == 4 and s(nb=need - 1) == 4 and s(q=5 * A + 8) == 2


def test_binding_refuses_shapes_and_types(b):
    """Mismatched tensors are caught before a pointer is taken."""
    i64 = torch.int64
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    k = z(3, 2, 128)
    with pytest.raises(AssertionError):
        b.pages_write(z(3, dt=torch.int32), k, k, z(4, 2, 64, 128), z(4, 2, 64, 128))
    with pytest.raises(AssertionError):
        b.pages_write(z(3, dt=i64), k, k, z(4, 3, 64, 128), z(4, 3, 64, 128))
    with pytest.raises(AssertionError):
        b.pages_write(z(3, dt=i64), k, k, z(4, 2, 64, 128, dt=torch.float32), z(4, 2, 64, 128, dt=torch.float32))
    with pytest.raises(AssertionError):
        b.pages_write(z(3, dt=i64), k.transpose(0, 2), k.transpose(0, 2), z(4, 2, 64, 128), z(4, 2, 64, 128))
    with pytest.raises(AssertionError):
        b.QuantPool(z(4, 2, 64, 64, dt=torch.uint8), z(4, 2, 64, 64, dt=torch.uint8), z(4, 2, 64, 4, dt=torch.uint8), z(4, 2, 64, 8, dt=torch.uint8)).c()
    with pytest.raises(AssertionError):
        b.pages_select(z(2, 2, dt=i64), z(4, 2, 128), None, 64, 4, z(2, 4, 128), 0.1, 100, z(2, 2, 8, dt=torch.int32))
    with pytest.raises(AssertionError):
        b.pages_resize(z(2, dt=i64), z(2, dt=i64), z(2, 4, dt=torch.int32), z(9, dt=torch.int32), z(2, dt=i64), z(3, dt=i64), z(2, dt=i64), z(2, dt=i64),
                       z(2, dt=i64), z(1, dt=torch.int32), 64)
    u8 = torch.uint8
    pool = b.QuantPool(z(4, 2, 64, 64, dt=u8), z(4, 2, 64, 64, dt=u8), z(4, 2, 64, 4, dt=u8), z(4, 2, 64, 4, dt=u8))
    with pytest.raises(AssertionError):
        b.pages_quantize(z(3, dt=i64), z(3, 3, 128), z(3, 3, 128), pool)
    with pytest.raises(AssertionError):
        b.pages_dequantize(z(1, dt=torch.int32), 65, pool, z(2, 65, 128), z(2, 65, 128))
    with pytest.raises(AssertionError):
        b.decode_attn_quantized(z(1, 2, dt=i64), pool, 4, 1, z(1, 4, 128), z(1, 4, 128), 0.1, 10, z(64, dt=u8))
    with pytest.raises(AssertionError):
        b.pages_summarize(z(2, 2, dt=i64), z(4, 2, 64, 128), None, z(4, 2, 64), z(4, 2, dt=torch.float32), 1)
    with pytest.raises(AssertionError):
        b.decode_attn_selected(z(1, 2, dt=i64), z(4, 2, 64, 128), z(4, 2, 64, 128), None, z(1, 2, 3, dt=i64), 2, 4, z(1, 8, 128), z(1, 8, 128), 0.1)


def test_binding_refuses_another_device(b):
    """Tensors that are not on the current CUDA device (here: on none) never reach a launch."""
    i64, k = torch.int64, torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    pages = torch.zeros((4, 2, 64, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        b._stream_for(k)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        b.pages_write(torch.zeros(3, dtype=i64), k, k, pages, pages)
