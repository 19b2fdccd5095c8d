"""Attention for chunks of new tokens, forks, compaction and copies of pages: what the library and the bindings refuse, on the host.  Dummy
pointers and tensors: every refusal comes before a launch, so no GPU is touched."""
import ctypes as C
import types

import pytest
import torch

from test_serving_bindings import BF16, F32, I32, I64, OnDevice, U8, made, pool_tensors

A = 0x100000  # sixteen-byte aligned, never read


@pytest.fixture(scope="module")
def b():
    from paper_2506_11418_b200 import binding
    return binding


def extend(b, **kw):
    a = dict(views=A, begin=2 * A, n_rows=10, k=3 * A, v=4 * A, logdeg=5 * A, n_pages=16, page=64, Bz=2, H=8, G=4, D=128, dtype=b.BF16, q=6 * A, row=4096,
             head=128, out=7 * A, scale=0.1, ws=8 * A, nb=b.extend_workspace_bytes(10, 8, 4, 128))
    a.update(kw)
    return b.lib.ckv_extend_attn_paged(*a.values(), None)


def extend_quantized(b, **kw):
    pool = dict(k_codes=A, v_codes=2 * A, k_scales=3 * A, v_scales=4 * A, deg_pages=None, logdeg_pages=5 * A)
    pool.update({k: kw.pop(k) for k in list(kw) if k in pool})
    a = dict(views=A, begin=2 * A, n_rows=10, pool=C.byref(b.CkvQuantPool(*pool.values())), n_pages=16, page=64, Bz=2, H=8, G=4, D=128, dtype=b.BF16, q=6 * A,
             row=4096, head=128, out=7 * A, scale=0.1, ws=8 * A, nb=b.extend_workspace_bytes(10, 8, 4, 128))
    a.update(kw)
    return b.lib.ckv_extend_attn_quantized(*a.values(), None)


@pytest.mark.parametrize("status,kw", [
    (1, dict(views=None)), (1, dict(begin=None)), (1, dict(q=None)), (1, dict(out=None)), (1, dict(n_rows=-1)), (1, dict(Bz=0)), (1, dict(H=0)), (1, dict(G=0)),
    (1, dict(row=-8)), (1, dict(head=-8)), (1, dict(n_pages=0)), (1, dict(dtype=9)), (1, dict(scale=float("nan"))), (1, dict(scale=float("inf"))),
    (2, dict(q=6 * A + 8)), (2, dict(out=7 * A + 8)), (2, dict(row=4100)), (2, dict(head=132)), (4, dict(ws=None)), (4, dict(nb=0)), (4, dict(ws=8 * A + 8)),
    (6, dict(dtype=0)), (6, dict(page=48)), (6, dict(page=16)), (6, dict(D=64)), (6, dict(G=9)), (6, dict(H=8193, G=1)), (6, dict(Bz=65536)),
    (6, dict(n_rows=1 << 27)), (6, dict(n_pages=1 << 22))])
def test_extend_refusals(b, status, kw):
    assert extend(b, **kw) == status
    assert extend_quantized(b, **kw) == status


def test_extend_pages_refusals(b):
    assert extend(b, k=None) == 1 and extend(b, v=None) == 1 and extend(b, k=3 * A + 8) == 2 and extend(b, v=3 * A + 8) == 2 and extend(b, logdeg=5 * A + 4) == 2
    assert extend_quantized(b, pool=None) == 1 and extend_quantized(b, logdeg_pages=5 * A + 4) == 2
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert extend_quantized(b, **{name: None}) == 1 and extend_quantized(b, **{name: A + 8}) == 2
    assert extend(b, n_rows=0) == 0 and extend_quantized(b, n_rows=0) == 0  # nothing to do: nothing is launched


def test_extend_workspace(b):
    n = b.extend_workspace_bytes
    assert n(-1, 8, 4, 128) == n(1, 0, 4, 128) == n(1, 8, 0, 128) == n(1, 8, 4, 0) == 0
    assert 0 < n(1, 8, 4, 128) < n(64, 8, 4, 128) == n(1 << 20, 8, 4, 128) < 64 << 20
    assert n(0, 8, 4, 128) > 0


def fork(b, **kw):
    a = dict(lens=A, n_in=2, parents=2 * A, keep=3 * A, n_out=3, page=64, tables=4 * A, tables_out=5 * A, stride=8, shared=6 * A, shared_out=7 * A, ring=8 * A,
             n_pages=16, state=9 * A, copies=10 * A, lens_out=11 * A, state_out=12 * A, status=13 * A, views=None, ws=14 * A, nb=b.pages_fork_workspace_bytes(16))
    a.update(kw)
    return b.lib.ckv_pages_fork(*a.values(), None)


@pytest.mark.parametrize("status,kw", [
    *[(1, {k: None}) for k in ("lens", "parents", "tables", "tables_out", "shared", "shared_out", "ring", "state", "copies", "lens_out", "state_out", "status")],
    *[(1, {k: 0}) for k in ("n_in", "n_out", "stride", "n_pages")],
    (1, dict(tables_out=4 * A + 32)), (1, dict(shared_out=6 * A + 60)), (1, dict(lens_out=A + 8)), (1, dict(lens_out=3 * A)), (1, dict(state_out=9 * A + 8)),
    (4, dict(ws=None)), (4, dict(nb=0)), (4, dict(ws=14 * A + 4)), (6, dict(page=40)), (6, dict(n_in=8193)), (6, dict(n_out=8193)), (6, dict(n_pages=1 << 31)),
    (6, dict(stride=1 << 31))])
def test_fork_refusals(b, status, kw):
    assert fork(b, **kw) == status


def compact(b, **kw):
    a = dict(lens=A, Bz=2, page=64, tables=2 * A, tables_out=3 * A, stride=8, shared=4 * A, shared_out=5 * A, ring=6 * A, n_pages=16, copies=7 * A, n_copies=5,
             state_out=8 * A, status=9 * A, views=None, ws=10 * A, nb=b.pages_compact_workspace_bytes(16))
    a.update(kw)
    return b.lib.ckv_pages_compact(*a.values(), None)


@pytest.mark.parametrize("status,kw", [
    *[(1, {k: None}) for k in ("lens", "tables", "tables_out", "shared", "shared_out", "ring", "copies", "state_out", "status")],
    *[(1, {k: 0}) for k in ("Bz", "stride", "n_pages")], (1, dict(n_copies=-1)), (1, dict(tables_out=2 * A + 32)), (1, dict(shared_out=4 * A + 60)),
    (4, dict(ws=None)), (4, dict(nb=0)), (4, dict(ws=10 * A + 4)), (6, dict(page=40)), (6, dict(Bz=8193)), (6, dict(n_pages=1 << 31)), (6, dict(n_copies=1 << 31)),
    (6, dict(stride=1 << 31))])
def test_compact_refusals(b, status, kw):
    assert compact(b, **kw) == status


def test_workspaces_of_pools(b):
    for f in (b.pages_fork_workspace_bytes, b.pages_compact_workspace_bytes):
        assert f(0) == f(-1) == f(1 << 31) == 0 and 0 < f(1) < f(1000)


@pytest.mark.parametrize("status,kw", [
    (1, dict(base=None)), (1, dict(layers=0)), (1, dict(rows=0)), (1, dict(row_bytes=0)), (1, dict(layer_bytes=-4)), (2, dict(base=A + 2)), (2, dict(row_bytes=6)),
    (2, dict(layer_bytes=6)), (1, dict(n_arrays=0)), (1, dict(H=0)), (1, dict(n=-1)), (1, dict(copies=None)), (1, dict(n_pages=0)), (6, dict(n=1 << 31)),
    (6, dict(n_pages=1 << 31)), (6, dict(H=65536)), (0, dict(n=0)), (0, dict(n=0, copies=None))])
def test_copy_refusals(b, status, kw):
    r = dict(base=A, layer_bytes=0, layers=1, rows=64, row_bytes=256)
    r.update({k: kw[k] for k in kw if k in r})
    a = dict(n_arrays=1, H=8, copies=2 * A, n=3, n_pages=16)
    a.update({k: kw[k] for k in kw if k in a})
    arr = (b.CkvPageArray * 1)(b.CkvPageArray(*r.values()))
    assert b.lib.ckv_pages_copy(arr, *a.values(), None) == status
    assert b.lib.ckv_pages_copy(None, *a.values(), None) == 1


# ---------------------------------------------------------------- bindings

@pytest.fixture
def noting(monkeypatch):
    """The bindings on tensors that claim to be on the current device, over a library that only notes which call was made."""
    from paper_2506_11418_b200 import binding
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    monkeypatch.setattr(binding, "lib", Library())
    monkeypatch.setattr(binding, "_raw_device", lambda: 0)
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    return types.SimpleNamespace(calls=calls, b=binding)


def arguments(name):
    """A call's arguments, all of them given: 2 sequences, 3 new rows, 2 KV heads, groups of 4, 4 pages of 64 tokens."""
    if name.startswith("extend"):
        a = dict(views=made(2, 2, dt=I64), q_begin=made(3, dt=I64), H=2, G=4, q=made(5, 8, 128), out=made(5, 8, 128), scale=0.1, workspace=made(1 << 16, dt=U8))
        if name == "extend_attn_paged":
            return dict(a, k_pages=made(4, 2, 64, 128), v_pages=made(4, 2, 64, 128), logdeg_pages=made(4, 2, 64, dt=F32))
        return dict(a, **pool_tensors())
    if name == "pages_copy":
        return dict(copies=made(5, 3, dt=I32), x0=made(4, 2, 64, 128), x1=made(4, 2, 64, dt=I32), x2=made(4, 2, 128))
    a = dict(lens=made(2, dt=I64), block_tables=made(2, 5, dt=I32), block_tables_out=made(2, 5, dt=I32), shared=made(9, dt=I32), shared_out=made(9, dt=I32),
             ring=made(9, dt=I32), copies=made(2, 3, dt=I32), ring_state_out=made(2, dt=I64), status=made(1, dt=I32), page_tokens=64,
             workspace=made(1 << 16, dt=U8), views=made(2, 2, dt=I64))
    if name == "pages_compact":
        return a
    return dict(a, parents=made(2, dt=I32), keep=made(2, dt=I64), lens_out=made(2, dt=I64), ring_state=made(2, dt=I64))


def call(b, name, a):
    a = dict(a)
    if name == "extend_attn_quantized":
        a["pool"] = b.QuantPool(*[a.pop(x) for x in ("k_codes", "v_codes", "k_scales", "v_scales", "deg_pages", "logdeg_pages")])
    if name == "pages_copy":
        return b.pages_copy(a["copies"], [a["x0"], a["x1"]], [a["x2"]])
    getattr(b, name)(**a)


CALLS = ("extend_attn_paged", "extend_attn_quantized", "pages_fork", "pages_compact", "pages_copy")


@pytest.mark.parametrize("name", CALLS)
def test_whole_arguments_reach_the_library(noting, name):
    call(noting.b, name, arguments(name))
    assert noting.calls[-1] == "ckv_" + name


TENSORS = [(name, x) for name in CALLS for x, t in arguments(name).items() if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("name,x", TENSORS)
@pytest.mark.parametrize("where", [-1, 1])
def test_every_tensor_is_on_the_current_device(noting, name, x, where):
    a = arguments(name)
    a[x].where = where
    with pytest.raises(ValueError):
        call(noting.b, name, a)
    assert not noting.calls


@pytest.mark.parametrize("name,x", [(n, x) for n, x in TENSORS if x not in ("workspace", "x0", "x1", "x2", "k_codes", "v_codes", "k_scales", "v_scales")])
def test_tensors_of_another_type_or_size_are_refused(noting, name, x):
    a, t = arguments(name), arguments(name)[x]
    wrong = {BF16: torch.float16, F32: I32, I32: F32, I64: torch.float64, U8: torch.int8}[t.dtype]
    with pytest.raises((AssertionError, KeyError)):
        call(noting.b, name, dict(a, **{x: made(*t.shape, dt=wrong)}))
    if x not in ("parents", "ring", "views", "copies", "lens") and name != "pages_copy":
        with pytest.raises(AssertionError):
            call(noting.b, name, dict(a, **{x: made(*t.shape[:-1], t.shape[-1] + 1, dt=t.dtype)}))
    assert not noting.calls


def test_arrays_of_another_shape_are_refused(noting):
    b, c = noting.b, made(5, 3, dt=I32)
    x = made(4, 2, 64, 128)
    for arrays, more in (([x, made(4, 2, 32, 128)], {}), ([x, made(5, 2, 64)], {}), ([x], dict(page_arrays=[made(4, 3, 128)])), ([x.transpose(0, 1)], {}),
                         ([made(2, 4, 2, 64), made(2, 5, 2, 64)], dict(stacked=True))):
        with pytest.raises(AssertionError):
            b.pages_copy(c, arrays, **more)
    with pytest.raises(AssertionError):
        b.pages_copy(made(5, 2, dt=I32), [x])
    with pytest.raises(AssertionError):
        b.pages_copy(made(5, 3, dt=I64), [x])
    b.pages_copy(c, [made(2, 4, 2, 64), made(7, 4, 2, 64, 3, dt=F32)], [made(1, 4, 2, dt=F32)], stacked=True)
    assert noting.calls == ["ckv_pages_copy"]
