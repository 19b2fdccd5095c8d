"""What the bindings of the serving calls look at before a pointer reaches the library, on the host: tensors that claim to be on
the current CUDA device, and a library that only notes which call was made."""
import types

import pytest
import torch

BF16, F32, F64, I32, I64, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8


class OnDevice(torch.Tensor):
    """A host tensor that says it is on CUDA device `where`."""
    where = 0

    def get_device(self):
        return self.where


def made(*shape, dt=BF16, where=0):
    t = torch.zeros(shape, dtype=dt).as_subclass(OnDevice)
    t.where = where
    return t


@pytest.fixture
def b(monkeypatch):
    from paper_2506_11418_b200 import binding
    binding_calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: binding_calls.append(name) or 0
    monkeypatch.setattr(binding, "lib", Library())
    monkeypatch.setattr(binding, "_raw_device", lambda: 0)
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    return types.SimpleNamespace(calls=binding_calls, **{k: getattr(binding, k) for k in dir(binding) if not k.startswith("__") and k != "calls"})


def pool_tensors():
    n, H, P = 4, 2, 64
    return dict(k_codes=made(n, H, P, 64, dt=U8), v_codes=made(n, H, P, 64, dt=U8), k_scales=made(n, H, P, 4, dt=U8), v_scales=made(n, H, P, 4, dt=U8),
                deg_pages=made(n, H, P, dt=I32), logdeg_pages=made(n, H, P, dt=F32))


POOL = ("k_codes", "v_codes", "k_scales", "v_scales", "deg_pages", "logdeg_pages")


def arguments(name):
    """A call's arguments, all of them given: 3 tokens or 2 sequences, 2 KV heads, groups of 4, 4 pages of 64 tokens."""
    kv = lambda n: made(n, 2, 128)  # noqa: E731
    pages = lambda: made(4, 2, 64, 128)  # noqa: E731
    views, q = made(2, 2, dt=I64), made(2, 8, 128)
    if name == "pages_resize":
        return dict(lens=made(2, dt=I64), new_lens=made(2, dt=I64), block_tables=made(2, 5, dt=I32), ring=made(9, dt=I32), ring_state=made(2, dt=I64),
                    slots=made(3, dt=I64), slot_begin=made(3, dt=I64), lens_out=made(2, dt=I64), ring_state_out=made(2, dt=I64), status=made(1, dt=I32),
                    page_tokens=64, views=views)
    if name == "pages_write":
        return dict(slots=made(3, dt=I64), k=kv(3), v=kv(3), k_pages=pages(), v_pages=pages(), deg_pages=made(4, 2, 64, dt=I32),
                    logdeg_pages=made(4, 2, 64, dt=F32), deg=made(3, 2, dt=I32))
    if name == "pages_summarize":
        return dict(views=views, k_pages=pages(), deg_pages=made(4, 2, 64, dt=I32), c_pages=made(4, 2, 128), clog_pages=made(4, 2, dt=F32), max_blocks=2,
                    from_lens=made(2, dt=I64))
    if name == "pages_select":
        return dict(views=views, c_pages=made(4, 2, 128), clog_pages=made(4, 2, dt=F32), page_tokens=64, G=4, q=q, scale=0.1, max_len=100,
                    selected=made(2, 2, 3, dt=I32))
    if name == "decode_attn_selected":
        return dict(views=views, k_pages=pages(), v_pages=pages(), logdeg_pages=made(4, 2, 64, dt=F32), selected=made(2, 2, 3, dt=I32), H=2, G=4, q=q,
                    out=made(2, 8, 128), scale=0.1)
    if name == "pages_quantize":
        return dict(slots=made(3, dt=I64), k=kv(3), v=kv(3), deg=made(3, 2, dt=I32), **pool_tensors())
    if name == "pages_dequantize":
        return dict(block_table=made(1, dt=I32), length=60, k=made(2, 60, 128), v=made(2, 60, 128), deg=made(2, 60, dt=I32), logdeg=made(2, 60, dt=F32),
                    **pool_tensors())
    return dict(views=views, H=2, G=4, q=q, out=made(2, 8, 128), scale=0.1, max_len=100, workspace=made(1 << 16, dt=U8), **pool_tensors())


CALLS = ("pages_resize", "pages_write", "pages_summarize", "pages_select", "decode_attn_selected", "pages_quantize", "pages_dequantize",
         "decode_attn_quantized")


def call(b, name, **change):
    a = {**arguments(name), **change}
    if "k_codes" in a:
        a["pool"] = b.QuantPool(*(a.pop(x) for x in POOL))
    getattr(b, name)(**a)


def refused(b, name, error=AssertionError, **change):
    with pytest.raises(error):
        call(b, name, **change)
    assert b.calls == []


@pytest.mark.parametrize("name", CALLS)
def test_whole_arguments_reach_the_library(b, name):
    call(b, name)
    assert b.calls == ["ckv_" + name]


@pytest.mark.parametrize("name", ["pages_write", "pages_quantize"])
def test_slots_are_64_bit_integers(b, name):
    """Another type of the same size in bytes is not a slot list: the library would read past its end, or read its bits as slots."""
    refused(b, name, slots=made(6, dt=I32))
    refused(b, name, slots=made(3, dt=F64))
    refused(b, name, slots=made(24, dt=U8))


def tensor_arguments():
    return [(name, x) for name in CALLS for x, v in arguments(name).items() if isinstance(v, torch.Tensor)]


@pytest.mark.parametrize("where", [-1, 1])
@pytest.mark.parametrize("name,x", tensor_arguments())
def test_every_tensor_is_on_the_current_device(b, name, x, where):
    """One tensor on the host or on another device among those of the current one: its pointer would be read or written by the kernel."""
    t = arguments(name)[x]
    t.where = where
    refused(b, name, ValueError, **{x: t})


@pytest.mark.parametrize("name", ["pages_write", "pages_quantize", "pages_dequantize", "decode_attn_quantized"])
def test_degrees_and_their_logarithms_are_not_exchanged(b, name):
    """Both have four bytes per row; exchanged, the attention would read integers as logarithms."""
    a = arguments(name)
    for x, y in (("deg_pages", "logdeg_pages"), ("deg", "logdeg")):
        if x in a and y in a:
            refused(b, name, **{x: a[y], y: a[x]})
        for z, dt in ((x, F32), (y, I32)):
            if z in a:
                refused(b, name, **{z: made(*a[z].shape, dt=dt)})


@pytest.mark.parametrize("name,x,dt", [("pages_summarize", "deg_pages", F32), ("pages_summarize", "clog_pages", I32), ("pages_select", "clog_pages", I32),
                                       ("decode_attn_selected", "logdeg_pages", I32)])
def test_degrees_are_integers_and_logarithms_fp32(b, name, x, dt):
    refused(b, name, **{x: made(*arguments(name)[x].shape, dt=dt)})


@pytest.mark.parametrize("dt,wrong", [(I64, F64), (I32, F32)])
@pytest.mark.parametrize("name,x", tensor_arguments())
def test_lengths_counts_and_views_are_integers(b, name, x, dt, wrong):
    """Floats of the same size would be read as bits."""
    t = arguments(name)[x]
    if t.dtype is dt:
        refused(b, name, **{x: made(*t.shape, dt=wrong)})


@pytest.mark.parametrize("name,x", [(n, x) for n, x in tensor_arguments() if x in ("lens", "new_lens", "lens_out", "from_lens", "views", "ring_state", "ring_state_out")])
def test_lengths_of_half_the_width_are_refused(b, name, x):
    t = arguments(name)[x]
    refused(b, name, **{x: made(t.shape[0], 2 * (t.numel() // t.shape[0]), dt=I32)})


def test_degrees_kept_as_logarithms_alone_are_not_returned_as_ones():
    """The library itself, on the host: the refusal comes before a launch."""
    import ctypes as C

    from paper_2506_11418_b200 import binding as lib
    A = 0x10000  # sixteen-byte aligned, never read

    def dequantize(deg, logdeg, deg_pages, logdeg_pages, n=0):
        p = lib.CkvQuantPool(A, 2 * A, 3 * A, 4 * A, deg_pages, logdeg_pages)
        return lib.lib.ckv_pages_dequantize(5 * A, n, C.byref(p), 64, 8, 128, lib.BF16, 6 * A, 7 * A, deg, logdeg, 3, None)
    assert dequantize(8 * A, None, None, 9 * A, n=3) == 1 and dequantize(8 * A, 10 * A, None, 9 * A, n=3) == 1 and dequantize(8 * A, None, None, 9 * A) == 1
    assert dequantize(None, 8 * A, None, 9 * A) == 0 and dequantize(8 * A, 10 * A, 9 * A, None) == 0 and dequantize(8 * A, 10 * A, None, None) == 0
