"""Attention of chunks of new tokens over a paged cache, bf16 and four-bit pages, against a plain implementation in 64 bits.

Tolerance (half a step of bf16: 2^-8 relative), for an output o = sum w v with the weights' sum one:
  the result's rounding          2^-8 |o|
  the weights', to bf16          2^-8 sum w |v|
  scores in fp32                 e = 2^-20 (sum |q k| scale + |bias|), as a relative error of every weight, in the numerator and
                                 the denominator: 2 e sum w |v|  (2^-20: 128 products in 8 or more steps, the exponential's 2^-22,
                                 the arguments' rounding in base two)
  sums over n slots in fp32      (2^-25 n + 2^-27 n) sum w |v|: the weights' sum, two accumulators of n / 2 additions of half a step,
                                 and n / 16 steps of the products' (2^-23 each, truncated)
  products below 2^-126          may count as zero (the tensor cores' subnormal products): n 2^-126, since a row's largest weight is one or
                                 more and so is the sum that divides them; and the output's rounding there, 2^-134
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128
SCALE = float(np.float32(1.0 / math.sqrt(D)))
I64, I32 = dict(dtype=torch.int64, device=DEV), dict(dtype=torch.int32, device=DEV)
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
KEY_BYTE = [16 * ((d % 32) // 8) + 4 * (d // 32) + (d % 8) // 2 for d in range(D)]
VALUE_BYTE = [8 * ((d % 32) // 4) + 2 * (d // 32) + (d % 4) // 2 for d in range(D)]


def lib():
    from paper_2506_11418_b200 import binding
    return binding


def blocks(n, P):
    return -(-n // P)


class Cache:
    """A batch's pages: `lens` slots each, pages in random places; what no sequence holds is NaN in every array."""

    def __init__(self, lens, H, P, kind="bf16", with_logdeg=True, seed=0, spread=1.0):
        g = torch.Generator(DEV).manual_seed(seed)
        self.lens, self.H, self.P, self.kind = lens, H, P, kind
        need = [blocks(n, P) for n in lens]
        n_pages = sum(need) + 3
        perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((len(lens), max(max(need), 1)), 2**31 - 1, **I32)  # (entries behind a sequence's last page are no page)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = perm[at:at + k]
            at += k
        self.table, self.n_pages = table, n_pages
        shape = (n_pages, H, P)
        held = torch.zeros(shape, dtype=torch.bool, device=DEV)
        for b, n in enumerate(lens):
            for i in range(need[b]):
                held[table[b, i].long(), :, :min(P, n - i * P)] = True
        self.held = held
        logdeg = torch.log(torch.randint(1, 50, shape, generator=g, device=DEV).float())
        self.logdeg = torch.where(held, logdeg, math.nan) if with_logdeg else None
        if kind == "bf16":
            self.k, self.v = (torch.where(held[..., None], torch.randn(shape + (D,), generator=g, device=DEV) * spread, math.nan).bfloat16() for _ in range(2))
        else:
            self.codes = [torch.randint(0, 256, shape + (D // 2,), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
            self.scales = [torch.where(held[..., None], torch.randint(123, 128, shape + (D // 32,), generator=g, device=DEV), 255).to(torch.uint8) for _ in range(2)]
        self.views = torch.tensor([[table.data_ptr() + 4 * table.stride(0) * b, n] for b, n in enumerate(lens)], **I64)

    def rows(self, b, h):
        """Keys, values and biases of one sequence and head in 64 bits."""
        pos = torch.arange(self.lens[b], device=DEV)
        at = (self.table[b, pos // self.P].long(), h, pos % self.P)
        bias = self.logdeg[at].double() if self.logdeg is not None else torch.zeros(len(pos), dtype=torch.float64, device=DEV)
        if self.kind == "bf16":
            return self.k[at].double(), self.v[at].double(), bias
        lv = torch.tensor(LEVELS + [-x for x in LEVELS], dtype=torch.float64, device=DEV)
        out = []
        for c, e, byte_of in zip(self.codes, self.scales, (KEY_BYTE, VALUE_BYTE)):
            c, d = c[at][:, byte_of].long(), torch.arange(D, device=DEV)
            out.append(torch.ldexp(lv[(c >> (4 * (d % 2))) % 16], e[at].int()[:, d // 32] - 127))
        return out[0], out[1], bias

    def call(self, q_begin, G, q, out, scale, workspace):
        b = lib()
        if self.kind == "bf16":
            b.extend_attn_paged(self.views, q_begin, self.k, self.v, self.logdeg, self.H, G, q, out, scale, workspace)
        else:
            b.extend_attn_quantized(self.views, q_begin, b.QuantPool(*self.codes, *self.scales, None, self.logdeg), self.H, G, q, out, scale, workspace)


def queries(n, H, G, seed, layout="plain"):
    g = torch.Generator(DEV).manual_seed(seed + 77)
    if layout == "fused":
        return torch.randn((n, H * (G + 2), D), generator=g, device=DEV).bfloat16()[:, :H * G]
    if layout == "heads first":
        return torch.randn((H * G, n + 3, D), generator=g, device=DEV).bfloat16().transpose(0, 1)[:n]
    return torch.randn((n, H * G, D), generator=g, device=DEV).bfloat16()


def workspace(n, H, G, fill=0xff):
    return torch.full((lib().extend_workspace_bytes(n, H, G, D),), fill, dtype=torch.uint8, device=DEV)


def expected(cache, new, G, q, scale, rows=None, exact_scores=False):
    """(outputs, bound) in 64 bits, [sum new, H * G, D]; rows: only these of every sequence's new tokens; exact_scores: the scores'
    differences do not round."""
    total = sum(new)
    o = torch.zeros((total, cache.H * G, D), dtype=torch.float64, device=DEV)
    bound = torch.zeros_like(o)
    at = 0
    for b, (n, m) in enumerate(zip(cache.lens, new)):
        if m and n:
            pick = torch.arange(m, device=DEV) if rows is None else torch.tensor([r for r in rows if r < m], device=DEV)
            for h in range(cache.H):
                k, v, bias = cache.rows(b, h)
                for j in range(h * G, (h + 1) * G):
                    x = q[at + pick, j].double()
                    s, size = x @ k.T * scale + bias, (x.abs() @ k.abs().T) * abs(scale) + bias.abs()
                    hidden = torch.arange(n, device=DEV) > (n - m + pick)[:, None]
                    s = s.masked_fill(hidden, -math.inf)
                    top = s.amax(1, keepdim=True)
                    w = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
                    w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
                    e = 2.0**-20 * size.masked_fill(w == 0, 0).amax(1, keepdim=True)  # (slots without weight have no part in it)
                    e = torch.zeros_like(e) if exact_scores else e
                    v_ = torch.where(torch.isfinite(v), v, 0.0)           # (infinities and NaN where they have a weight alone)
                    o[at + pick, j] = torch.where((w > 0).double() @ (~torch.isfinite(v)).double() > 0, math.nan, w @ v_)
                    v = v_
                    bound[at + pick, j] = 2.0**-8 * (w @ v).abs() + (2.0**-8 + 2 * e + (2.0**-25 + 2.0**-27) * n) * (w @ v.abs()) + n * 2.0**-126 + 2.0**-134
        at += m
    return o, bound


def check(cache, new, G, scale=SCALE, seed=0, layout="plain", pad=2, rows=None, exact_scores=False):
    total = sum(new)
    q = queries(total + pad, cache.H, G, seed, layout)
    out = torch.full((total + pad, cache.H * G, D), 7.0, dtype=torch.bfloat16, device=DEV)
    begin = torch.tensor(np.concatenate([[0], np.cumsum(new)]), **I64)
    ws = workspace(total + pad, cache.H, G)
    cache.call(begin, G, q, out, scale, ws)
    assert lib().workspace_status(ws) == 0
    o, bound = expected(cache, new, G, q, scale, rows, exact_scores)
    assert (out[total:] == 7.0).all()                                     # rows behind the last sequence's
    got = out[:total].double()
    if rows is not None:
        at, keep = 0, []
        for m in new:
            keep += [at + r for r in rows if r < m]
            at += m
        got, o, bound = got[keep], o[keep], bound[keep]
    off = (got - o).abs()
    assert torch.isfinite(got).all()
    worst = (off / bound.clamp(min=1e-30)).max().item()
    print(f"[extend] {cache.kind} lens {cache.lens[:6]} new {new[:6]} H {cache.H} G {G} P {cache.P}: max abs err {off.max().item():.2e}, of the bound {worst:.2f}")
    assert (off <= bound).all()
    return out


KINDS = ("bf16", "quantized")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("G", range(1, 9))
def test_group_sizes(kind, G):
    check(Cache([300, 37, 129], 2, 64, kind, seed=G), [77, 37, 1], G)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("P", [32, 64, 128, 256, 1024])
@pytest.mark.parametrize("lens,new", [
    ([1], [1]), ([32], [32]), ([33], [1]), ([127, 128, 129], [127, 128, 129]), ([500], [3]), ([1000, 1, 64, 257], [65, 1, 64, 130])])
def test_shapes(kind, P, lens, new):
    check(Cache(lens, 2, P, kind, seed=P), new, 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,new,H,G", [
    ([4096], [1], 8, 4), ([4100], [17], 8, 4), ([20000], [2], 1, 8), ([5000] * 7, [1] * 7, 3, 5), ([70], [70], 8, 1), ([2000, 3000], [900, 1100], 8, 4),
    ([9000, 30, 700, 8000], [1, 30, 650, 257], 4, 7), ([40] * 300, [1] * 300, 2, 4), ([1500], [1500], 1, 3), ([64] * 40, [32] * 40, 1, 4)])
def test_how_the_work_is_shared(kind, lens, new, H, G):
    """Few rows over many slots, many rows, many short sequences: every way in which thread blocks share and join the work."""
    check(Cache(lens, H, 64, kind, seed=len(lens)), new, G)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,m,H,G,pad", [
    (5000, 4000, 8, 4, 2), (3000, 3000, 4, 8, 0), (2500, 2600, 8, 8, 1), (1200, 1184, 8, 4, 0), (9000, 1185, 8, 4, 0), (700, 600, 2, 4, 9000), (4000, 3777, 3, 7, 0),
    (20000, 1184, 8, 4, 0), (300, 300, 64, 8, 0)])
def test_one_large_chunk(kind, n, m, H, G, pad):
    """One sequence with more items than SMs (or rows for them): items are dealt whole, the rest in stretches."""
    check(Cache([n], H, 64, kind, seed=m), [m], G, pad=pad, rows=sorted({0, 1, 31, 32, 63, 64, 500, m // 2, m - 65, m - 64, m - 2, m - 1} & set(range(m))))


@pytest.mark.parametrize("kind", KINDS)
def test_sequences_without_tokens_or_slots(kind):
    """No new tokens, no slots at all, and more new tokens than slots: the first of them have nothing to attend to."""
    check(Cache([0, 100, 0, 5, 200, 3], 2, 32, kind), [0, 0, 4, 9, 50, 3], 4)
    out = check(Cache([0], 2, 32, kind), [6], 4)
    assert (out[:6] == 0).all()
    out = check(Cache([10], 1, 32, kind), [300], 4)
    assert (out[:290] == 0).all() and (out[290:300] != 0).any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", ["fused", "heads first"])
def test_strides_of_the_queries(kind, layout):
    check(Cache([700, 90], 3, 64, kind), [100, 90], 3, layout=layout)


@pytest.mark.parametrize("kind", KINDS)
def test_all_degrees_one_and_scales(kind):
    check(Cache([600, 90], 2, 64, kind, with_logdeg=False), [100, 90], 4)
    for scale in (0.0, -0.05, 1.0):
        check(Cache([600, 90], 2, 64, kind), [100, 90], 4, scale=scale)


def test_scores_far_apart():
    """Scores of hundreds, whose maximum moves all the time: rows are rescaled again and again."""
    check(Cache([3000], 2, 64, spread=8.0), [200], 4, scale=1.0)
    c = Cache([2000], 1, 64)
    pos = torch.arange(2000, device=DEV)
    c.logdeg[c.table[0, pos // 64].long(), 0, pos % 64] = pos.float() / 10      # ever larger: every tile has a new maximum
    check(c, [300], 4)
    c.logdeg[c.table[0, pos // 64].long(), 0, pos % 64] = -pos.float() / 10
    check(c, [300], 4)


@pytest.mark.parametrize("kind", KINDS)
def test_masked_by_log_degrees(kind):
    """A log-degree of minus infinity takes a slot out; a row that has no others gets zeros."""
    c = Cache([900], 2, 64, kind)
    pos = torch.arange(900, device=DEV)
    at = lambda s: (c.table[0, pos[s] // 64].long(), slice(None), pos[s] % 64)  # noqa: E731
    c.logdeg[at(slice(0, 500))] = -math.inf
    check(c, [200], 4)
    # all slots of most rows at the type's lowest or highest value, next to which the products vanish in 32 and in 64 bits: equal weights
    for far in (torch.finfo(torch.float32).min, torch.finfo(torch.float32).max):
        c.logdeg[at(slice(0, 900))] = far
        check(c, [200], 4, exact_scores=True)
    c.logdeg[at(slice(0, 899))] = torch.finfo(torch.float32).min
    check(c, [200], 4)
    c.logdeg[at(slice(0, 800))] = -math.inf
    c.logdeg[at(slice(800, 900))] = 0
    out = check(c, [200], 4)
    assert (out[:100] == 0).all()


@pytest.mark.parametrize("keys,values", [((60, 126), (127, 250)), ((0, 3), (20, 60)), ((120, 128), (2, 240)), ((127, 129), (1, 9))])
def test_scales_far_apart(keys, values):
    """Groups' powers of two over all of their range; unpacking is exact."""
    c = Cache([700], 2, 64, "quantized", seed=keys[1])
    g = torch.Generator(DEV).manual_seed(values[0])
    for x, (a, b) in zip(c.scales, (keys, values)):
        x.copy_(torch.where(c.held[..., None], torch.randint(a, b, x.shape, generator=g, device=DEV), 255))
    c.logdeg = c.logdeg.clamp(max=2.0)                                    # (sums of weights times 2^125 stay numbers)
    check(c, [90], 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,new,G", [([700], [300], 4), ([40], [40], 4), ([3000], [20], 4), ([5], [9], 4), ([90], [70], 3), ([5000], [130], 8)])
def test_values_that_are_not_finite(kind, lens, new, G):
    """Infinities and NaN in a new token's value: the tokens before it do not see them, the others do."""
    c = Cache(lens, 2, 64, kind, seed=4)
    n, m = lens[0], new[0]
    at = lambda t: (c.table[0, t // 64].long(), slice(None), t % 64)  # noqa: E731
    bad = sorted({n - 1, n - 2, max(n - m, 0) + min(m, n) // 2} & set(range(n)))
    for i, t in enumerate(bad):
        if kind == "bf16":
            c.v[at(t)[0], 0, t % 64, 5 + 40 * i] = [math.inf, math.nan, -math.inf][i]
        else:
            c.scales[1][at(t)[0], 0, t % 64, i] = 255                     # a group of NaN
    total = m + 2
    q = queries(total, 2, G, 4)
    out = torch.full((total, 2 * G, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = workspace(total, 2, G)
    c.call(torch.tensor([0, m], **I64), G, q, out, SCALE, ws)
    assert lib().workspace_status(ws) == 0
    o, bound = expected(c, new, G, q, SCALE)
    seen = torch.arange(m, device=DEV) + n - m                            # each token's last slot
    clean = seen < bad[0]
    got = out[:m].double()
    assert torch.isfinite(got[clean]).all() and ((got - o).abs() <= bound)[clean].all()
    assert torch.isfinite(got[:, G:]).all() and ((got - o).abs() <= bound)[:, G:].all()  # the other KV head's
    for i, t in enumerate(bad):                                           # who sees one has it in its columns, and nowhere else
        cols = slice(5 + 40 * i, 6 + 40 * i) if kind == "bf16" else slice(32 * i, 32 * i + 32)
        rows = seen >= t
        assert not torch.isfinite(got[rows][:, :G, cols]).any() or not rows.any()
        ok = seen < t
        assert torch.isfinite(got[ok][:, :G, cols]).all() and ((got - o).abs() <= bound)[ok][:, :G, cols].all()


def test_a_long_sequence():
    check(Cache([131072 + 77], 1, 64, seed=3), [200], 4, rows=[0, 1, 63, 64, 100, 198, 199])
    check(Cache([100000], 1, 64, "quantized", seed=3), [70], 8, rows=[0, 1, 15, 16, 69])


def test_pool_past_32_bits():
    """Pages whose offsets in bytes and elements pass 2^31 and 2^32."""
    H, P = 8, 64
    n_pages = (1 << 33) // (H * P * D * 2) + 40                            # keys of 8 GiB
    c = Cache([500], H, P, seed=5)
    far = torch.tensor([n_pages - 1, 3, n_pages - 40, n_pages // 2 + 1, n_pages // 4 + 1, 17, n_pages - 2, n_pages // 2 - 1], **I32)
    k, v = (torch.empty((n_pages, H, P, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    logdeg = torch.empty((n_pages, H, P), device=DEV)
    for x, y in ((k, c.k), (v, c.v), (logdeg, c.logdeg)):
        x[far.long()] = y[c.table[0].long()]
    c.k, c.v, c.logdeg = k, v, logdeg
    c.table[0] = far
    check(c, [130], 4)


@pytest.mark.parametrize("kind", KINDS)
def test_many_calls_one_after_the_other(kind):
    """Short items whose pieces have one step each, many times over without a pause: results repeat to the bit."""
    lens = [1 + 37 * b % 300 for b in range(90)]
    c, new = Cache(lens, 4, 64, kind), [min(n, 1 + 11 * n % 200) for n in lens]
    total = sum(new)
    q, begin, ws = queries(total, 4, 4, 1), torch.tensor(np.concatenate([[0], np.cumsum(new)]), **I64), workspace(total, 4, 4)
    outs = [torch.zeros_like(q) for _ in range(2)]
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    c.call(begin, 4, q, outs[0], SCALE, ws)
    for _ in range(300):
        c.call(begin, 4, q, outs[1], SCALE, ws)
        bad += (outs[0] != outs[1]).sum() + ws[:4].view(torch.int32)[0].abs()
    assert bad.item() == 0
