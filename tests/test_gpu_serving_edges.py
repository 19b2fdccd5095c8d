"""The serving calls where a step changes what the calls before it left behind, and at sizes where a launch changes form.
Tolerances as in test_gpu_serving.py."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import parity_util as PU
from paper_2506_11418_b200 import synth
from test_gpu_serving import (D, DEV, I32, I64, SCALE, blocks, lib, paged_batch, quant_attention, quant_batch, select_case, select_plain,
                              summaries_plain)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- summaries of sequences that shrink

@pytest.mark.parametrize("P,H", [(32, 3), (64, 8)])
@pytest.mark.parametrize("bound", ["tight", "loose"])
def test_summaries_of_sequences_that_shrink(P, H, bound):
    """The last block that is left loses the tokens that were dropped, and the selection scores it without them, though it is not
    always chosen.  Beside them sequences that grow, stay, and start."""
    b = lib()
    old = [20 * P + 5, 20 * P + 5, 12 * P, 9 * P + 1, 30 * P, 8 * P - 1, 700, 15 * P + 3, 0, 5 * P]
    new = [11 * P + 7, 11 * P, 11 * P + 1, 9 * P, 1, 0, 701, 15 * P + 3, 40, 5 * P]
    s = paged_batch([max(o, n) for o, n in zip(old, new)], H, P, seed=P, deg_top=60)
    views = lambda lens: b.paged_views([s["tables"][i] for i in range(len(lens))], lens, DEV)  # noqa: E731
    cp, cl = torch.full((s["n_pages"], H, D), 9.0, dtype=torch.bfloat16, device=DEV), torch.full((s["n_pages"], H), 9.0, device=DEV)
    b.pages_summarize(views(old), s["kp"], s["dp"], cp, cl, max(blocks(n, P) for n in old))
    most = 2 if bound == "tight" else 40
    b.pages_summarize(views(new), s["kp"], s["dp"], cp, cl, most, torch.tensor(old, **I64))
    got_c, got_l, tables = PU.to_np64(cp), cl.cpu().numpy(), s["tables"].cpu().numpy()
    s["lens"] = new
    for i, n in enumerate(new):
        for blk, (c, lg, mag) in enumerate(summaries_plain(s, i, 0, True)):
            p = tables[i, blk]
            assert np.all(np.abs(got_c[p] - c) <= 2.0 ** -8 * np.abs(c) + (P + 2) * 2.0 ** -24 * mag), f"sequence {i}, block {blk}"
            np.testing.assert_allclose(got_l[p], lg, rtol=1e-6, atol=1e-7)
        for blk in range(blocks(n, P), blocks(old[i], P)):              # blocks that were given back: nobody's, and left alone
            assert np.all(np.isfinite(got_l[tables[i, blk]]))
    G, k = 4, 4
    q = synth.queries(len(new), H * G, D, seed=3, dtype="bf16", device=DEV)
    sel = torch.full((len(new), H, k), -9, **I32)
    b.pages_select(views(new), cp, cl, P, G, q, SCALE, max(new), sel)
    qn, got = PU.to_np64(q), sel.cpu().numpy()
    for i, n in enumerate(new):
        p = tables[i, :blocks(n, P)]
        for h in range(H):
            want = select_plain(qn[i, h * G:(h + 1) * G], got_c[p, h], got_l[p, h].astype(np.float64), SCALE, 0, 0, k) if n else []
            assert got[i, h].tolist() == want + [-1] * (k - len(want)), f"sequence {i}, head {h}"


# ---------------------------------------------------------------- degrees of four-bit pools that keep one of their two forms

@pytest.mark.parametrize("with_deg,with_logdeg", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_degrees_come_back_from_every_kind_of_pool(dt, with_deg, with_logdeg):
    """What a pool keeps of the degrees comes back, as degrees, as logarithms or both; what it does not keep is refused, not made one."""
    b = lib()
    n, H, P = 777, 3, 64
    g = torch.Generator(DEV).manual_seed(1)
    k, v = (torch.randn((n, H, D), generator=g, device=DEV).to(dt) for _ in range(2))
    deg = torch.randint(1, 70000, (n, H), generator=g, **I32)
    table = torch.randperm(blocks(n, P) + 2, generator=torch.Generator().manual_seed(2)).to(torch.int32).to(DEV)
    pos = torch.arange(n, device=DEV)
    slots = table.long()[pos // P] * P + pos % P
    pool = b.QuantPool.empty(len(table), H, P)
    pool.deg_pages, pool.logdeg_pages = pool.deg_pages if with_deg else None, pool.logdeg_pages if with_logdeg else None
    b.pages_quantize(slots, k, v, pool, deg)
    want = deg.t() if with_deg or with_logdeg else torch.ones((H, n), **I32)
    for ask_deg in (False, True):
        ko, vo = (torch.zeros((H, n + 1, D), dtype=dt, device=DEV) for _ in range(2))
        do, lo = torch.full((H, n + 1), -3, **I32) if ask_deg else None, torch.full((H, n + 1), -3.0, device=DEV)
        if ask_deg and with_logdeg and not with_deg:
            with pytest.raises(b.CkvError):
                b.pages_dequantize(table, n, pool, ko, vo, do, lo)
            assert torch.all(do == -3) and torch.all(lo == -3) and torch.all(ko == 0)
            continue
        b.pages_dequantize(table, n, pool, ko, vo, do, lo)
        torch.testing.assert_close(lo[:, :n], torch.log(want.double()).float(), rtol=1e-6, atol=1e-7)
        assert torch.all(lo[:, n:] == -3)
        if ask_deg:
            assert torch.equal(do[:, :n], want) and torch.all(do[:, n:] == -3)
        if with_logdeg and not with_deg:  # as they are stored, bit for bit
            assert torch.equal(lo[:, :n], pool.logdeg_pages.transpose(0, 1).reshape(H, -1)[:, slots])


# ---------------------------------------------------------------- batches whose sums fill the shared memory that needs no opt-in

def test_resize_of_every_batch_size_about_the_shared_memory_limit():
    """In a fresh process, where no larger batch has raised the kernel's limit before."""
    code = """
import sys
sys.path[:0] = [{tests!r}, {root!r}]
import os
import subprocess
import sys

import numpy as np
import test_gpu_serving as T
for Bz in (3400, 3412, 3413, 3414, 4076, 4077, 4078, 4090, 4094, 4095):
    rng = np.random.default_rng(Bz)
    old, new = rng.integers(0, 70, Bz), rng.integers(0, 70, Bz)
    need = sum(T.blocks(max(int(o), int(n)), 32) for o, n in zip(old, new))
    T.check_resize(old.tolist(), new.tolist(), 32, 4, need, 5, Bz)
for Bz in (4096, 8192, 4095):
    T.check_resize([1] * Bz, [2] * Bz, 32, 4, Bz, 5, Bz)
print("resized")
"""
    here = os.path.dirname(os.path.abspath(__file__))
    res = subprocess.run([sys.executable, "-c", code.format(tests=here, root=os.path.dirname(here))], capture_output=True, text=True, timeout=200)
    assert res.returncode == 0 and "resized" in res.stdout, res.stdout + res.stderr


# ---------------------------------------------------------------- selection: the path through 64 bits beyond 8192 blocks

LONG = [([24576 * 32, 9000 * 32 - 7], 64), ([8193 * 32, 16384 * 32, 40], 3000)]


@pytest.mark.parametrize("lens,k", LONG)
def test_select_equal_scores_of_very_long_sequences(lens, k):
    """All summaries equal, a few different ones, and chosen blocks that straddle a thread's run of words."""
    def same(cp, cl, q, tables):
        cp[:], cl[:] = cp[:1], 0.5
    select_case(lens, 1, 4, 32, k, 1, 2, seed=1, with_clog=True, change=same)

    def few(cp, cl, q, tables):
        p = torch.arange(cp.shape[0], device=DEV) % 5
        cp[:], cl[:] = cp[p], cl[p]
    select_case(lens, 1, 4, 32, k, 0, 1, seed=2, change=few)
    select_case(lens, 1, 4, 32, k, 2, 0, seed=3, change=few)


@pytest.mark.parametrize("lens,k", LONG)
def test_select_values_that_are_not_finite_in_very_long_sequences(lens, k):
    def odd(cp, cl, q, tables):
        cp[::7, 0, 3] = float("nan")
        cp[3::11, 0, 5] = float("inf")
        cp[5::13, 0, 9] = float("-inf")
        cl[2::17] = float("-inf")
    select_case(lens, 1, 2, 32, k, 1, 2, seed=5, change=odd)

    def nan(cp, cl, q, tables):
        q[:] = float("nan")
    select_case(lens, 1, 4, 32, k, 1, 2, seed=7, change=nan)


def test_select_products_below_the_normal_range():
    """Scores whose products are subnormal in 32 bits, brought back by the scale, next to ordinary ones through the log-degree."""
    def tiny(cp, cl, q, tables):
        cp.mul_(2.0 ** -66)
        q.mul_(2.0 ** -66)
        cl[:] = 0.0
    for scale in (2.0 ** 6, 2.0 ** 30, 2.0 ** 120, -2.0 ** 100):
        select_case([64 * 700, 64 * 100], 2, 4, 64, 30, 1, 1, seed=21, scale=scale, change=tiny)


@pytest.mark.parametrize("q_exp,c_exp", [(-75, -75), (-20, -124), (-110, -34)])
def test_select_products_that_32_bits_do_not_hold(q_exp, c_exp):
    """Products below 2^-149, zeros in 32 bits, that a large scale makes scores of: the bound on the 32-bit scores counts what they lose."""
    def tiny(cp, cl, q, tables):
        cp.mul_(2.0 ** c_exp)
        q.mul_(2.0 ** q_exp)
        cl[:] = 0.0
    for scale in (2.0 ** 120, -2.0 ** 127):
        select_case([64 * 700, 64 * 100], 2, 4, 64, 30, 1, 1, seed=22, scale=scale, change=tiny)


# ---------------------------------------------------------------- four-bit attention: NaN through the second kernel

def test_quantized_attention_nan_group_is_seen_across_shares():
    """As for a batch of one cluster per pair: a NaN scale reaches the heads that read it and no other, whatever part of the
    sequence holds it and however many partials are joined."""
    b = lib()
    lens, H, G, P = [3000, 40, 2000, 1, 777, 4000] * 6, 4, 4, 64
    pool, views, seqs, tables = quant_batch(lens, H, P, seed=61)
    q = synth.queries(len(lens), H * G, D, seed=1, dtype="bf16", device=DEV)
    ws = torch.empty(b.decode_quantized_workspace_bytes(len(lens), H, G, D, 4000), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    b.decode_attn_quantized(views, pool, H, G, q, out, SCALE, 4000, ws)
    assert torch.all(torch.isfinite(out.float()))
    want = torch.zeros((len(lens), H, G, D), dtype=torch.bool, device=DEV)
    for seq, h, pos, group in ((0, 0, 0, 0), (2, 3, 1999, 2), (3, 1, 0, 3), (5, 2, 2222, 1), (35, 3, 3999, 0)):
        pool.v_scales[tables[seq, pos // P].item(), h, pos % P, group] = 255
        want[seq, h, :, 32 * group:32 * group + 32] = True
    b.decode_attn_quantized(views, pool, H, G, q, out, SCALE, 4000, ws)
    assert torch.equal(torch.isnan(out).view_as(want), want)
    for seq, h, pos, group in ((6, 0, 2999, 0), (8, 1, 5, 3), (9, 2, 0, 1)):
        pool.k_scales[tables[seq, pos // P].item(), h, pos % P, group] = 255
        want[seq, h] = True
    b.decode_attn_quantized(views, pool, H, G, q, out, SCALE, 4000, ws)
    assert torch.equal(torch.isnan(out).view_as(want), want)


def test_quantized_attention_past_2_to_the_31_tokens():
    """A block table that names the same pages again and again: the softmax over all of them is that over the pages once, each token
    weighted by how often it is met."""
    b = lib()
    H, G, P, laps, extra = 1, 2, 1 << 15, 1 << 15, (1 << 15) + 4321
    pool, _, seqs, tables = quant_batch([2 * P], H, P, seed=71)
    n = 2 * P * laps + extra                                             # past 2^31, its last tile not a whole one
    assert n > 2 ** 31 and n % 32
    K, V, deg = seqs[0]
    table = torch.cat([tables[0].repeat(laps), tables[0]])
    views = b.paged_views([table], [n], DEV)
    q = synth.queries(1, H * G, D, seed=2, dtype="bf16", device=DEV)
    out = torch.empty_like(q)
    ws = torch.empty(b.decode_quantized_workspace_bytes(1, H, G, D, n), dtype=torch.uint8, device=DEV)
    b.decode_attn_quantized(views, pool, H, G, q, out, SCALE, n, ws)
    times = laps + (np.arange(2 * P) < extra)
    PU.check_attention(PU.to_np64(out[0]), PU.to_np64(q[0]), K, V, deg * times, SCALE, "bf16", "2^31 tokens")


@pytest.mark.parametrize("Bz", [1, 12])
def test_quantized_attention_at_the_ends_of_its_range(Bz):
    """Values up to 2^121 / len, keys up to 2^104, through one cluster per pair and through shares; log-degrees up to log 7."""
    H, G, n = 8, 4, 1000

    def largest(x, top):  # the largest magnitude becomes 0.99 top, the others follow
        x *= 0.99 * top / x.abs().max()
    quant_attention([n, 37] * Bz, H, G, 64, seed=81, v_change=lambda V: largest(V, 2.0 ** 121 / n))

    def rising(V):
        V *= torch.exp2(torch.linspace(-60, 0, V.shape[1], device=DEV))[None, :, None]
        largest(V, 2.0 ** 121 / n)
    quant_attention([n, 37] * Bz, H, G, 64, seed=82, v_change=rising, deg_top=1)
    # the keys' largest are 15 or so: within a factor of two or three of 2^104; queries that bring the scores back
    quant_attention([n, 37] * Bz, H, G, 64, seed=83, k_scale=2.0 ** 99, q_change=lambda q: q.mul_(2.0 ** -99))
