"""The serving calls against plain implementations in 64 bits: block tables and slot maps, writes through a slot map, page
summaries, the selection of pages and the attention over it, four-bit pages and the attention that reads them, and a run
of them together.

Tolerances (half a step of a type, relative: bf16 2^-8, fp16 2^-11, fp32 2^-24)
  integers         equal.
  codes, values    equal: quantisation is comparisons and exact scalings.
  log-degrees      1e-6 relative (logf).
  mean keys        the result's rounding to bf16, and the fp32 sum's: page + 2 roundings of sum w |k| / sum w.
  attention, bf16  parity_util.check_attention's bound.
  attention, 4 bit the result's rounding to bf16; each weight's to fp16 (2^-11 relative, and twice that for the products before
                   it); weights below 2^-21 of the group's largest are multiples of 2^-31 of it, off by half of that, times a
                   level of 6 at most and a token each; scores in fp32: 2^-20 of sum |q k| scale + |bias|, as a relative error
                   of every weight, in the numerator and the denominator.
"""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import ckv_oracle as O
from paper_2506_11418_b200 import synth
import parity_util as PU

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128
SCALE = float(np.float32(1.0 / math.sqrt(D)))
I64, I32 = dict(dtype=torch.int64, device=DEV), dict(dtype=torch.int32, device=DEV)


def lib():
    from paper_2506_11418_b200 import binding
    return binding


def blocks(n, P):
    return -(-n // P)


# ---------------------------------------------------------------- block tables and slot maps

def resize_state(old, P, row, n_pages, head, seed):
    """A consistent state: every page in exactly one row or in the queue."""
    rng = np.random.default_rng(seed)
    perm = rng.permutation(n_pages).astype(np.int32)
    tables, at = np.full((len(old), row), -5, np.int32), 0
    for b, n in enumerate(old):
        k = blocks(n, P)
        tables[b, :k] = perm[at:at + k]
        at += k
    ring = np.full(n_pages, -6, np.int32)
    ring[(head + np.arange(n_pages - at)) % n_pages] = perm[at:]
    return tables, ring, [head, n_pages - at]


def resize_plain(old, new, P, tables, ring, state, n_slots):
    """One sequence after the other; None if the step cannot be done."""
    tables, ring = tables.copy(), ring.copy()
    head, count = state
    n_pages, row = len(ring), tables.shape[1]
    queue = [ring[(head + i) % n_pages] for i in range(count)]
    for b in range(len(old)):
        queue += [tables[b, i] for i in range(blocks(new[b], P), blocks(old[b], P))]
    for i, p in enumerate(queue[count:]):
        ring[(head + count + i) % n_pages] = p
    slots, begin, taken = [], [0], 0
    for b in range(len(old)):
        for i in range(blocks(old[b], P), blocks(new[b], P)):
            tables[b, i] = queue[taken]
            taken += 1
        slots += [int(tables[b, p // P]) * P + p % P for p in range(old[b], new[b])]
        begin.append(len(slots))
    return tables, ring, [(head + taken) % n_pages, len(queue) - taken], slots + [-1] * (n_slots - len(slots)), begin


def resize_call(old, new, P, tables, ring, state, n_slots, with_views=True):
    b, Bz = lib(), len(old)
    t = dict(lens=torch.tensor(old, **I64), new=torch.tensor(new, **I64), tables=torch.from_numpy(tables).to(DEV), ring=torch.from_numpy(ring).to(DEV),
             state=torch.tensor(state, **I64), slots=torch.full((n_slots,), -9, **I64), begin=torch.full((Bz + 1,), -9, **I64),
             lens_out=torch.full((Bz,), -9, **I64), state_out=torch.full((2,), -9, **I64), status=torch.full((1,), -9, **I32),
             views=torch.full((Bz, 2), -9, **I64) if with_views else None)

    def call():
        b.pages_resize(t["lens"], t["new"], t["tables"], t["ring"], t["state"], t["slots"], t["begin"], t["lens_out"], t["state_out"], t["status"], P,
                       t["views"])
    call()
    return t, call


def check_resize(old, new, P, row, n_pages, head, seed, spare=3):
    tables, ring, state = resize_state(old, P, row, n_pages, head, seed)
    n_slots = sum(max(0, n - o) for o, n in zip(old, new)) + spare
    t, call = resize_call(old, new, P, tables, ring, state, n_slots)
    want = resize_plain(old, new, P, tables, ring, state, n_slots)
    for _ in range(2):  # the same call again repeats its results
        assert t["status"].item() == 0
        for got, ref in zip((t["tables"], t["ring"], t["state_out"], t["slots"], t["begin"], t["lens_out"]), (*want, new)):
            np.testing.assert_array_equal(got.cpu().numpy(), np.asarray(ref))
        v = t["views"].cpu().numpy()
        np.testing.assert_array_equal(v[:, 0], t["tables"].data_ptr() + 4 * row * np.arange(len(old)))
        np.testing.assert_array_equal(v[:, 1], new)
        assert t["lens"].tolist() == list(old) and t["state"].tolist() == state
        call()


@pytest.mark.parametrize("old,new,P,n_pages,head", [
    ([0], [1], 32, 1, 0), ([1], [0], 32, 1, 0), ([63], [64], 64, 1, 0), ([64], [65], 64, 2, 1), ([0], [0], 64, 4, 3), ([5, 70], [5, 70], 64, 9, 8),
    ([0, 0, 0], [64, 1, 129], 64, 7, 5),                     # the queue wraps
    ([640, 0], [0, 640], 64, 10, 7),                         # every page that is taken was given in the same call
    ([640, 0, 64], [65, 500, 0], 64, 12, 11)])               # some from the queue, then given ones
def test_resize_small(old, new, P, n_pages, head):
    check_resize(old, new, P, 12, n_pages, head, seed=len(old) + P)


@pytest.mark.parametrize("Bz,P,top,seed", [(7, 32, 300, 0), (64, 64, 9000, 1), (257, 128, 2000, 2), (300, 256, 40000, 3), (1000, 32, 999, 4), (8192, 32, 70, 5)])
def test_resize_batches(Bz, P, top, seed):
    rng = np.random.default_rng(seed)
    old, new = rng.integers(0, top + 1, Bz), rng.integers(0, top + 1, Bz)
    kind = rng.integers(0, 5, Bz)
    old[kind == 0], new[kind == 1] = 0, 0
    new = np.where(kind == 2, np.minimum(old + 1, top), new)
    need = sum(blocks(int(n), P) for n in old) + sum(max(0, blocks(int(n), P) - blocks(int(o), P)) for o, n in zip(old, new))
    give = sum(max(0, blocks(int(o), P) - blocks(int(n), P)) for o, n in zip(old, new))
    n_pages = max(1, need - give // 2)                       # part of what is taken has to be given first
    check_resize(old.tolist(), new.tolist(), P, blocks(top, P) + 2, n_pages, int(rng.integers(0, n_pages)), seed, spare=int(rng.integers(0, 400)))


@pytest.mark.parametrize("status,old,new,row,n_pages,n_slots,state", [
    (1, [64, 0], [64, 65], 4, 2, 100, None), (1, [128, 0], [64, 200], 4, 2, 300, None), (2, [10, 20], [10, 257], 4, 20, 300, None),
    (3, [10, 20], [12, 21], 4, 20, 2, None), (4, [-1, 20], [10, 21], 4, 20, 40, None), (4, [10, 20], [10, -3], 4, 20, 40, None),
    (4, [257, 20], [10, 21], 4, 20, 40, None), (4, [10, 20], [11, 21], 4, 20, 40, [20, 3]), (4, [10, 20], [11, 21], 4, 20, 40, [-1, 3]),
    (4, [10, 20], [11, 21], 4, 20, 40, [0, 21]), (4, [10, 20], [0, 0], 4, 20, 40, [0, 19]), (4, [10, 20], [11, 21], 4, 20, 40, [0, -1]),
    (2, [10, 2**62], [10, 2**62], 4, 20, 40, None), (2, [10, 20], [2**62, 2**62], 4, 20, 40, None)])
def test_resize_that_cannot_be_done(status, old, new, row, n_pages, n_slots, state):
    if old[1] == 2**62:
        status = 4
    held = [min(max(n, 0), 256) for n in old]
    tables, ring, s = resize_state(held, 64, row, n_pages, 1, seed=3)
    state = state or s
    t, _ = resize_call(old, new, 64, tables, ring, state, n_slots)
    assert t["status"].item() == status
    np.testing.assert_array_equal(t["tables"].cpu().numpy(), tables)
    np.testing.assert_array_equal(t["ring"].cpu().numpy(), ring)
    assert t["state_out"].tolist() == state and t["lens_out"].tolist() == old and t["begin"].tolist() == [0, 0, 0]
    assert t["slots"].tolist() == [-1] * n_slots and t["views"][:, 1].tolist() == held  # (never more than a row holds)


# ---------------------------------------------------------------- writes through a slot map

def token_rows(n, H, dt, layout, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    if layout == "step":
        return tuple(torch.randn((n, H, D), generator=g, device=DEV).to(dt) for _ in range(2))
    if layout == "mixed":  # keys of a step, values of a slab
        return (torch.randn((n, H, D), generator=g, device=DEV).to(dt),
                torch.randn((H, n + 3, D), generator=g, device=DEV).to(dt)[:, :n].transpose(0, 1))
    if layout == "broadcast":  # one row for all heads
        return tuple(torch.randn((n, 1, D), generator=g, device=DEV).to(dt).expand(n, H, D) for _ in range(2))
    if layout == "fused":  # slices of a projection's rows
        x = torch.randn((n, 6 * H + 1, D), generator=g, device=DEV).to(dt)
        return x[:, H:2 * H], x[:, 3 * H:4 * H]
    return tuple(torch.randn((H, n + 5, D), generator=g, device=DEV).to(dt)[:, :n].transpose(0, 1) for _ in range(2))


def slot_list(n, n_pages, P, seed):
    """n distinct slots anywhere, some of them nobody's."""
    g = torch.Generator().manual_seed(seed)
    s = torch.randperm(n_pages * P, generator=g)[:n]
    for i, bad in ((1, -1), (4, -2**40), (7, n_pages * P), (10, 2**62)):
        if n > i + 3:
            s[i] = bad
    return s.to(DEV)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,H,P,layout,with_deg", [(1, 1, 32, "step", False), (17, 3, 64, "fused", True), (1500, 8, 64, "slab", True), (333, 2, 128, "fused", False),
                                                   (2000, 8, 32, "step", True), (99, 4, 64, "mixed", True), (40, 8, 32, "broadcast", False),
                                                   (1, 3, 32, "slab", True), (70, 1, 32, "fused", False)])
def test_write(dt, n, H, P, layout, with_deg):
    b = lib()
    n_pages = n // P + 4
    k, v = token_rows(n, H, dt, layout, n)
    deg = torch.randint(1, 70000, (H, n), **I32).t() if with_deg else None
    slots = slot_list(n, n_pages, P, n)
    kp, vp = (torch.randn((n_pages, H, P, D), device=DEV).to(dt) for _ in range(2))
    dp, lp = torch.full((n_pages, H, P), 77, **I32), torch.full((n_pages, H, P), 3.0, device=DEV)
    want = [x.clone() for x in (kp, vp, dp, lp)]
    ok = (slots >= 0) & (slots < n_pages * P)
    page, off = slots[ok] // P, slots[ok] % P
    dg = deg if with_deg else torch.ones((n, H), **I32)
    want[0][page, :, off], want[1][page, :, off], want[2][page, :, off] = k[ok], v[ok], dg[ok]
    want[3][page, :, off] = torch.log(dg[ok].double()).float()
    b.pages_write(slots, k, v, kp, vp, dp, lp, deg)
    for got, ref in zip((kp, vp, dp), want):
        assert torch.equal(got, ref)
    torch.testing.assert_close(lp, want[3], rtol=1e-6, atol=1e-7)
    before = kp.clone(), vp.clone()
    b.pages_write(slots[:0], k[:0], v[:0], kp, vp)                      # nothing to write
    b.pages_write(slots, k, v, kp, vp)                                  # rows alone, no degrees
    assert torch.equal(kp, before[0]) and torch.equal(vp, before[1]) and torch.equal(dp, want[2])


# ---------------------------------------------------------------- page summaries

def paged_batch(lens, H, P, seed, deg_top=7, junk=float("nan")):
    """A bf16 pool with junk wherever no sequence has tokens, degrees, and one table row per sequence."""
    need = [blocks(n, P) for n in lens]
    n_pages = sum(need) + 5
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    kp = torch.full((n_pages, H, P, D), junk, dtype=torch.bfloat16, device=DEV)
    vp = torch.full_like(kp, junk)
    dp, lp = torch.full((n_pages, H, P), -7, **I32), torch.full((n_pages, H, P), junk, device=DEV)
    tables = torch.zeros((len(lens), max(need + [1]) + 1), **I32)
    at = 0
    for i, n in enumerate(lens):
        tab = perm[at:at + need[i]].to(DEV)
        at += need[i]
        tables[i, :need[i]] = tab
        if n == 0:
            continue
        K = synth.ar1_keys(1, H, n, D, (0.7, 0.95), 0.5, seed=seed + 40 + i, dtype="bf16", device=DEV)[0]
        V = synth.normal_values(1, H, n, D, seed=seed + 40 + i, dtype="bf16", device=DEV)[0]
        deg = torch.randint(1, deg_top + 1, (H, n), device=DEV, dtype=torch.int32, generator=torch.Generator(DEV).manual_seed(seed + i))
        lib().pages_scatter(tab, n, K, V, deg, kp, vp, dp, lp)
    views = lib().paged_views([tables[i] for i in range(len(lens))], lens, DEV)
    return dict(kp=kp, vp=vp, dp=dp, lp=lp, tables=tables, views=views, lens=lens, H=H, P=P, n_pages=n_pages)


def summaries_plain(s, i, first, with_deg):
    """Mean keys [blocks, H, D], log-degrees [blocks, H] and sum w |k| / sum w of one sequence's blocks from `first` on, 64 bits."""
    n, P, out = s["lens"][i], s["P"], []
    for blk in range(first, blocks(n, P)):
        p, m = int(s["tables"][i, blk]), min(P, n - blk * P)
        K = PU.to_np64(s["kp"][p, :, :m])
        w = s["dp"][p, :, :m].cpu().numpy().astype(np.float64) if with_deg else np.ones(K.shape[:2])
        out.append(((w[..., None] * K).sum(1) / w.sum(1)[:, None], np.log(w.sum(1)), (w[..., None] * np.abs(K)).sum(1) / w.sum(1)[:, None]))
    return out


@pytest.mark.parametrize("P,H,with_deg,deg_top", [(32, 1, True, 7), (64, 8, True, 70000), (128, 2, False, 7), (256, 3, True, 1)])
def test_summaries(P, H, with_deg, deg_top):
    b = lib()
    lens = [1, P - 1, P, P + 1, 0, 1000, 5 * P + 17]
    s = paged_batch(lens, H, P, seed=P, deg_top=deg_top)
    cp, cl = torch.full((s["n_pages"], H, D), 9.0, dtype=torch.bfloat16, device=DEV), torch.full((s["n_pages"], H), 9.0, device=DEV)
    most = max(blocks(n, P) for n in lens)
    b.pages_summarize(s["views"], s["kp"], s["dp"] if with_deg else None, cp, cl, most)

    def check(cp, cl, firsts):
        touched = set()
        got_c, got_l = PU.to_np64(cp), cl.cpu().numpy()
        for i in range(len(lens)):
            for j, (c, lg, mag) in enumerate(summaries_plain(s, i, firsts[i], with_deg)):
                p = int(s["tables"][i, firsts[i] + j])
                touched.add(p)
                assert np.all(np.abs(got_c[p] - c) <= 2.0 ** -8 * np.abs(c) + (P + 2) * 2.0 ** -24 * mag)
                np.testing.assert_allclose(got_l[p], lg, rtol=1e-6, atol=1e-7)
        rest = [p for p in range(s["n_pages"]) if p not in touched]
        assert np.all(got_c[rest] == 9) and np.all(got_l[rest] == 9)    # other pages' summaries stay as they were
    check(cp, cl, [0] * len(lens))
    # from a length on: blocks before the one that holds the token stay as they were
    cp.fill_(9.0), cl.fill_(9.0)
    begin = [min(n, max(0, n - 3)) for n in lens]
    b.pages_summarize(s["views"], s["kp"], s["dp"] if with_deg else None, cp, cl, 2, torch.tensor(begin, **I64))
    check(cp, cl, [x // P for x in begin])


def test_summaries_bound_on_blocks():
    b = lib()
    s = paged_batch([640, 100], 2, 64, seed=1)
    cp, cl = torch.full((s["n_pages"], 2, D), 9.0, dtype=torch.bfloat16, device=DEV), torch.full((s["n_pages"], 2), 9.0, device=DEV)
    b.pages_summarize(s["views"], s["kp"], s["dp"], cp, cl, 3)
    done = [int(p) for p in s["tables"][0, :3]] + [int(p) for p in s["tables"][1, :2]]
    assert sorted(torch.nonzero((cl != 9).all(1))[:, 0].tolist()) == sorted(done)


# ---------------------------------------------------------------- selection

def select_plain(q, c, clog, scale, first, last, k):
    """q [G, D], c [n, D], clog [n] or None, 64 bits: the chosen blocks in ascending order."""
    n = len(c)
    with np.errstate(all="ignore"):
        s = (q @ c.T) * scale
        s = np.where(np.isnan(s).any(0), np.nan, s.max(0)) + (clog if clog is not None else 0.0)
    always = [i < first or i >= n - last for i in range(n)]
    rank = sorted(range(n), key=lambda i: (not always[i], np.isnan(s[i]), -s[i] if not np.isnan(s[i]) else 0.0, i))
    return sorted(rank[:k])


def select_case(lens, H, G, P, k, first, last, seed, with_clog=True, scale=SCALE, change=None):
    b = lib()
    need = [blocks(n, P) for n in lens]
    n_pages = sum(need) + 3
    g = torch.Generator(DEV).manual_seed(seed)
    cp = torch.randn((n_pages, H, D), generator=g, device=DEV).bfloat16()
    cl = torch.log(torch.randint(1, 300, (n_pages, H), generator=g, device=DEV).float())
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).to(DEV)
    tables = torch.zeros((len(lens), max(need + [1])), **I32)
    for i, m in enumerate(need):
        tables[i, :m] = perm[sum(need[:i]):sum(need[:i]) + m]
    q = torch.randn((len(lens), H * G, D), generator=g, device=DEV).bfloat16()
    if change:
        change(cp, cl, q, tables)
    views = b.paged_views([tables[i] for i in range(len(lens))], lens, DEV)
    out = torch.full((len(lens), H, k), -9, **I32)
    b.pages_select(views, cp, cl if with_clog else None, P, G, q, scale, max(lens), out, first, last)
    cn, ln, qn, tn = PU.to_np64(cp), cl.cpu().numpy().astype(np.float64), PU.to_np64(q), tables.cpu().numpy()
    got = out.cpu().numpy()
    for i in range(len(lens)):
        for h in range(H):
            p = tn[i, :need[i]]
            want = select_plain(qn[i, h * G:(h + 1) * G], cn[p, h], ln[p, h] if with_clog else None, scale, first, last, k)
            assert got[i, h].tolist() == want + [-1] * (k - len(want)), f"sequence {i}, head {h}"


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_select_group_sizes(G):
    select_case([1, 5000, 64 * 33, 64 * 33 + 1, 0, 9999], 2, G, 64, 33, 1, 2, seed=G)


@pytest.mark.parametrize("lens,H,P,k,first,last", [
    ([131072], 8, 64, 64, 1, 2),                              # clusters of eight CTAs
    ([131072 - 31], 2, 32, 500, 0, 1),                        # 4095 blocks
    ([3000 + 997 * i % 9000 for i in range(20)], 7, 64, 16, 2, 3),   # clusters of two
    ([100 + 1297 * i % 9000 for i in range(50)], 8, 128, 9, 0, 0),   # one CTA per pair
    ([4096], 1, 64, 1, 0, 0), ([4096], 1, 64, 63, 31, 32), ([4096], 3, 64, 64, 0, 0), ([4097], 3, 64, 64, 3, 0), ([65 * 256], 1, 256, 2, 1, 1),
    ([8192 * 32 - 31, 8193 * 32 - 31, 8191 * 32, 40], 1, 32, 200, 1, 1),   # on both sides of 8192 blocks
    ([24576 * 32], 1, 32, 1000, 1, 1)])                       # the largest number of blocks
def test_select_shapes(lens, H, P, k, first, last):
    select_case(lens, H, 4, P, k, first, last, seed=k)


def test_select_ties_go_to_the_first_block():
    def same(cp, cl, q, tables):
        cp[:] = cp[:1]
        cl[:] = 0.5
    select_case([64 * 100, 64 * 700], 2, 4, 64, 20, 1, 2, seed=1, change=same)

    def few(cp, cl, q, tables):                               # five different summaries, each many times
        p = torch.arange(cp.shape[0], device=DEV) % 5
        cp[:], cl[:] = cp[p], cl[p]
    select_case([64 * 100, 64 * 700], 2, 4, 64, 30, 0, 1, seed=2, change=few)

    def zeros(cp, cl, q, tables):                             # plus and minus zero are equal
        cp[:] = 0.0
        cp[::3] = -0.0
        cl[:] = 0.0
    select_case([64 * 100], 2, 4, 64, 30, 0, 1, seed=3, change=zeros)


def test_select_near_ties_are_decided_in_64_bits():
    """Scores that differ by one part in 2^40: invisible to 32 bits, and every block's neighbour in rank is that near."""
    def near(cp, cl, q, tables):
        cp[:], cl[:], q[:] = 0.0, 0.0, 0.0
        q[..., 0], q[..., 1] = 1.0, 2.0 ** -40
        cp[..., 0] = 1.0
        cp[..., 1] = torch.randperm(cp.shape[0], device=DEV)[:, None].bfloat16() % 128
    select_case([64 * 120], 2, 3, 64, 40, 1, 1, seed=4, with_clog=False, change=near)


def test_select_values_that_are_not_finite():
    def odd(cp, cl, q, tables):
        cp[::7, 0, 3] = float("nan")
        cp[3::11, 1, 5] = float("inf")
        cp[5::13, 0, 9] = float("-inf")
        cl[2::17] = float("-inf")
    select_case([64 * 100, 64 * 30], 2, 4, 64, 25, 1, 2, seed=5, change=odd)
    select_case([64 * 100], 2, 2, 64, 97, 1, 2, seed=6, change=odd)

    def all_nan(cp, cl, q, tables):
        q[:] = float("nan")
    select_case([64 * 100], 2, 4, 64, 25, 1, 2, seed=7, change=all_nan)


def test_select_scores_far_from_zero_and_outliers():
    def offset(cp, cl, q, tables):                            # scores near 1000 that differ by less than a 32-bit step
        cl.add_(1000.0)
        cp.mul_(1e-4)
    select_case([64 * 700, 64 * 90], 2, 4, 64, 30, 1, 1, seed=11, change=offset)
    select_case([64 * 700], 2, 4, 64, 1, 0, 0, seed=12, change=offset)

    def outliers(cp, cl, q, tables):                          # a few pages far above and below all others
        cp[::97] *= 3000.0
        cp[5::131] *= -1e6
    select_case([64 * 1500, 64 * 700], 2, 4, 64, 40, 1, 1, seed=13, change=outliers)
    select_case([64 * 1500, 64 * 700], 2, 4, 64, 3, 0, 0, seed=14, change=outliers)

    def channel(cp, cl, q, tables):                           # one large channel: products that cancel
        cp[..., 7] = 200.0
        q[..., 7] = 50.0
        cp[..., 8] = 200.0
        q[..., 8] = -50.0
    select_case([64 * 1500, 64 * 700], 2, 4, 64, 40, 1, 1, seed=15, change=channel)


def test_select_scale_and_missing_log_degrees():
    select_case([6400, 640], 2, 4, 64, 12, 1, 1, seed=8, scale=-0.25)
    select_case([6400, 640], 2, 4, 64, 12, 1, 1, seed=9, scale=0.0)
    select_case([6400, 640], 2, 4, 64, 12, 1, 1, seed=10, with_clog=False)


# ---------------------------------------------------------------- attention over selected pages

def check_selected(s, selected, q, out, G, with_logdeg, what):
    """Eq. 3 over the concatenation of the listed blocks' tokens."""
    H, P, results = s["H"], s["P"], []
    sel, lens = selected.cpu().numpy(), s["lens"]
    for i, n in enumerate(lens):
        for h in range(H):
            pos = np.concatenate([np.arange(e * P, min((e + 1) * P, n)) for e in sel[i, h] if 0 <= e < blocks(n, P)] + [np.zeros(0, int)]).astype(int)
            got = PU.to_np64(out[i, h * G:(h + 1) * G])
            if len(pos) == 0:
                assert np.all(got == 0)
                continue
            p = s["tables"][i].cpu().numpy()[pos // P]
            at = (torch.from_numpy(p).long().to(DEV), h, torch.from_numpy(pos % P).to(DEV))
            K, V, deg = PU.to_np64(s["kp"][at])[None], PU.to_np64(s["vp"][at])[None], s["dp"][at].cpu().numpy().astype(np.int64)[None]
            r = PU.check_attention(got, PU.to_np64(q[i, h * G:(h + 1) * G]), K, V, deg if with_logdeg else None, SCALE, "bf16", f"{what}, {i}, {h}")
            results.append(r)
    PU.summarize_attention(results, what, require_sensitive=False)


def listing(lens, H, P, k, seed, order="sorted"):
    rng = np.random.default_rng(seed)
    sel = np.full((len(lens), H, k), -1, np.int32)
    for i, n in enumerate(lens):
        for h in range(H):
            m = min(k, blocks(n, P))
            e = rng.permutation(blocks(n, P))[:m]
            sel[i, h, :m] = np.sort(e) if order == "sorted" else e
    return torch.from_numpy(sel).to(DEV)


@pytest.mark.parametrize("lens,H,G,P,k,with_logdeg", [
    ([1, 63, 64, 65, 1000, 0, 4100, 2500, 96], 2, 4, 64, 8, True), ([1, 31, 32, 33, 500], 3, 1, 32, 3, False), ([5000], 1, 8, 64, 64, True),
    ([20000], 8, 4, 64, 130, True), ([9000] * 20, 8, 4, 64, 5, True), ([3000, 777], 8, 5, 128, 20, True), ([10000, 9000, 100], 4, 2, 256, 4, True),
    ([700] * 30, 2, 3, 64, 9, True), ([40000], 2, 7, 64, 600, False), ([900] * 200, 1, 6, 64, 15, True)])
def test_attention_over_selected_pages(lens, H, G, P, k, with_logdeg):
    """Lists of every length, the last block and its empty tail among them; junk behind each sequence's end is NaN."""
    b = lib()
    s = paged_batch(lens, H, P, seed=k)
    sel = listing(lens, H, P, k, seed=k)
    for i, n in enumerate(lens):  # the last, partial block in some of the lists
        if 0 < k < blocks(n, P):
            sel[i, 0, -1] = blocks(n, P) - 1
    q = synth.queries(len(lens), H * G, D, seed=11, dtype="bf16", device=DEV)
    out = torch.full_like(q, 5.0)
    b.decode_attn_selected(s["views"], s["kp"], s["vp"], s["lp"] if with_logdeg else None, sel, H, G, q, out, SCALE)
    check_selected(s, sel, q, out, G, with_logdeg, f"selected, page {P}, {k} of {[blocks(n, P) for n in lens][:9]}")


def test_attention_over_odd_lists():
    """No order, gaps, numbers past the end, blocks listed twice, an empty list: as they say."""
    b = lib()
    lens, H, G, P, k = [2000, 2000, 2000, 2000, 130, 0], 2, 4, 64, 12
    s = paged_batch(lens, H, P, seed=3)
    sel = listing(lens, H, P, k, seed=3, order="any")
    sel[0, 0, ::2] = -1
    sel[0, 1, 3] = 31                                          # the last, partial one, early in the list
    sel[1, 0, 4:9] = torch.tensor([7, 7, 7, 31, 31], **I32)
    sel[1, 1] = -1
    sel[2, 0, :6] = torch.tensor([32, 2**31 - 1, 5, -2**31, 33, 6], **I32)
    sel[2, 1] = torch.tensor([-1] * 11 + [31], **I32)
    sel[3, 0] = 40
    sel[4, 1] = torch.tensor([2, 1, 0, 2, 3, -1, -1, 0, 0, 0, -1, -1], **I32)
    q = synth.queries(len(lens), H * G, D, seed=12, dtype="bf16", device=DEV)
    out = torch.full_like(q, 5.0)
    b.decode_attn_selected(s["views"], s["kp"], s["vp"], s["lp"], sel, H, G, q, out, SCALE)
    check_selected(s, sel, q, out, G, True, "odd lists")


def test_attention_over_all_pages_is_the_paged_attention():
    b = lib()
    lens, H, G, P = [4000, 64, 1, 2222], 4, 4, 64
    s = paged_batch(lens, H, P, seed=4, junk=0.0)
    q = synth.queries(len(lens), H * G, D, seed=13, dtype="bf16", device=DEV)
    out, ref = torch.empty_like(q), torch.empty_like(q)
    sel = listing(lens, H, P, 63, seed=1)
    b.decode_attn_selected(s["views"], s["kp"], s["vp"], s["lp"], sel, H, G, q, out, SCALE)
    ws = torch.empty(b.decode_workspace_bytes(len(lens), H, G, D, 4000), dtype=torch.uint8, device=DEV)
    b.decode_attn_paged(s["views"], s["kp"], s["vp"], s["lp"], H, G, q, ref, SCALE, 4000, ws)
    assert (out.float() - ref.float()).abs().max().item() <= 2 * PU.ATTN_BAR["bf16"] * 0.5
    check_selected(s, sel, q, out, G, True, "all pages")


# ---------------------------------------------------------------- four-bit pages

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize_plain(x):
    """x [..., 128] float64 (values of bf16 or fp32) -> the values that the codes stand for."""
    y = x.reshape(*x.shape[:-1], 4, 32)
    top = np.abs(y).max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        e = np.where(np.isfinite(top) & (top > 0), np.frexp(np.where(np.isfinite(top), top, 1.0))[1] - 3, -127)
        e = np.maximum(e, -127)
        m = np.minimum(np.abs(y) / 2.0 ** e, 6.0)
        order = np.array([0, 2, 4, 6, 1, 3, 5, 7])              # of two equally near levels the even code
        near = order[np.abs(m[..., None] - LEVELS[order]).argmin(-1)]
        out = np.sign(y) * LEVELS[near] * 2.0 ** e
    return np.where(np.isfinite(top), out, np.nan).reshape(x.shape)


def odd_rows(k):
    """Rows where quantisation can go wrong: zeros, one element, ties between levels, subnormals, the largest, infinities, NaN."""
    n = k.shape[0]
    lv = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 4.0, 7.96875, 0.0, -0.25, -2.5, -7.0, -0.0], device=DEV, dtype=k.dtype)
    ties = torch.cat([lv, lv]).repeat(4)
    rows = [torch.zeros(D, device=DEV, dtype=k.dtype), ties, ties * 2.0 ** 100, ties * 2.0 ** -100, ties * 2.0 ** -126, ties * 2.0 ** -130]
    one = torch.zeros(D, device=DEV, dtype=k.dtype)
    one[77] = -3.0
    big = torch.full((D,), torch.finfo(k.dtype).max, device=DEV, dtype=k.dtype)
    inf, nan = ties.clone(), ties.clone()
    inf[40], nan[100] = float("inf"), float("nan")
    rows += [one, big, inf, nan]
    for i, r in enumerate(rows):
        if 2 * i + 1 < n:
            k[2 * i] = r
            k[2 * i + 1] = -r


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,H,P,layout", [(1, 1, 32, "step"), (65, 3, 64, "fused"), (2047, 8, 64, "slab"), (300, 2, 256, "step"), (77, 4, 32, "mixed"),
                                          (3, 1, 64, "fused"), (9601, 8, 64, "slab")])
def test_quantize_and_back(dt, n, H, P, layout):
    b = lib()
    k, v = token_rows(n, H, dt, layout, n)
    if n > 20:
        odd_rows(k)
        odd_rows(v)
    deg = torch.randint(1, 70000, (H, n), **I32).t()
    n_pages = blocks(n, P) + 3
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(n)).to(torch.int32).to(DEV)
    pos = torch.arange(n, device=DEV)
    slots = table.long()[pos // P] * P + pos % P
    pool = b.QuantPool.empty(n_pages, H, P)
    for x in (pool.k_codes, pool.v_codes, pool.k_scales, pool.v_scales):
        x.fill_(0x5a)
    pool.deg_pages.fill_(77)
    b.pages_quantize(slots, k, v, pool, deg)
    for out_dt in (dt, torch.float32):
        ko, vo = (torch.full((H, n + 2, D), 7.0, dtype=out_dt, device=DEV) for _ in range(2))
        do, lo = torch.full((H, n + 2), -3, **I32), torch.full((H, n + 2), -3.0, device=DEV)
        b.pages_dequantize(table, n, pool, ko, vo, do, lo)
        for got, src in ((ko, k), (vo, v)):
            np.testing.assert_array_equal(PU.to_np64(got[:, :n]), quantize_plain(PU.to_np64(src.transpose(0, 1))))
            assert torch.all(got[:, n:] == 7)
        assert torch.equal(do[:, :n], deg.t()) and torch.all(do[:, n:] == -3)
        torch.testing.assert_close(lo[:, :n], torch.log(deg.t().double()).float(), rtol=1e-6, atol=1e-7)
    # rows that no slot names are as they were
    mine = torch.zeros(n_pages * P, dtype=torch.bool, device=DEV)
    mine[slots] = True
    left = ~mine.view(n_pages, 1, P).expand(-1, H, -1)
    for x in (pool.k_codes, pool.v_codes, pool.k_scales, pool.v_scales):
        assert torch.all(x[left] == 0x5a)
    assert torch.all(pool.deg_pages[left] == 77)


def test_quantize_skips_slots_that_are_nobodys():
    b = lib()
    k, v = token_rows(40, 2, torch.bfloat16, "step", 1)
    slots = slot_list(40, 3, 32, 2)
    pool = b.QuantPool.empty(3, 2, 32)
    b.pages_quantize(slots, k, v, pool)
    ok = (slots >= 0) & (slots < 96)
    written = pool.deg_pages.transpose(1, 2).reshape(96, 2)
    assert torch.all(written[slots[ok]] == 1) and int(written.sum()) == 2 * int(ok.sum())
    assert torch.all(pool.logdeg_pages == 0)


def quant_batch(lens, H, P, seed, k_scale=1.0, v_change=None, deg_top=7):
    """Sequences in a four-bit pool whose other rows hold junk with NaN scales, and their values in 64 bits."""
    b = lib()
    need = [blocks(n, P) for n in lens]
    n_pages = sum(need) + 4
    g = torch.Generator(DEV).manual_seed(seed)
    pool = b.QuantPool.empty(n_pages, H, P)
    for x in (pool.k_codes, pool.v_codes):
        x.copy_(torch.randint(0, 256, x.shape, generator=g, device=DEV, dtype=torch.uint8))
    for x in (pool.k_scales, pool.v_scales):
        x.fill_(255)
    pool.logdeg_pages.fill_(float("nan"))
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    tables, seqs, at = torch.zeros((len(lens), max(need + [1])), **I32), [], 0
    for i, n in enumerate(lens):
        tables[i, :need[i]] = perm[at:at + need[i]].to(DEV)
        at += need[i]
        if n == 0:
            seqs.append(None)
            continue
        K = synth.ar1_keys(1, H, n, D, (0.7, 0.95), 0.5, seed=seed + i, dtype="f32", device=DEV)[0] * k_scale
        V = synth.normal_values(1, H, n, D, seed=seed + i, dtype="f32", device=DEV)[0]
        if v_change:
            v_change(V)
        deg = torch.randint(1, deg_top + 1, (H, n), generator=g, device=DEV, dtype=torch.int32)
        pos = torch.arange(n, device=DEV)
        slots = tables[i].long()[pos // P] * P + pos % P
        b.pages_quantize(slots, K.transpose(0, 1), V.transpose(0, 1), pool, deg.t())
        seqs.append((quantize_plain(PU.to_np64(K)), quantize_plain(PU.to_np64(V)), deg.cpu().numpy().astype(np.int64)))
    views = b.paged_views([tables[i] for i in range(len(lens))], lens, DEV)
    return pool, views, seqs, tables


def quant_attention(lens, H, G, P, seed, with_logdeg=True, q_change=None, scale=SCALE, max_len=None, **kw):
    b = lib()
    pool, views, seqs, _ = quant_batch(lens, H, P, seed, **kw)
    if not with_logdeg:
        pool.logdeg_pages = None
    q = synth.queries(len(lens), H * G, D, seed=seed + 5, dtype="bf16", device=DEV)
    if q_change:
        q_change(q)
    out = torch.full_like(q, 5.0)
    max_len = max_len or max(lens)
    ws = torch.empty(b.decode_quantized_workspace_bytes(len(lens), H, G, D, max_len), dtype=torch.uint8, device=DEV)
    b.decode_attn_quantized(views, pool, H, G, q, out, scale, max_len, ws)
    worst = 0.0
    for i, n in enumerate(lens):
        got = PU.to_np64(out[i])
        if n == 0:
            assert np.all(got == 0)
            continue
        K, V, deg = seqs[i]
        qn = PU.to_np64(q[i]).reshape(H, G, D)
        bias = np.log(deg) if with_logdeg else np.zeros(deg.shape)
        s = np.einsum("hgd,hnd->hgn", qn, K) * scale + bias[:, None]
        err_s = 2.0 ** -20 * (np.einsum("hgd,hnd->hgn", np.abs(qn), np.abs(K)) * abs(scale) + np.abs(bias)[:, None])
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        ref = np.einsum("hgn,hnd->hgd", w, V)
        # every weight: twice half an fp16 step, its score's error, and what lies below 2^-21 of the group's largest weight
        # (a group's largest level is 4 or 6, so its unit is scale_v / 4, and 6 levels times 2^-32 are 1.5 x 2^-32 of w scale_v)
        rel = 2.0 ** -10 + 2 * err_s.max(-1, keepdims=True)
        scale_v = 2.0 ** np.floor(np.log2(np.maximum(np.abs(V).reshape(H, n, 4, 32).max(-1), 2.0 ** -120)))
        floor = 1.5 * 2.0 ** -32 * n * (w[..., None] * scale_v[:, None]).max(2)
        bound = 2.0 ** -8 * np.abs(ref) + rel * np.einsum("hgn,hnd->hgd", w, np.abs(V)) + np.repeat(floor, 32, -1)
        err = np.abs(got.reshape(H, G, D) - ref)
        assert np.all(err <= bound), f"sequence {i} (len {n}): {np.max(err / bound):.2f} x the bound"
        worst = max(worst, float(np.max(err / bound)))
    print(f"[quantized attention] lens {lens[:8]}, H {H}, G {G}, page {P}: worst error {worst:.2f} of the bound")


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_quantized_attention_group_sizes(G):
    quant_attention([1, 63, 64, 65, 1000, 0, 31, 32, 33], 2, G, 64, seed=G)


@pytest.mark.parametrize("lens,H,G,P,with_logdeg", [
    ([20000], 8, 4, 64, True), ([9000, 8200, 2, 0], 2, 8, 32, True), ([777] * 20, 8, 4, 128, True), ([5000 - 97 * i for i in range(40)], 8, 2, 256, False),
    ([16416], 1, 1, 64, True), ([1], 1, 1, 32, False), ([300 + 13 * i for i in range(90)], 1, 4, 64, True), ([40000, 5, 12345], 8, 4, 64, True),
    ([50001], 1, 4, 64, True), ([33, 66001], 1, 8, 32, True), ([70000], 4, 3, 64, False),   # shares of more than one tile, many partials per row
    ([2000 + 31 * i for i in range(8)], 8, 4, 64, True), ([600 + 37 * i for i in range(16)], 8, 4, 64, True)])   # 16 and 8 combining warps
def test_quantized_attention_shapes(lens, H, G, P, with_logdeg):
    """Batches on both sides of the launch choice (one cluster per pair, or splits joined by a second kernel)."""
    quant_attention(lens, H, G, P, seed=len(lens), with_logdeg=with_logdeg)


def test_quantized_attention_longer_bound_than_lengths():
    quant_attention([100, 1], 8, 4, 64, seed=3, max_len=50000)
    quant_attention([100, 1] * 50, 8, 4, 64, seed=3, max_len=50000)


@pytest.mark.parametrize("Bz", [1, 12])
def test_quantized_attention_scales_far_apart(Bz):
    """Values whose groups differ by up to 2^60 between tokens: the tokens that matter must not be lost to fp16's range,
    be their scale the largest or the smallest of the sequence."""
    def wide(V):
        n = V.shape[1]
        e = torch.randint(-30, 31, (V.shape[0], n, 4, 1), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).float()
        V.copy_((V.view(V.shape[0], n, 4, 32) * torch.exp2(e)).view(V.shape))
    quant_attention([2000, 37] * Bz, 8, 4, 64, seed=21, v_change=wide)

    def rising(V):  # later tokens far larger, then far smaller
        n = V.shape[1]
        V *= torch.exp2(torch.linspace(-40, 40, n, device=DEV))[None, :, None]
    quant_attention([2000, 37] * Bz, 8, 4, 64, seed=22, v_change=rising)
    quant_attention([2000, 37] * Bz, 8, 4, 64, seed=23, v_change=lambda V: (rising(V), V.copy_(V.flip(1))))
    quant_attention([500] * Bz, 8, 4, 64, seed=24, v_change=lambda V: V.mul_(2.0 ** -100))
    quant_attention([500] * Bz, 8, 4, 64, seed=25, v_change=lambda V: V[:, ::2].zero_())


def test_quantized_attention_queries_far_apart():
    """Query rows of very different size in one group, rows of zeros, sharp softmax, keys large or small."""
    def change(q):
        q[:, 0] *= 2.0 ** 30
        q[:, 1] *= 2.0 ** -30
        q[:, 2] = 0.0
        q[:, 3] *= 8.0
    def small(q):
        change(q)
        q[:, 0] *= 2.0 ** -58
    quant_attention([900, 64], 2, 4, 64, seed=31, q_change=small)
    quant_attention([900, 64], 2, 4, 64, seed=32, q_change=lambda q: q.mul_(2.0 ** 40), k_scale=2.0 ** -40)
    quant_attention([900, 64], 2, 4, 64, seed=33, q_change=lambda q: q.mul_(2.0 ** -100), k_scale=2.0 ** 100)
    quant_attention([900, 64], 2, 4, 64, seed=34, scale=0.0)
    quant_attention([900, 64], 2, 4, 64, seed=35, scale=-0.25)


def test_quantized_attention_nan_group_is_seen():
    """A key or value group that was not finite makes the heads that read it NaN, and no other sequence or head."""
    b = lib()
    lens, H, G, P = [200, 200, 200], 2, 4, 64
    pool, views, seqs, tables = quant_batch(lens, H, P, seed=41)
    q = synth.queries(3, H * G, D, seed=1, dtype="bf16", device=DEV)
    pool.v_scales[tables[1, 1].item(), 0, 5, 2] = 255
    out = torch.empty_like(q)
    ws = torch.empty(b.decode_quantized_workspace_bytes(3, H, G, D, 200), dtype=torch.uint8, device=DEV)
    b.decode_attn_quantized(views, pool, H, G, q, out, SCALE, 200, ws)
    bad = torch.isnan(out)
    assert torch.all(bad[1, :G, 64:96]) and int(bad.sum()) == G * 32
    pool.k_scales[tables[2, 0].item(), 1, 63, 0] = 255
    b.decode_attn_quantized(views, pool, H, G, q, out, SCALE, 200, ws)
    bad = torch.isnan(out)
    assert torch.all(bad[2, G:]) and int(bad.sum()) == G * 32 + G * D


# ---------------------------------------------------------------- together

class Serving:
    """A batch that is served step by step: lengths on the device, tables and free pages from pages_resize, new tokens
    written through the slot map, summaries of what changed, attention over selected pages, and the same cache in four bits."""

    def __init__(self, Bz, H, G, P, n_pages, row, seed):
        b = lib()
        self.b, self.Bz, self.H, self.G, self.P = b, Bz, H, G, P
        self.lens = [torch.zeros(Bz, **I64), torch.zeros(Bz, **I64)]
        self.state = [torch.tensor([0, n_pages], **I64), torch.zeros(2, **I64)]
        self.now = 0
        self.tables, self.ring = torch.zeros((Bz, row), **I32), torch.arange(n_pages, **I32)
        self.begin, self.status, self.views = torch.zeros(Bz + 1, **I64), torch.zeros(1, **I32), torch.zeros((Bz, 2), **I64)
        self.kp, self.vp = (torch.full((n_pages, H, P, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        self.dp, self.lp = torch.zeros((n_pages, H, P), **I32), torch.full((n_pages, H, P), float("nan"), device=DEV)
        self.cp, self.cl = torch.zeros((n_pages, H, D), dtype=torch.bfloat16, device=DEV), torch.zeros((n_pages, H), device=DEV)
        self.quant = b.QuantPool.empty(n_pages, H, P)
        self.gen = torch.Generator(DEV).manual_seed(seed)

    def step(self, new_lens, k, v, slots, q, out, out4, selected, max_len, ws):
        b, i, o = self.b, self.now, 1 - self.now
        b.pages_resize(self.lens[i], new_lens, self.tables, self.ring, self.state[i], slots, self.begin, self.lens[o], self.state[o], self.status, self.P,
                       self.views)
        b.pages_write(slots, k, v, self.kp, self.vp, self.dp, self.lp)
        b.pages_quantize(slots, k, v, self.quant)
        b.pages_summarize(self.views, self.kp, self.dp, self.cp, self.cl, -(-max_len // self.P), self.lens[i])
        b.pages_select(self.views, self.cp, self.cl, self.P, self.G, q, SCALE, max_len, selected, 1, 1)
        b.decode_attn_selected(self.views, self.kp, self.vp, self.lp, selected, self.H, self.G, q, out, SCALE)
        b.decode_attn_quantized(self.views, self.quant, self.H, self.G, q, out4, SCALE, max_len, ws)
        self.now = o


class Mirror:
    """The same sequences as plain lists of rows on the host."""

    def __init__(self, Bz):
        self.k, self.v = [None] * Bz, [None] * Bz

    def step(self, old, new, k, v):
        at = 0
        for b, (o, n) in enumerate(zip(old, new)):
            m = max(0, n - o)
            if self.k[b] is None:
                self.k[b], self.v[b] = k[:0], v[:0]
            self.k[b] = torch.cat([self.k[b][:min(o, n)], k[at:at + m]])
            self.v[b] = torch.cat([self.v[b][:min(o, n)], v[at:at + m]])
            at += m

    def check(self, s, q, out, out4, selected, what):
        sel, G, P = selected.cpu().numpy(), s.G, s.P
        for b in range(s.Bz):
            n = self.k[b].shape[0]
            K, V = PU.to_np64(self.k[b].transpose(0, 1)), PU.to_np64(self.v[b].transpose(0, 1))
            for h in range(s.H):
                rows, qn = slice(h * G, (h + 1) * G), PU.to_np64(q[b, h * G:(h + 1) * G])
                if n == 0:
                    assert torch.all(out[b, rows] == 0) and torch.all(out4[b, rows] == 0) and np.all(sel[b, h] == -1)
                    continue
                c = np.stack([O.bf16_round(K[h, i:i + P].mean(0)) for i in range(0, n, P)])
                lg = np.log([min(P, n - i) for i in range(0, n, P)])
                score = (qn @ c.T * SCALE).max(0) + lg
                mine = [e for e in sel[b, h] if e >= 0]
                assert len(mine) == min(sel.shape[2], blocks(n, P)) and mine == sorted(set(mine)) and 0 in mine and blocks(n, P) - 1 in mine
                # means may differ in their last bit: a chosen block is at most that much worse than one that was left out
                other = [e for e in range(blocks(n, P)) if e not in mine]
                free = [e for e in mine if e not in (0, blocks(n, P) - 1)]
                if other and free:
                    slack = 2 * 2.0 ** -7 * np.abs(qn).sum(1).max() * np.abs(c).max() * SCALE
                    assert min(score[free]) >= max(score[other]) - slack
                pos = np.concatenate([np.arange(e * P, min(n, (e + 1) * P)) for e in mine])
                PU.check_attention(PU.to_np64(out[b, rows]), qn, K[h:h + 1, pos], V[h:h + 1, pos], None, SCALE, "bf16", f"{what}, {b}, {h}")
                K4, V4 = quantize_plain(K[h:h + 1]), quantize_plain(V[h:h + 1])
                PU.check_attention(PU.to_np64(out4[b, rows]), qn, K4, V4, None, SCALE, "bf16", f"{what}, four bits, {b}, {h}")


STEPS = [[300, 0, 64, 129, 1000], [301, 1, 65, 130, 1001], [302, 700, 0, 131, 250], [0, 701, 512, 132, 251], [900, 702, 513, 0, 252], [901, 703, 514, 1, 0]]


def buffers(s, total, k_sel, max_len):
    b = s.b
    q = torch.randn((s.Bz, s.H * s.G, D), generator=s.gen, device=DEV).bfloat16()
    k, v = (torch.randn((total, s.H, D), generator=s.gen, device=DEV).bfloat16() for _ in range(2))
    ws = torch.empty(b.decode_quantized_workspace_bytes(s.Bz, s.H, s.G, D, max_len), dtype=torch.uint8, device=DEV)
    return (k, v, torch.full((total,), -9, **I64), q, torch.full_like(q, 5.0), torch.full_like(q, 5.0), torch.full((s.Bz, s.H, k_sel), -9, **I32), max_len, ws)


@pytest.mark.parametrize("P,G", [(32, 4), (64, 8)])
def test_serving_steps(P, G):
    """Prompts, single tokens, sequences that shrink (compressed), finish and start again, in one tight pool."""
    s, m = Serving(5, 2, G, P, n_pages=2 * sum(blocks(n, P) for n in STEPS[0]), row=blocks(1100, P), seed=1), Mirror(5)
    old = [0] * 5
    for i, new in enumerate(STEPS):
        args = buffers(s, sum(max(0, n - o) for o, n in zip(old, new)) + 2 * (i % 2), 6, max(new))
        s.step(torch.tensor(new, **I64), *args)
        assert s.status.item() == 0
        m.step(old, new, args[0], args[1])
        m.check(s, args[3], args[4], args[5], args[6], f"step {i}")
        used = sum(blocks(n, P) for n in new)
        assert s.state[s.now][1].item() == s.ring.numel() - used        # every page is in a row or in the queue
        head, count = s.state[s.now].tolist()
        free = s.ring[(head + torch.arange(count, device=DEV)) % s.ring.numel()].tolist()
        held = [p for b, n in enumerate(new) for p in s.tables[b, :blocks(n, P)].tolist()]
        assert sorted(free + held) == list(range(s.ring.numel()))
        old = new


def test_serving_steps_replayed_from_graphs():
    """Two captured steps (lengths and queue change sides), replayed with new lengths, tokens and queries in the same buffers; run on
    a side stream."""
    P, G = 64, 4
    s, m = Serving(5, 2, G, P, n_pages=80, row=20, seed=2), Mirror(5)
    total, max_len = 2300, 1280
    args = buffers(s, total, 6, max_len)
    k, v, slots, q, out, out4, selected, _, ws = args
    new = torch.zeros(5, **I64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(new, *args)                                               # (sets launch attributes outside a capture)
        s.step(new, *args)
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                s.step(new, *args)
            graphs.append(g)
        old = [0] * 5
        for i, want in enumerate(STEPS):
            for x in (k, v, q):
                x.copy_(torch.randn(x.shape, generator=s.gen, device=DEV))
            new.copy_(torch.tensor(want))
            graphs[i % 2].replay()
            side.synchronize()
            assert s.status.item() == 0 and s.lens[1 - i % 2].tolist() == want
            m.step(old, want, k, v)
            m.check(s, q, out, out4, selected, f"replayed step {i}")
            old = want


def test_calls_on_two_streams_do_not_interfere():
    """The same batch attended to on two streams at once, with a workspace each: bit for bit the result of one call alone."""
    b = lib()
    lens, H, G, P = [3000, 700, 64, 1] * 12, 4, 4, 64
    pool, views, _, _ = quant_batch(lens, H, P, seed=51)
    s = paged_batch(lens, H, P, seed=52)
    sel = listing(lens, H, P, 7, seed=1)
    q = synth.queries(len(lens), H * G, D, seed=2, dtype="bf16", device=DEV)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(q) for _ in range(2)] for _ in range(3)]
    wss = [torch.empty(b.decode_quantized_workspace_bytes(len(lens), H, G, D, 3000), dtype=torch.uint8, device=DEV) for _ in range(3)]
    b.decode_attn_quantized(views, pool, H, G, q, outs[2][0], SCALE, 3000, wss[2])
    b.decode_attn_selected(s["views"], s["kp"], s["vp"], s["lp"], sel, H, G, q, outs[2][1], SCALE)
    torch.cuda.synchronize()
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                b.decode_attn_quantized(views, pool, H, G, q, outs[i][0], SCALE, 3000, wss[i])
                b.decode_attn_selected(s["views"], s["kp"], s["vp"], s["lp"], sel, H, G, q, outs[i][1], SCALE)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i][0], outs[2][0]) and torch.equal(outs[i][1], outs[2][1])


def test_empty_batches():
    """Sequences without tokens: nothing is summarised, nothing selected, outputs are zeros; a step in which nothing grows."""
    b = lib()
    for Bz in (1, 40):
        lens, H, G, P = [0] * Bz, 8, 4, 64
        s = paged_batch(lens, H, P, seed=Bz)
        pool, views, _, _ = quant_batch(lens, H, P, seed=Bz)
        cp, cl = torch.full((s["n_pages"], H, D), 9.0, dtype=torch.bfloat16, device=DEV), torch.full((s["n_pages"], H), 9.0, device=DEV)
        b.pages_summarize(s["views"], s["kp"], None, cp, cl, 3)
        assert torch.all(cp == 9) and torch.all(cl == 9)
        q = synth.queries(Bz, H * G, D, seed=1, dtype="bf16", device=DEV)
        for max_len in (0, 1000):
            sel, out = torch.full((Bz, H, 4), -9, **I32), torch.full_like(q, 5.0)
            b.pages_select(s["views"], cp, cl, P, G, q, SCALE, max_len, sel)
            assert torch.all(sel == -1)
            b.decode_attn_selected(s["views"], s["kp"], s["vp"], s["lp"], sel, H, G, q, out, SCALE)
            assert torch.all(out == 0)
            out.fill_(5.0)
            ws = torch.empty(b.decode_quantized_workspace_bytes(Bz, H, G, D, max_len), dtype=torch.uint8, device=DEV)
            b.decode_attn_quantized(views, pool, H, G, q, out, SCALE, max_len, ws)
            assert torch.all(out == 0)
    check_resize([70, 5], [3, 5], 64, 4, 9, 2, seed=1, spare=0)          # no slots at all


def test_pools_past_32_bits():
    """Pools whose elements and bytes pass 2^31 and 2^32, with pages at both ends in use."""
    b = lib()
    H, G, P, n = 8, 4, 64, 64 * 40 + 9
    n_pages = 2**32 // (H * P * 64) + 700                                # four-bit codes past 2^32 bytes, keys past 2^33 elements
    ids = torch.cat([torch.arange(20), torch.arange(n_pages - 21, n_pages)]).to(torch.int32).to(DEV)[torch.randperm(41)]
    pos = torch.arange(n, device=DEV)
    slots = ids.long()[pos // P] * P + pos % P
    K = synth.ar1_keys(1, H, n, D, (0.7, 0.95), 0.5, seed=5, dtype="bf16", device=DEV)[0].transpose(0, 1).contiguous()
    V = synth.normal_values(1, H, n, D, seed=5, dtype="bf16", device=DEV)[0].transpose(0, 1).contiguous()
    deg = torch.randint(1, 8, (n, H), **I32)
    views, scale = b.paged_views([ids], [n], DEV), SCALE
    q = synth.queries(1, H * G, D, seed=6, dtype="bf16", device=DEV)
    kp, vp = (torch.empty((n_pages, H, P, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dp, lp = torch.empty((n_pages, H, P), **I32), torch.empty((n_pages, H, P), device=DEV)
    b.pages_write(slots, K, V, kp, vp, dp, lp, deg)
    s = dict(kp=kp, vp=vp, dp=dp, lp=lp, tables=ids[None], views=views, lens=[n], H=H, P=P, n_pages=n_pages)
    for blk in (0, 17, 40):
        m = min(P, n - blk * P)
        assert torch.equal(kp[ids[blk].item(), :, :m], K[blk * P:blk * P + m].transpose(0, 1))
    cp, cl = torch.empty((n_pages, H, D), dtype=torch.bfloat16, device=DEV), torch.empty((n_pages, H), device=DEV)
    b.pages_summarize(views, kp, dp, cp, cl, 41)
    got = PU.to_np64(cp[ids.long()])
    for j, (c, _, mag) in enumerate(summaries_plain(s, 0, 0, True)):
        assert np.all(np.abs(got[j] - c) <= 2.0 ** -8 * np.abs(c) + (P + 2) * 2.0 ** -24 * mag)
    sel, out = torch.full((1, H, 12), -9, **I32), torch.empty_like(q)
    b.pages_select(views, cp, cl, P, G, q, scale, n, sel, 1, 1)
    qn, cn, ln = PU.to_np64(q[0]), got, cl[ids.long()].cpu().numpy().astype(np.float64)
    for h in range(H):
        assert sel[0, h].tolist() == select_plain(qn[h * G:(h + 1) * G], cn[:, h], ln[:, h], scale, 1, 1, 12)
    b.decode_attn_selected(views, kp, vp, lp, sel, H, G, q, out, scale)
    check_selected(s, sel, q, out, G, True, "far pages")
    del kp, vp, dp, lp, cp, cl, s
    torch.cuda.empty_cache()
    pool = b.QuantPool(*(torch.empty((n_pages, H, P, w), dtype=torch.uint8, device=DEV) for w in (64, 64, 4, 4)),
                       torch.empty((n_pages, H, P), **I32), torch.empty((n_pages, H, P), device=DEV))
    b.pages_quantize(slots, K, V, pool, deg)
    ko, vo = (torch.empty((H, n, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    b.pages_dequantize(ids, n, pool, ko, vo)
    Kq, Vq = quantize_plain(PU.to_np64(K.transpose(0, 1))), quantize_plain(PU.to_np64(V.transpose(0, 1)))
    np.testing.assert_array_equal(PU.to_np64(ko), Kq)
    np.testing.assert_array_equal(PU.to_np64(vo), Vq)
    ws = torch.empty(b.decode_quantized_workspace_bytes(1, H, G, D, n), dtype=torch.uint8, device=DEV)
    b.decode_attn_quantized(views, pool, H, G, q, out, scale, n, ws)
    for h in range(H):
        rows = slice(h * G, (h + 1) * G)
        PU.check_attention(PU.to_np64(out[0, rows]), qn[rows], Kq[h:h + 1], Vq[h:h + 1], deg.t()[h:h + 1].cpu().numpy().astype(np.int64), scale,
                           "bf16", f"far four-bit pages, head {h}")


def test_first_calls_inside_a_capture():
    """In a fresh process every call's first run is inside a stream capture; replayed, the graph gives the eager results."""
    code = """
import sys
sys.path[:0] = [{tests!r}, {root!r}]
import torch
import test_gpu_serving as T
from paper_2506_11418_b200 import binding as b
lens, H, G, P = [700, 64, 1, 300], 2, 4, 64
g = torch.Generator("cuda").manual_seed(1)
n_pages = 30
k, v = (torch.randn((sum(lens), H, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
old, new = torch.zeros(4, **T.I64), torch.tensor(lens, **T.I64)
tables, ring = torch.zeros((4, 12), **T.I32), torch.arange(n_pages, **T.I32)
state, state_out, lens_out = torch.tensor([0, n_pages], **T.I64), torch.zeros(2, **T.I64), torch.zeros(4, **T.I64)
slots, begin, status, views = torch.zeros(sum(lens), **T.I64), torch.zeros(5, **T.I64), torch.ones(1, **T.I32), torch.zeros((4, 2), **T.I64)
kp, vp = (torch.zeros((n_pages, H, P, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
dp, lp = torch.zeros((n_pages, H, P), **T.I32), torch.zeros((n_pages, H, P), device="cuda")
cp, cl = torch.zeros((n_pages, H, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((n_pages, H), device="cuda")
pool = b.QuantPool.empty(n_pages, H, P)
q = torch.randn((4, H * G, 128), generator=g, device="cuda").bfloat16()
sel, o1, o2 = torch.zeros((4, H, 3), **T.I32), torch.zeros_like(q), torch.zeros_like(q)
ws = torch.zeros(b.decode_quantized_workspace_bytes(4, H, G, 128, 700), dtype=torch.uint8, device="cuda")
ko, vo = (torch.zeros((H, 700, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
def step():
    b.pages_resize(old, new, tables, ring, state, slots, begin, lens_out, state_out, status, P, views)
    b.pages_write(slots, k, v, kp, vp, dp, lp)
    b.pages_quantize(slots, k, v, pool)
    b.pages_summarize(views, kp, dp, cp, cl, 11, old)
    b.pages_select(views, cp, cl, P, G, q, 0.09, 700, sel, 1, 1)
    b.decode_attn_selected(views, kp, vp, lp, sel, H, G, q, o1, 0.09)
    b.decode_attn_quantized(views, pool, H, G, q, o2, 0.09, 700, ws)
    b.pages_dequantize(tables[0], 700, pool, ko, vo)
outs = (tables, slots, views, kp, vp, cp, cl, sel, o1, o2, ko, vo)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
first = [x.clone() for x in outs]
assert status.item() == 0 and o1.abs().sum().item() > 0 and o2.abs().sum().item() > 0
for x in (kp, vp, cp, cl, sel, o1, o2, ko, vo):
    x.zero_()
step()
torch.cuda.synchronize()
assert all(torch.equal(x, y) for x, y in zip(first, outs))
print("captured")
"""
    here = os.path.dirname(os.path.abspath(__file__))
    res = subprocess.run([sys.executable, "-c", code.format(tests=here, root=os.path.dirname(here))], capture_output=True, text=True, timeout=200)
    assert res.returncode == 0 and "captured" in res.stdout, res.stdout + res.stderr
