"""Sequences that share pages: forks, compaction and the copies of pages, against sequential implementations in Python (everything is
equal: whole numbers and copied bits), and a run of them together with writes and attention for chunks of new tokens."""
import math

import numpy as np
import pytest
import torch

import test_gpu_extend as X

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128
I64, I32 = X.I64, X.I32
OK, NO_PAGES, TABLE_FULL, LIST_FULL, INCONSISTENT = range(5)


def lib():
    from paper_2506_11418_b200 import binding
    return binding


def blocks(n, P):
    return -(-n // P)


class Pool:
    """Rows of a table, which pages they share, and the queue of free pages, on the host."""

    def __init__(self, lens, P, n_pages, width=None, together=1, head=0, seed=0):
        rng = np.random.default_rng(seed)
        self.P, self.n_pages, self.lens = P, n_pages, list(lens)
        need = [blocks(n, P) for n in lens]
        self.table = np.full((len(lens), width or max(max(need), 1)), -5, np.int32)
        self.shared = np.zeros(n_pages, np.int32)
        perm, at = rng.permutation(n_pages).astype(np.int32), 0
        for b, n in enumerate(need):
            first = b // together * together
            common = min(lens[b], lens[first]) // P // 2 if b > first else 0
            self.table[b, :common] = self.table[first, :common]
            self.shared[self.table[b, :common]] += 1
            self.table[b, common:n] = perm[at:at + n - common]
            at += n - common
        assert at <= n_pages
        self.ring = np.full(n_pages, -6, np.int32)
        self.ring[(head + np.arange(n_pages - at)) % n_pages] = perm[at:]
        self.state = [head, n_pages - at]

    def rows(self, b):
        return self.table[b, :blocks(self.lens[b], self.P)].tolist()


def fork_plain(pool, parents, keep):
    """The new pool and the copies; a status in place of both if it cannot be done."""
    P, n_pages = pool.P, pool.n_pages
    keep = [pool.lens[p] if k is None and p >= 0 else k for p, k in zip(parents, keep or [None] * len(parents))]
    if any(not -1 <= p < len(pool.lens) or (p >= 0 and not 0 <= k <= pool.lens[p]) for p, k in zip(parents, keep)):
        return INCONSISTENT
    keep = [0 if p < 0 else k for p, k in zip(parents, keep)]
    holders = {}
    for b in range(len(pool.lens)):
        for q in pool.rows(b):
            holders.setdefault(q, int(pool.shared[q]) + 1)
    old = sorted(holders)
    for b in range(len(pool.lens)):
        for q in pool.rows(b):
            holders[q] -= 1
    if min(holders.values(), default=0) < 0:
        return INCONSISTENT
    new = object.__new__(Pool)
    new.P, new.n_pages, new.lens, new.shared, new.ring = P, n_pages, keep, pool.shared.copy(), pool.ring.copy()
    new.table = np.full((len(parents), pool.table.shape[1]), -9, np.int32)
    for b, (p, n) in enumerate(zip(parents, keep)):
        new.table[b, :blocks(n, P)] = pool.table[p, :blocks(n, P)] if p >= 0 else 0
        for q in new.table[b, :n // P].tolist():
            holders[q] += 1
    takes, writers = [], set()
    for b, n in enumerate(keep):
        if n % P:
            q = int(new.table[b, n // P])
            if holders[q] == 0 and q not in writers:
                writers.add(q)
            else:
                takes.append((b, q, n % P))
    head, count = pool.state
    for q in old:
        left = holders[q] + (q in writers)
        new.shared[q] = max(left - 1, 0)
        if left == 0:
            new.ring[(head + count) % n_pages] = q
            count += 1
    if len(takes) > count:
        return NO_PAGES
    copies = []
    for b, q, n in takes:
        new.table[b, keep[b] // P] = new.ring[head]
        copies.append([q, int(new.ring[head]), n])
        head, count = (head + 1) % n_pages, count - 1
    new.state = [head, count]
    return new, copies


def fork_call(pool, parents, keep=None, with_views=True):
    b, n_out = lib(), len(parents)
    t = dict(lens=torch.tensor(pool.lens, **I64), parents=torch.tensor(parents, **I32), keep=None if keep is None else torch.tensor(keep, **I64),
             table=torch.from_numpy(pool.table).to(DEV), table_out=torch.full((n_out, pool.table.shape[1]), -9, **I32),
             shared=torch.from_numpy(pool.shared).to(DEV), shared_out=torch.full((pool.n_pages,), -9, **I32), ring=torch.from_numpy(pool.ring).to(DEV),
             state=torch.tensor(pool.state, **I64), copies=torch.full((n_out, 3), -9, **I32), lens_out=torch.full((n_out,), -9, **I64),
             state_out=torch.full((2,), -9, **I64), status=torch.full((1,), -9, **I32), views=torch.full((n_out, 2), -9, **I64) if with_views else None,
             workspace=torch.full((b.pages_fork_workspace_bytes(pool.n_pages),), 0xff, dtype=torch.uint8, device=DEV))

    def call():
        b.pages_fork(t["lens"], t["parents"], t["keep"], t["table"], t["table_out"], t["shared"], t["shared_out"], t["ring"], t["state"], t["copies"],
                     t["lens_out"], t["state_out"], t["status"], pool.P, t["workspace"], t["views"])
    call()
    return t, call


def check_fork(pool, parents, keep=None, twice=True):
    t, call = fork_call(pool, parents, keep)
    want = fork_plain(pool, parents, keep)
    for _ in range(2 if twice else 1):
        if isinstance(want, int):
            assert t["status"].item() == want
            assert (t["copies"] == -1).all() and t["state_out"].tolist() == pool.state and (t["shared_out"].cpu().numpy() == pool.shared).all()
            assert (t["table_out"] == -9).all() and (t["lens_out"] == -9).all() and (t["ring"].cpu().numpy() == pool.ring).all() and (t["views"] == -9).all()
        else:
            new, copies = want
            assert t["status"].item() == OK
            assert (t["table_out"].cpu().numpy() == new.table).all()      # entries behind a row's last page as they were
            assert (t["shared_out"].cpu().numpy() == new.shared).all()
            assert (t["ring"].cpu().numpy() == new.ring).all() and t["state_out"].tolist() == new.state and t["lens_out"].tolist() == new.lens
            assert t["copies"].tolist() == copies + [[-1] * 3] * (len(parents) - len(copies))
            assert t["views"].tolist() == [[t["table_out"].data_ptr() + 4 * t["table_out"].stride(0) * b, n] for b, n in enumerate(new.lens)]
        call()                                                            # the same call again gives the same
    return want


@pytest.mark.parametrize("P", [32, 64])
@pytest.mark.parametrize("lens,parents,keep", [
    ([100], [0], None), ([100], [0, 0, 0], None), ([128], [0, 0], None), ([100], [-1], None), ([0], [0, 0], None), ([1], [0, 0], None),
    ([200, 70], [1, 0], None), ([200, 70], [0, 0, 1, -1, 1], [200, 64, 70, 0, 3]), ([200], [0, 0, 0], [199, 130, 129]), ([200], [0], [0]),
    ([90, 90, 90], [2, 2, -1], None), ([300, 10, 0, 45], [3, 0, 0, 2, 1, 0], [45, 300, 256, 0, 10, 31])])
def test_fork_small(P, lens, parents, keep):
    check_fork(Pool(lens, P, 40, width=12, head=37), parents, keep)


@pytest.mark.parametrize("rows_in,rows_out,together,n_pages,seed", [
    (4, 9, 2, 200, 0), (64, 64, 4, 3000, 1), (200, 31, 1, 9001, 2), (31, 500, 8, 2000, 3), (1, 1000, 1, 1200, 4), (700, 700, 7, 30000, 5)])
def test_fork_batches(rows_in, rows_out, together, n_pages, seed):
    rng = np.random.default_rng(seed)
    P = [32, 64, 128][seed % 3]
    lens = rng.integers(0, 40 * P, rows_in).tolist()
    while sum(blocks(n, P) for n in lens) > n_pages:
        lens = [n // 2 for n in lens]
    pool = Pool(lens, P, n_pages, width=41, together=together, head=n_pages - 2, seed=seed)
    for step in range(4):                                                 # several steps, each from what the last one left
        parents = rng.integers(-1, len(pool.lens), rows_out).tolist()
        if step % 2:                                                      # most rows go on as they are
            parents = [b if b < len(pool.lens) and rng.random() < 0.9 else p for b, p in enumerate(parents)]
        keep = None if step == 1 else [0 if p < 0 else pool.lens[p] if rng.random() < 0.5 else int(rng.integers(0, pool.lens[p] + 1)) for p in parents]
        want = check_fork(pool, parents, keep)
        if isinstance(want, int):
            break
        pool = want[0]
        held = {q for b in range(len(pool.lens)) for q in pool.rows(b)}
        free = {int(pool.ring[(pool.state[0] + i) % n_pages]) for i in range(pool.state[1])}
        assert not held & free and len(held) + len(free) == n_pages       # every page is held or free
        count = np.zeros(n_pages, np.int64)
        for b in range(len(pool.lens)):
            np.add.at(count, pool.rows(b), 1)
        assert (pool.shared == np.maximum(count - 1, 0)).all()


def test_fork_holders_outside_the_call():
    """A page that a row of another table holds as well stays, and is copied before it is written to."""
    pool = Pool([100, 70], 64, 20, width=4)
    pool.shared[pool.rows(0)[1]] = 2
    pool.shared[pool.rows(1)[0]] = 1
    new, copies = check_fork(pool, [0, 0, -1])
    assert len(copies) == 2 and new.shared[pool.rows(0)[1]] == 1 and new.shared[pool.rows(1)[0]] == 0


def broken(**kw):
    pool = Pool([100, 70], 64, 20, width=4)
    for k, v in kw.items():
        if k == "page":
            pool.table[0, 1] = v
        elif k == "len":
            pool.lens[0] = v
        elif k == "shared":
            pool.shared[pool.rows(0)[0]] = v
        else:
            setattr(pool, k, v)
    return pool


@pytest.mark.parametrize("kw,parents,keep", [
    (dict(page=20), [0], None), (dict(page=-1), [0], None), (dict(page=2**31 - 1), [-1], None), (dict(len=257), [1], None), (dict(len=-1), [1], None),
    (dict(len=2**62), [0], None), (dict(shared=-1), [0], None), (dict(state=[20, 3]), [0], None), (dict(state=[0, 21]), [0], None), (dict(state=[-1, 3]), [0], None),
    (dict(), [2], None), (dict(), [-2], None), (dict(), [0], [101]), (dict(), [0], [-1]), (dict(state=[0, 20]), [-1], None)])
def test_fork_states_that_cannot_be(kw, parents, keep):
    pool = broken(**kw)
    t, _ = fork_call(pool, parents, keep)
    assert t["status"].item() == INCONSISTENT
    assert (t["copies"] == -1).all() and (t["table_out"] == -9).all() and (t["lens_out"] == -9).all() and (t["ring"].cpu().numpy() == pool.ring).all()
    assert t["state_out"].tolist() == pool.state and (t["shared_out"].cpu().numpy() == pool.shared).all()


def test_fork_without_pages():
    pool = Pool([100], 64, 4, width=4)
    assert check_fork(pool, [0, 0, 0, 0]) == NO_PAGES                     # three copies, two free pages
    assert not isinstance(check_fork(pool, [0, 0, 0]), int)
    pool = Pool([64, 100, 100], 64, 6, width=4)                           # the pages that a row gives are taken in the same call
    new, copies = check_fork(pool, [1, 1, 2])
    assert len(copies) == 1 and copies[0][1] in pool.rows(0) + [int(pool.ring[pool.state[0]])]


def compact_plain(pool):
    held = sorted({q for b in range(len(pool.lens)) for q in pool.rows(b)})
    U = len(held)
    holes, to, copies = [q for q in range(U) if q not in set(held)], {}, []
    shared = np.zeros_like(pool.shared)
    for q in held:
        to[q] = q
        if q >= U:
            to[q] = holes[len(copies)]
            copies.append([q, to[q], pool.P])
        shared[to[q]] = pool.shared[q]
    table = np.full_like(pool.table, -9)
    for b in range(len(pool.lens)):
        table[b, :len(pool.rows(b))] = [to[q] for q in pool.rows(b)]
    ring = pool.ring.copy()
    ring[:pool.n_pages - U] = np.arange(U, pool.n_pages)
    return table, shared, ring, [0, pool.n_pages - U], copies


def compact_call(pool, n_copies):
    b = lib()
    t = dict(lens=torch.tensor(pool.lens, **I64), table=torch.from_numpy(pool.table).to(DEV), table_out=torch.full(pool.table.shape, -9, **I32),
             shared=torch.from_numpy(pool.shared).to(DEV), shared_out=torch.full((pool.n_pages,), -9, **I32), ring=torch.from_numpy(pool.ring).to(DEV),
             copies=torch.full((n_copies, 3), -9, **I32), state_out=torch.full((2,), -9, **I64), status=torch.full((1,), -9, **I32),
             views=torch.full((len(pool.lens), 2), -9, **I64),
             workspace=torch.full((b.pages_compact_workspace_bytes(pool.n_pages),), 0xff, dtype=torch.uint8, device=DEV))

    def call():
        b.pages_compact(t["lens"], t["table"], t["table_out"], t["shared"], t["shared_out"], t["ring"], t["copies"], t["state_out"], t["status"], pool.P,
                        t["workspace"], t["views"])
    call()
    return t, call


@pytest.mark.parametrize("lens,n_pages,together", [
    ([100], 2, 1), ([100], 50, 1), ([0], 7, 1), ([0, 0, 300], 9, 1), ([64, 65, 700, 1], 100, 1), ([500] * 12, 200, 4), ([900] * 300, 9000, 3),
    ([2000] * 40, 70001, 1), ([64] * 8192, 8192, 1)])
def test_compact(lens, n_pages, together):
    pool = Pool(lens, 64, n_pages, width=33, together=together, head=1, seed=len(lens))
    table, shared, ring, state, copies = compact_plain(pool)
    t, call = compact_call(pool, len(copies) + 3)
    for _ in range(2):
        assert t["status"].item() == OK
        assert (t["table_out"].cpu().numpy() == table).all() and (t["shared_out"].cpu().numpy() == shared).all()
        assert (t["ring"].cpu().numpy() == ring).all() and t["state_out"].tolist() == state
        assert t["copies"].tolist() == copies + [[-1] * 3] * 3
        assert t["views"].tolist() == [[t["table_out"].data_ptr() + 4 * t["table_out"].stride(0) * b, n] for b, n in enumerate(lens)]
        call()
    if copies:
        t, _ = compact_call(pool, len(copies) - 1)
        assert t["status"].item() == LIST_FULL and (t["copies"] == -1).all() and (t["table_out"] == -9).all() and (t["shared_out"] == -9).all()
        assert (t["ring"].cpu().numpy() == pool.ring).all() and (t["state_out"] == -9).all()


@pytest.mark.parametrize("kw", [dict(page=20), dict(page=-3), dict(len=257), dict(len=-1)])
def test_compact_states_that_cannot_be(kw):
    pool = broken(**kw)
    t, _ = compact_call(pool, 20)
    assert t["status"].item() == INCONSISTENT and (t["copies"] == -1).all() and (t["table_out"] == -9).all() and (t["state_out"] == -9).all()


# ---------------------------------------------------------------- copies

def arrays_of(kind, shape, g):
    r = lambda dt, *more: torch.randint(0, 100, shape + more, generator=g, device=DEV).to(dt)  # noqa: E731
    if kind == "bf16":
        return [r(torch.bfloat16, D), r(torch.bfloat16, D), r(torch.int32), r(torch.float32)]
    if kind == "f32":
        return [r(torch.float32, D), r(torch.float32, D), r(torch.int32)]
    return [r(torch.uint8, 64), r(torch.uint8, 64), r(torch.uint8, 4), r(torch.uint8, 4), r(torch.int32), r(torch.float32)]


@pytest.mark.parametrize("kind", ["bf16", "f32", "four bits"])
@pytest.mark.parametrize("L,n_pages,H,P,n", [(None, 9, 1, 32, 3), (1, 40, 3, 64, 11), (5, 64, 8, 128, 20), (3, 700, 2, 32, 333), (None, 50, 8, 256, 25)])
def test_copies(kind, L, n_pages, H, P, n):
    g = torch.Generator(DEV).manual_seed(n)
    rng = np.random.default_rng(n)
    lead = () if L is None else (L,)
    arrays = arrays_of(kind, lead + (n_pages, H, P), g)
    summaries = [torch.randn(lead + (n_pages, H, D), generator=g, device=DEV).bfloat16(), torch.randn(lead + (n_pages, H), generator=g, device=DEV)]
    perm = rng.permutation(n_pages)
    copies = [[int(perm[rng.integers(n, n_pages)]), int(perm[i]), int(rng.integers(1, P + 1))] for i in range(n)]
    copies[-1][2] = P + 7                                                 # more tokens than the page has: all of them
    want = [x.clone() for x in arrays + summaries]
    lay = (slice(None),) * len(lead)
    for src, dst, m in copies:
        for x in want[:len(arrays)]:
            x[lay + (dst, slice(None), slice(0, m))] = x[lay + (src, slice(None), slice(0, m))].clone()
        for x in want[len(arrays):]:
            x[lay + (dst,)] = x[lay + (src,)].clone()
    copies.insert(n // 2, [n_pages, copies[0][1], 5])                     # pages that the pool does not have, and nothing to copy
    copies.insert(n // 2, [int(perm[-1]), -1, 5])
    copies.insert(n // 2, [int(perm[-1]), copies[0][1], 0])
    table = torch.tensor(copies + [[-1] * 3] * (n % 7), **I32)
    lib().pages_copy(table, arrays, summaries, stacked=L is not None)
    for x, y in zip(arrays + summaries, want):
        assert torch.equal(x, y)


def test_copies_of_nothing_and_of_lists_of_every_length():
    x = torch.arange(600 * 32, device=DEV, dtype=torch.float32).view(600, 1, 32)
    lib().pages_copy(torch.full((0, 3), -1, **I32), [x])
    for listed in (0, 1, 2, 3, 254, 255, 256, 257, 299):
        for spare in (0, 1, 300, 70000):
            y = x.clone()
            copies = torch.full((listed + spare, 3), -1, **I32)
            copies[:listed, 0], copies[:listed, 1], copies[:listed, 2] = torch.arange(listed, device=DEV), 300 + torch.arange(listed, device=DEV), 32
            lib().pages_copy(copies, [y])
            want = x.clone()
            want[300:300 + listed] = x[:listed]
            assert torch.equal(y, want)


def test_copies_past_32_bits():
    """Pages whose offsets in bytes pass 2^32, in many layers' arrays."""
    n_pages, H, P = 20000, 8, 128                                         # 5.2 GB
    x = torch.zeros((n_pages, H, P, D), dtype=torch.bfloat16, device=DEV)
    x[3], x[n_pages - 1] = 1.0, 2.0
    lib().pages_copy(torch.tensor([[3, n_pages - 2, P], [n_pages - 1, 4, 100]], **I32), [x])
    assert (x[n_pages - 2] == 1).all() and (x[4, :, :100] == 2).all() and (x[4, :, 100:] == 0).all()
    many = [torch.full((4, 1, 32), float(i), device=DEV) for i in range(150)]  # more arrays than one launch takes
    for i, y in enumerate(many):
        y[1] = -i
    lib().pages_copy(torch.tensor([[1, 3, 32]], **I32), many)
    assert all((y[3] == -i).all() and (y[2] == i).all() for i, y in enumerate(many))


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("kind", ["bf16", "quantized"])
@pytest.mark.parametrize("graph", [False, True])
def test_a_prompt_in_chunks_samples_beams_and_a_compact_pool(kind, graph):
    """Two prompts arrive in chunks, are forked into samples, which decode single tokens and speculative ones, lose some of them and are
    forked again; then the pool is made compact.  After each step the new tokens' attention is that over the whole history of their row."""
    b, H, G, P, n_pages = lib(), 2, 4, 32, 160
    rng = np.random.default_rng(8)
    g = torch.Generator(DEV).manual_seed(8)
    rand = lambda n: torch.randn((n, H, D), generator=g, device=DEV).bfloat16()  # noqa: E731
    width, most = 24, 8
    if kind == "bf16":
        arrays = [torch.full((n_pages, H, P, D), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    else:
        pool = b.QuantPool.empty(n_pages, H, P)
        arrays = [pool.k_codes, pool.v_codes, pool.k_scales, pool.v_scales]
        for x in arrays[2:]:
            x.fill_(255)
    arrays += [torch.zeros((n_pages, H, P), **I32), torch.full((n_pages, H, P), math.nan, device=DEV)]
    tables = [torch.full((most, width), -1, **I32) for _ in range(2)]
    lens, new_lens = torch.zeros(most, **I64), torch.zeros(most, **I64)
    shared = [torch.zeros(n_pages, **I32) for _ in range(2)]
    ring, state = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32), [torch.tensor([0, n_pages], **I64), torch.zeros(2, **I64)]
    slots, begin, lens_out = torch.zeros(600, **I64), torch.zeros(most + 1, **I64), torch.zeros(most, **I64)
    status, views = torch.zeros(1, **I32), torch.zeros((most, 2), **I64)
    copies, parents, keep = torch.zeros((n_pages, 3), **I32), torch.zeros(most, **I32), torch.zeros(most, **I64)
    k_in, v_in, q, out = rand(600), rand(600), torch.zeros((600, H * G, D), dtype=torch.bfloat16, device=DEV), torch.zeros((600, H * G, D), dtype=torch.bfloat16, device=DEV)
    deg_in = torch.ones((600, H), **I32)
    ws, fork_ws = X.workspace(600, H, G), torch.zeros(b.pages_fork_workspace_bytes(n_pages), dtype=torch.uint8, device=DEV)

    def grow():
        b.pages_resize(lens, new_lens, tables[0], ring, state[0], slots, begin, lens_out, state[1], status, P, views)
        if kind == "bf16":
            b.pages_write(slots, k_in, v_in, arrays[0], arrays[1], arrays[2], arrays[3], deg_in)
            b.extend_attn_paged(views, begin, arrays[0], arrays[1], arrays[3], H, G, q, out, X.SCALE, ws)
        else:
            p = b.QuantPool(*arrays)
            b.pages_quantize(slots, k_in, v_in, p, deg_in)
            b.extend_attn_quantized(views, begin, p, H, G, q, out, X.SCALE, ws)
        lens.copy_(lens_out)
        state[0].copy_(state[1])

    def fork():
        b.pages_fork(lens, parents, keep, tables[0], tables[1], shared[0], shared[1], ring, state[0], copies[:most], lens_out, state[1], status, P, fork_ws, views)
        b.pages_copy(copies[:most], arrays)
        tables[0].copy_(tables[1])
        shared[0].copy_(shared[1])
        lens.copy_(lens_out)
        state[0].copy_(state[1])

    def compact():
        b.pages_compact(lens, tables[0], tables[1], shared[0], shared[1], ring, copies, state[1], status, P, fork_ws, views)
        b.pages_copy(copies, arrays)
        tables[0].copy_(tables[1])
        shared[0].copy_(shared[1])
        state[0].copy_(state[1])

    run = {"grow": grow, "fork": fork, "compact": compact}
    if graph:
        graphs = {}
        torch.cuda.synchronize()
        for name, f in run.items():
            graphs[name] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graphs[name]):
                f()
        run = {name: x.replay for name, x in graphs.items()}
    history = [[torch.zeros((0, H, D), dtype=torch.bfloat16, device=DEV)] * 2 + [torch.zeros((0, H), **I32)] for _ in range(most)]

    def tokens(new):
        total = sum(new)
        k_in.copy_(rand(600)); v_in.copy_(rand(600)); q.copy_(torch.randn((600, H * G, D), generator=g, device=DEV))
        deg_in.copy_(torch.randint(1, 9, (600, H), generator=g, device=DEV))
        out.fill_(7.0)
        new_lens.copy_(lens + torch.tensor(new, **I64))
        run["grow"]()
        assert status.item() == 0 and b.workspace_status(ws) == 0
        at = 0
        for r, n in enumerate(new):
            history[r] = [torch.cat([x, y[at:at + n]]) for x, y in zip(history[r], (k_in, v_in, deg_in))]
            at += n
        assert lens.tolist() == [len(h[0]) for h in history]
        fake = object.__new__(X.Cache)
        fake.kind, fake.H, fake.lens = kind, H, [len(h[0]) for h in history]
        rows = [[x.transpose(0, 1).double() if x.dim() == 3 else torch.log(x.T.double()) for x in h] for h in history]
        if kind == "quantized":
            import test_gpu_serving as S
            rows = [[torch.from_numpy(S.quantize_plain(x.cpu().numpy())).to(DEV) if x.dim() == 3 and x.shape[1] else x for x in h] for h in rows]
        fake.rows = lambda r, h: tuple(x[h] for x in rows[r])
        o, bound = X.expected(fake, new, G, q, X.SCALE)
        assert ((out[:total].double() - o).abs() <= bound).all()
        assert (out[total:] == 7.0).all()

    def forked(p, kept):
        parents.copy_(torch.tensor(p, **I32)); keep.copy_(torch.tensor(kept, **I64))
        run["fork"]()
        assert status.item() == 0
        history[:] = [[x[:n].clone() for x in history[max(r, 0)]] for r, n in zip(p, kept)]
        assert lens.tolist() == [len(h[0]) for h in history]

    n = lambda r: len(history[r][0])  # noqa: E731
    tokens([70, 33, 0, 0, 0, 0, 0, 0])                                    # two prompts, in chunks
    tokens([130, 5, 0, 0, 0, 0, 0, 0])
    forked([0, 1, 0, 0, 1, -1, 0, 1], [n(0), n(1), n(0), n(0), n(1), 0, 150, 32])  # samples, and prefixes used again
    for _ in range(3):
        tokens([1, 1, 1, 1, 1, 0, 1, 1])
    tokens([4, 1, 6, 1, 40, 0, 3, 2])                                     # speculative tokens
    forked([0, 2, 2, 2, 4, 4, 6, -1], [n(0) - 3, n(2), n(2) - 6, n(2) - 1, n(4), 17, n(6), 0])
    tokens([1, 1, 2, 1, 1, 20, 1, 9])
    run["compact"]()
    assert status.item() == 0
    held = set(tables[0][r, i].item() for r in range(most) for i in range(blocks(n(r), P)))
    assert held == set(range(len(held))) and state[0].tolist() == [0, n_pages - len(held)]
    for x in arrays:                                                      # nothing behind the front is needed any more
        x[len(held):] = 255 if x.dtype is torch.uint8 else 0 if x.dtype is torch.int32 else math.nan
    forked([0, 0, 1, 2, 4, 5, 6, 7], [n(0), n(0), n(1), n(2), n(4), n(5), n(6), n(7)])
    tokens([3, 1, 1, 30, 1, 1, 1, 1])
    forked([-1] * 8, [0] * 8)
    assert (shared[0] == 0).all() and state[0][1].item() == n_pages       # all pages are free again
