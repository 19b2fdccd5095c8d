"""What is measured of attention for chunks of new tokens over a paged cache (bf16 and four-bit pages), and of sequences that share
pages: forking, freeing and copying them, and compacting a pool.

Every kind of case has a plain form (elementary torch operations, 32 bits) and the calls a user's program makes of the library.
Shapes: D = 128 throughout, pools [n_pages, H, page, D] (with the layers in front where pages are copied), block tables int32
[batch, blocks], query head j reads KV head j // G.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda"
SCALE = float(np.float32(1.0 / math.sqrt(D)))  # as a call's 32-bit argument has it

# Four-bit pages.  A row of 128 elements is 64 bytes of codes (two per byte, the even element in the low half) and four
# scale bytes, one per 32 elements: value = level(code) * 2^(scale - 127).  Where the bytes of a row sit:
#   keys:   byte 16 t + 4 j + i holds elements 32 j + 8 t + 2 i and the one after it   (t, j, i < 4)
#   values: byte  8 g + 2 j + i holds elements 32 j + 4 g + 2 i and the one after it   (g < 8, j < 4, i < 2)
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
_KEY_BYTE = [16 * ((d % 32) // 8) + 4 * (d // 32) + (d % 8) // 2 for d in range(D)]
_VALUE_BYTE = [8 * ((d % 32) // 4) + 2 * (d // 32) + (d % 4) // 2 for d in range(D)]


def listed():
    return [
        # one conversation goes on: a short question after 4096 slots
        dict(name="extend-question", kind="extend", batch=1, heads=8, group=4, page=64, lo=4113, hi=4113, new=17, single=0.0),
        # eight prompts arrive at once, nothing is cached yet
        dict(name="extend-prompts", kind="extend", batch=8, heads=8, group=4, page=64, lo=100, hi=2048, new=2048, single=0.0),
        # a scheduler step: a dozen sequences decode, four prompts are in the middle of their chunks
        dict(name="extend-mixed", kind="extend", batch=16, heads=8, group=4, page=64, lo=1024, hi=16384, new=512, single=0.75),
        # a chunk of a long prompt
        dict(name="extend-chunk", kind="extend", batch=1, heads=8, group=4, page=64, lo=32768, hi=32768, new=2048, single=0.0),
        # the last, large chunk of a longer one
        dict(name="extend-long", kind="extend", batch=1, heads=8, group=4, page=64, lo=49152, hi=49152, new=4096, single=0.0),
        # five speculative tokens each are verified over four-bit pages
        dict(name="quantized-verify", kind="quantized", batch=32, heads=8, group=4, page=64, lo=4097, hi=16384, new=5, single=0.0),
        # a chunk of a long prompt over four-bit pages
        dict(name="quantized-chunk", kind="quantized", batch=1, heads=8, group=4, page=64, lo=32768, hi=32768, new=1024, single=0.0),
        # eight samples of one prompt, all layers
        dict(name="fork-samples", kind="fork", rows_in=1, rows_out=8, heads=8, page=64, layers=32, lo=8191, hi=8191, together=1, trim=False),
        # a beam search's step over a batch, and prefixes that are used again
        dict(name="fork-beams", kind="fork", rows_in=64, rows_out=64, heads=8, page=64, layers=8, lo=500, hi=4000, together=4, trim=True),
        # a small pool, one layer of a model
        dict(name="compact-layer", kind="compact", rows=4, heads=8, page=64, layers=1, lo=500, hi=2000, together=2, spare=0.5),
        # a pool is made half as large
        dict(name="compact-pool", kind="compact", rows=32, heads=8, page=64, layers=8, lo=1000, hi=8000, together=4, spare=1.0),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["extend", "extend", "quantized", "quantized", "fork", "compact"])
    page, heads, group = rng.choice([32, 64, 128, 256]), rng.choice([1, 2, 3, 4, 8]), rng.randint(1, 8)
    if kind == "fork":
        hi = _log_uniform(rng, 64, 8192)
        rows = _log_uniform(rng, 1, max(1, 65536 // hi))
        return dict(kind=kind, rows_in=rows, rows_out=_log_uniform(rng, 1, 64), heads=heads, page=page, layers=rng.choice([1, 2, 4, 8]),
                    lo=_log_uniform(rng, 1, hi), hi=hi, together=rng.randint(1, 4), trim=rng.random() < 0.5)
    if kind == "compact":
        hi = _log_uniform(rng, 64, 8192)
        rows = _log_uniform(rng, 1, max(1, 65536 // hi))
        return dict(kind=kind, rows=rows, heads=heads, page=page, layers=rng.choice([1, 2, 4, 8]), lo=_log_uniform(rng, 1, hi), hi=hi,
                    together=rng.randint(1, 4), spare=rng.choice([0.1, 0.5, 1.0, 2.0]))
    hi = _log_uniform(rng, 16, 32768)
    batch = _log_uniform(rng, 1, max(1, min(32, 131072 // hi)))
    # (the plain form holds a weight for every query and slot: 2^32 of them at most)
    new = _log_uniform(rng, 1, min(hi, 2048, max(1, 2**32 // (batch * hi * heads * group))))
    return dict(kind=kind, batch=batch, heads=heads, group=group, page=page, lo=_log_uniform(rng, 1, hi), hi=hi, new=new,
                single=rng.choice([0.0, 0.0, 0.5, 0.9]))


def _rng(case):
    """Lengths and parents are a matter of the case, not of the seed."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lens(case, rows):
    rng = _rng(case)
    lens = [_log_uniform(rng, case["lo"], case["hi"]) for _ in range(rows)]
    lens[0] = case["hi"]
    if len(lens) > 1:
        lens[-1] = case["lo"]
    return lens


def _new(case, lens):
    """New tokens of every sequence, its last ones: single tokens, or up to `new` of them."""
    rng = _rng(case)
    n = [1 if b and rng.random() < case["single"] else min(x, case["new"]) for b, x in enumerate(lens)]
    return n


def _blocks(n, page):
    return (n + page - 1) // page


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _tables(need, n_pages, together, seed):
    """Block tables over a permuted pool; every `together` rows share the first half of the pages that all of them have.  Also the
    pages that no row holds, and how many rows hold a page beside its first."""
    perm = torch.randperm(n_pages, generator=_gen(seed), device=DEV).cpu().numpy().astype(np.int32)
    table, shared, at = np.full((len(need), max(max(need), 1)), -1, np.int32), np.zeros(n_pages, np.int32), 0
    for b, n in enumerate(need):
        first = b // together * together
        common = min(need[first:first + together]) // 2 if b > first else 0
        table[b, :common] = table[first, :common]
        shared[table[b, :common]] += 1
        table[b, common:n] = perm[at:at + n - common]
        at += n - common
    return table, perm[at:], shared


def _used(need, together):
    return sum(n - (min(need[b // together * together:][:together]) // 2 if b % together else 0) for b, n in enumerate(need))


def _views(table, lens):
    """ckv_paged_view: the address of a sequence's row of the table, and its length."""
    return torch.tensor([[table.data_ptr() + 4 * table.stride(0) * b, n] for b, n in enumerate(lens)], dtype=torch.int64, device=DEV)


def _degrees(shape, g):
    """Cluster degrees as two ratio-1 rounds leave them: mostly 1 to 7."""
    return torch.randint(1, 8, shape, generator=g, device=DEV, dtype=torch.int32)


def _fork_inputs(case):
    rng = _rng(case)
    lens = _lens(case, case["rows_in"])
    parents = [rng.randrange(-1 if case["trim"] else 0, len(lens)) for _ in range(case["rows_out"])]
    keep = [0 if p < 0 else rng.randint(0, lens[p]) if case["trim"] and rng.random() < 0.25 else lens[p] for p in parents]
    return lens, parents, keep


def prepare(case, seed):
    g = _gen(1000003 * (seed + 1) + 17)
    kind, page, H = case["kind"], case["page"], case["heads"]
    st = dict(case=case)
    i64, i32 = dict(dtype=torch.int64, device=DEV), dict(dtype=torch.int32, device=DEV)
    if kind in ("fork", "compact"):
        L = case["layers"]
        lens = _lens(case, case["rows_in"] if kind == "fork" else case["rows"])
        need = [_blocks(n, page) for n in lens]
        used = _used(need, case["together"])
        n_pages = used + (case["rows_out"] if kind == "fork" else max(1, int(used * case["spare"])))
        table, free, shared = _tables(need, n_pages, case["together"], seed)
        head = n_pages // 3
        ring = np.full(n_pages, -1, np.int32)
        ring[(head + np.arange(len(free))) % n_pages] = free
        rows = case["rows_out"] if kind == "fork" else case["rows"]
        deg = _degrees((L, n_pages, H, page), g)
        st.update(lens=torch.tensor(lens, **i64), table=torch.from_numpy(table).to(DEV), shared=torch.from_numpy(shared).to(DEV),
                  ring=torch.from_numpy(ring).to(DEV), ring_state=torch.tensor([head, len(free)], **i64), free=len(free),
                  table_out=torch.full((rows, table.shape[1]), -1, **i32), shared_out=torch.full((n_pages,), -7, **i32),
                  lens_out=torch.full((rows,), -7, **i64), ring_state_out=torch.full((2,), -7, **i64), status=torch.full((1,), -7, **i32),
                  views=torch.zeros((rows, 2), **i64), copies=torch.full((rows if kind == "fork" else min(used, n_pages - used), 3), -7, **i32),
                  workspace=torch.empty(64 + 16 * (n_pages + rows) + (1 << 16), dtype=torch.uint8, device=DEV),
                  k_pages=torch.randn((L, n_pages, H, page, D), generator=g, device=DEV, dtype=torch.bfloat16),
                  v_pages=torch.randn((L, n_pages, H, page, D), generator=g, device=DEV, dtype=torch.bfloat16),
                  deg_pages=deg, logdeg_pages=torch.log(deg.float()))
        if kind == "fork":
            _, parents, keep = _fork_inputs(case)
            st.update(parents=torch.tensor(parents, **i32), keep=torch.tensor(keep, **i64))
        return st
    lens = _lens(case, case["batch"])
    new = _new(case, lens)
    need = [_blocks(n, page) for n in lens]
    n_pages, total = sum(need) + 9, sum(new)
    table, _, _ = _tables(need, n_pages, 1, seed)
    table = torch.from_numpy(np.maximum(table, 0)).to(DEV)
    begin = np.concatenate([[0], np.cumsum(new)])
    row_seq = np.repeat(np.arange(len(lens)), new)
    st.update(table=table, lens=torch.tensor(lens, **i64), new=torch.tensor(new, **i64), most=max(new), total=total,
              q_begin=torch.tensor(begin, **i64), row_seq=torch.tensor(row_seq, **i64), row_pos=torch.tensor(np.arange(total) - begin[row_seq], **i64),
              views=_views(table, lens))
    deg = _degrees((n_pages, H, page), g)
    if kind == "quantized":
        codes = [torch.randint(0, 256, (n_pages, H, page, D // 2), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        scales = [torch.randint(123, 127, (n_pages, H, page, D // 32), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        st["pool"] = [codes[0], codes[1], scales[0], scales[1], deg, torch.log(deg.float())]
    else:
        st.update(k_pages=torch.randn((n_pages, H, page, D), generator=g, device=DEV, dtype=torch.bfloat16),
                  v_pages=torch.randn((n_pages, H, page, D), generator=g, device=DEV, dtype=torch.bfloat16), logdeg_pages=torch.log(deg.float()))
    # queries are rows of a fused q, k, v projection, three of padding behind the last
    qkv = torch.randn((total + 3, H * (case["group"] + 2), D), generator=g, device=DEV, dtype=torch.bfloat16)
    st.update(q=qkv[:, :H * case["group"]], out=torch.zeros((total + 3, H * case["group"], D), dtype=torch.bfloat16, device=DEV),
              workspace=torch.empty(64 << 20, dtype=torch.uint8, device=DEV))
    return st


def run(state):
    kind = state["case"]["kind"]
    return {"extend": _run_extend, "quantized": _run_extend, "fork": _run_fork, "compact": _run_compact}[kind](state)


# ---- attention of every sequence's new tokens to its slots up to their own

def _run_extend(st):
    case = st["case"]
    H, G, page, quantized = case["heads"], case["group"], case["page"], case["kind"] == "quantized"
    if own:
        from paper_2506_11418_b200 import binding as b
        if quantized:
            b.extend_attn_quantized(st["views"], st["q_begin"], b.QuantPool(*st["pool"]), H, G, st["q"], st["out"], SCALE, st["workspace"])
        else:
            b.extend_attn_paged(st["views"], st["q_begin"], st["k_pages"], st["v_pages"], st["logdeg_pages"], H, G, st["q"], st["out"], SCALE, st["workspace"])
        return st["out"]
    pages = st["table"].long()
    k = _from_codes(st["pool"][0], st["pool"][2], pages, _KEY_BYTE) if quantized else st["k_pages"][pages].transpose(1, 2).flatten(2, 3).float()
    bias = (st["pool"][5] if quantized else st["logdeg_pages"])[pages].transpose(1, 2).flatten(2, 3)
    i, t = torch.arange(st["most"], device=DEV), torch.arange(k.shape[2], device=DEV)
    rows = torch.where(i < st["new"][:, None], st["q_begin"][:-1, None] + i, 0)          # [batch, most] rows of q, padded
    q = st["q"][rows].unflatten(2, (H, G)).permute(0, 2, 1, 3, 4).flatten(2, 3).float()  # [batch, H, most * G, D]
    s = q @ k.transpose(2, 3)
    del k
    s.mul_(SCALE).add_(bias[:, :, None])
    hidden = t > (st["lens"] - st["new"])[:, None, None] + i[:, None]                    # [batch, most, slots]
    s.view(len(rows), H, st["most"], G, -1).masked_fill_(hidden[:, None, :, None], -math.inf)
    s.sub_(s.amax(3, keepdim=True)).exp_()
    v = _from_codes(st["pool"][1], st["pool"][3], pages, _VALUE_BYTE) if quantized else st["v_pages"][pages].transpose(1, 2).flatten(2, 3).float()
    o = (s @ torch.where((t < st["lens"][:, None])[:, None, :, None], v, 0.0)) / s.sum(3, keepdim=True)
    o = o.unflatten(2, (st["most"], G)).permute(0, 2, 1, 3, 4).flatten(2, 3)             # [batch, most, H * G, D]
    st["out"][:st["total"]] = o[st["row_seq"], st["row_pos"]].bfloat16()
    return st["out"]


def _from_codes(codes, scales, pages, byte_of):
    """The rows of a batch's pages in 32 bits: [batch, H, slots, D]."""
    c = codes[pages].transpose(1, 2).flatten(2, 3)[..., byte_of]
    odd = torch.arange(D, device=DEV) % 2 == 1
    c = torch.where(odd, c >> 4, c & 15).int()
    lv = torch.tensor(LEVELS + [-x for x in LEVELS], device=DEV)
    e = scales[pages].transpose(1, 2).flatten(2, 3).int() - 127
    return lv[c] * torch.ldexp(torch.ones((), device=DEV), e).repeat_interleave(32, 3)


# ---- forks: row b of the new table holds the first keep[b] tokens of row parents[b] of the old one

def _listed(table, lens, page):
    """Which entries of a table hold pages."""
    return torch.arange(table.shape[1], device=DEV) < ((lens + page - 1) // page)[:, None]


def _count(pages, mask, n_pages):
    return torch.zeros(n_pages, dtype=torch.int32, device=DEV).index_add_(0, torch.where(mask, pages, 0).flatten().long(), mask.flatten().int())


def _run_fork(st):
    page = st["case"]["page"]
    if own:
        from paper_2506_11418_b200 import binding as b
        b.pages_fork(st["lens"], st["parents"], st["keep"], st["table"], st["table_out"], st["shared"], st["shared_out"], st["ring"], st["ring_state"],
                     st["copies"], st["lens_out"], st["ring_state_out"], st["status"], page, st["workspace"], st["views"])
        b.pages_copy(st["copies"], [st["k_pages"], st["v_pages"], st["deg_pages"], st["logdeg_pages"]], stacked=True)
        return _tables_out(st)
    n_pages, ring, rows = st["shared"].numel(), st["ring"], torch.arange(st["parents"].numel(), device=DEV)
    head, count = st["ring_state"][0], st["ring_state"][1]
    before = _count(st["table"], _listed(st["table"], st["lens"], page), n_pages)
    outside = st["shared"] + 1 - before                                   # holders that are no rows of this call (pages of `before` only)
    keep = torch.where(st["parents"] < 0, 0, st["keep"])
    t = st["table"][st["parents"].clamp(min=0).long()]
    full = torch.arange(t.shape[1], device=DEV) < (keep // page)[:, None]
    tail = t.gather(1, (keep // page).clamp(max=t.shape[1] - 1)[:, None])[:, 0]
    tail = torch.where(keep % page > 0, tail, n_pages).long()             # the page that a row goes on writing to
    first = torch.full((n_pages + 1,), rows.numel(), device=DEV).scatter_reduce_(0, tail, rows, "amin")
    alone = torch.nn.functional.pad(_count(t, full, n_pages) + outside, (0, 1)) == 0
    takes = (tail < n_pages) & ~(alone[tail] & (first[tail] == rows))     # rows that need a page of their own
    listed_ = _listed(t, keep, page)
    after = _count(t, listed_ & ~(takes[:, None] & ~full), n_pages)
    freed = (before > 0) & (outside + after == 0)
    n_freed, n_taken = freed.sum(), takes.sum()
    # freed pages behind the queue's last, in order; pages taken from its front, freed ones last
    order = torch.arange(n_pages, device=DEV)
    freed_pages = torch.sort(torch.where(freed, order, n_pages)).values
    at = (head + count + order) % n_pages
    queue = torch.where(order < count, ring[(head + order) % n_pages].long(), freed_pages[(order - count).clamp(min=0)])
    ring[at] = torch.where(order < n_freed, freed_pages, ring[at].long()).int()
    mine = queue[(takes.cumsum(0) - 1).clamp(min=0)]
    where_ = (torch.arange(t.shape[1], device=DEV) == (keep // page)[:, None]) & takes[:, None]
    st["table_out"].copy_(torch.where(listed_, torch.where(where_, mine[:, None].int(), t), st["table_out"]))
    st["shared_out"].copy_(torch.where(before > 0, (outside + after - 1).clamp(min=0), st["shared"]))
    entry = torch.stack([tail.clamp(max=n_pages - 1), mine, keep % page], 1).int()
    by = torch.sort((~takes).int(), stable=True).indices                  # rows that copy first
    st["copies"].copy_(torch.where((rows < n_taken)[:, None], entry[by], -1))
    st["lens_out"].copy_(keep)
    st["ring_state_out"].copy_(torch.stack([(head + n_taken) % n_pages, count + n_freed - n_taken]))
    st["status"].zero_()
    _copy(st)
    return _tables_out(st)


def _copy(st):
    """Rows of pages, as listed; an entry that lists nothing copies onto itself a page that no entry writes."""
    src, dst, n = st["copies"].long().unbind(1)
    idle, still = src < 0, src[:1].clamp(min=0)
    src, dst = torch.where(idle, still, src), torch.where(idle, still, dst)
    mine = (torch.arange(st["case"]["page"], device=DEV) < n[:, None])[:, None]          # [copies, 1, page]
    st["k_pages"][:, dst] = torch.where(mine[..., None], st["k_pages"][:, src], st["k_pages"][:, dst])
    st["v_pages"][:, dst] = torch.where(mine[..., None], st["v_pages"][:, src], st["v_pages"][:, dst])
    st["deg_pages"][:, dst] = torch.where(mine, st["deg_pages"][:, src], st["deg_pages"][:, dst])
    st["logdeg_pages"][:, dst] = torch.where(mine, st["logdeg_pages"][:, src], st["logdeg_pages"][:, dst])


def _tables_out(st):
    names = ("table_out", "shared_out", "ring", "ring_state_out", "copies", "status", "k_pages", "v_pages", "deg_pages", "logdeg_pages")
    return {x: st[x] for x in names + (("lens_out",) if st["case"]["kind"] == "fork" else ())}


# ---- compaction: every page that a row holds to the front of the pool

def _run_compact(st):
    page = st["case"]["page"]
    if own:
        from paper_2506_11418_b200 import binding as b
        b.pages_compact(st["lens"], st["table"], st["table_out"], st["shared"], st["shared_out"], st["ring"], st["copies"], st["ring_state_out"],
                        st["status"], page, st["workspace"], st["views"])
        b.pages_copy(st["copies"], [st["k_pages"], st["v_pages"], st["deg_pages"], st["logdeg_pages"]], stacked=True)
        return _tables_out(st)
    n_pages, most = st["shared"].numel(), st["copies"].shape[0]
    order, listed_ = torch.arange(n_pages, device=DEV), _listed(st["table"], st["lens"], page)
    held = _count(st["table"], listed_, n_pages) > 0
    n_held = held.sum()
    moves, hole = held & (order >= n_held), ~held & (order < n_held)
    src = torch.sort(torch.where(moves, order, n_pages)).values[:most]    # pages that move, and where they go, in order
    dst = torch.sort(torch.where(hole, order, n_pages)).values[:most]
    to = torch.cat([order, order[:1]]).scatter(0, src, dst)[:n_pages]     # (entry n_pages is nobody's)
    st["table_out"].copy_(torch.where(listed_, to[st["table"].clamp(min=0).long()].int(), st["table_out"]))
    gone = torch.cat([st["shared"].new_zeros(1), st["shared"]])           # in front: a page that no row shares
    back = torch.cat([torch.where(held, order, -1), order[:1]]).scatter(0, dst, torch.where(src < n_pages, src, -1))[:n_pages]
    st["shared_out"].copy_(gone[torch.where(order < n_held, back, -1) + 1])
    st["ring"].copy_(torch.where(order < n_pages - n_held, (order + n_held).int(), st["ring"]))
    st["ring_state_out"].copy_(torch.stack([n_held * 0, n_pages - n_held]))
    st["copies"].copy_(torch.where((src < n_pages)[:, None], torch.stack([src, dst, torch.full_like(src, page)], 1), -1))
    st["status"].zero_()
    _copy(st)
    return _tables_out(st)


# ---- 64 bits, each operator from its definition

def exact(case, seed):
    st = prepare(case, seed)
    kind, page = case["kind"], case["page"]
    if kind in ("fork", "compact"):
        table, ring, shared = (st[x].cpu().numpy() for x in ("table", "ring", "shared"))
        out, n_pages, (head, count) = st["table_out"].cpu().numpy(), len(shared), st["ring_state"].tolist()
        lens, copies = st["lens"].tolist(), []
        holders = {}                                                      # of every page that a row lists
        for b, n in enumerate(lens):
            for p in table[b, :_blocks(n, page)].tolist():
                holders[p] = int(shared[p]) + 1
        new_shared = shared.copy()
        if kind == "compact":
            n_held, to = len(holders), {}
            holes = [p for p in range(n_held) if p not in holders]
            new_shared[:] = 0
            for p in sorted(holders):
                to[p] = p if p < n_held else holes[len(copies)]
                if p >= n_held:
                    copies.append([p, to[p], page])
                new_shared[to[p]] = shared[p]
            for b, n in enumerate(lens):
                for i in range(_blocks(n, page)):
                    out[b, i] = to[int(table[b, i])]
            ring[:n_pages - n_held] = np.arange(n_held, n_pages)
            head, count = 0, n_pages - n_held
        else:
            listed_before = sorted(holders)
            for b, n in enumerate(lens):
                for p in table[b, :_blocks(n, page)].tolist():
                    holders[p] -= 1                                       # what is left: holders outside the call
            parents, keep = st["parents"].tolist(), st["keep"].tolist()
            keep = [0 if p < 0 else n for p, n in zip(parents, keep)]
            whole = [table[p, :n // page].tolist() if p >= 0 else [] for p, n in zip(parents, keep)]
            for pages in whole:
                for p in pages:
                    holders[p] += 1
            copying = []
            for b, (p, n) in enumerate(zip(parents, keep)):
                out[b, :n // page] = whole[b]
                if n % page:
                    q = int(table[p, n // page])
                    if holders[q] == 0:
                        holders[q], out[b, n // page] = -1, q             # nobody else's: this row goes on with it
                    else:
                        copying.append((b, q, n % page))
            for q in listed_before:
                left = abs(holders[q])
                new_shared[q] = max(left - 1, 0)
                if left == 0:
                    ring[(head + count) % n_pages] = q
                    count += 1
            for b, q, n in copying:
                out[b, keep[b] // page] = ring[head]
                copies.append([q, int(ring[head]), n])
                head, count = (head + 1) % n_pages, count - 1
        for src, dst, n in copies:
            for x in ("k_pages", "v_pages", "deg_pages", "logdeg_pages"):
                st[x][:, dst, :, :n] = st[x][:, src, :, :n]
        copies += [[-1, -1, -1]] * (st["copies"].shape[0] - len(copies))
        t = torch.from_numpy
        r = dict(table_out=t(out), shared_out=t(new_shared), ring=t(ring), ring_state_out=torch.tensor([head, count]), copies=torch.tensor(copies).int(),
                 status=torch.zeros(1, dtype=torch.int32), k_pages=None, v_pages=None, deg_pages=st["deg_pages"], logdeg_pages=st["logdeg_pages"].double())
        if st["k_pages"].numel() < 1 << 28:
            r.update(k_pages=st["k_pages"].double(), v_pages=st["v_pages"].double())
        return dict(r, lens_out=torch.tensor(keep)) if kind == "fork" else r
    H, G, lens, new = case["heads"], case["group"], st["lens"].tolist(), st["new"].tolist()
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    lv = torch.tensor(LEVELS + [-x for x in LEVELS], dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        pos = torch.arange(n, device=DEV)
        p = st["table"][b, pos // page].long()
        for h in range(H):
            where_ = (p, h, pos % page)
            if kind == "quantized":
                rows = []
                for c, e, byte_of in ((st["pool"][0], st["pool"][2], _KEY_BYTE), (st["pool"][1], st["pool"][3], _VALUE_BYTE)):
                    c, rank = c[where_][:, byte_of].long(), torch.arange(D, device=DEV)
                    rows.append(lv[(c >> (4 * (rank % 2))) % 16] * 2.0 ** (e[where_].double()[:, rank // 32] - 127))
                k, v, bias = rows[0], rows[1], st["pool"][5][where_].double()
            else:
                k, v, bias = (st[x][where_].double() for x in ("k_pages", "v_pages", "logdeg_pages"))
            for j in range(G):
                s = st["q"][at:at + m, h * G + j].double() @ k.T * SCALE + bias
                s = torch.where(torch.tril(torch.ones_like(s, dtype=torch.bool), n - m), s, -math.inf)
                out[at:at + m, h * G + j] = torch.softmax(s, 1) @ v
        at += m
    return out


def work(case):
    """Every input read once, every output written once; products of the plain definitions."""
    kind, page, H = case["kind"], case["page"], case["heads"]
    if kind in ("fork", "compact"):
        lens = _lens(case, case["rows_in"] if kind == "fork" else case["rows"])
        need = [_blocks(n, page) for n in lens]
        used = _used(need, case["together"])
        row = 2 * case["layers"] * H * (4 * D + 8)                        # a token's rows in all layers, read and written
        if kind == "compact":
            n_pages = used + max(1, int(used * case["spare"]))
            moved = used * (n_pages - used) // n_pages                    # (what of a random pool's held pages is behind its front)
            return dict(bytes=moved * page * row + 8 * sum(need) + 12 * n_pages, flops=0)
        # one row goes on with its parent's last page, further ones copy what it holds
        lens, parents, keep = _fork_inputs(case)
        seen, copied = set(), 0
        for p, n in zip(parents, keep):
            if n % page and (p, n // page) in seen:
                copied += n % page
            seen.add((p, n // page))
        n_pages = used + case["rows_out"]
        return dict(bytes=copied * row + 4 * sum(need) + 4 * sum(_blocks(n, page) for n in keep) + 8 * n_pages, flops=0)
    lens = _lens(case, case["batch"])
    new, G = _new(case, lens), case["group"]
    seen = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))  # visible (token, slot) pairs
    per = 2 * (D // 2 + D // 32) + 4 if kind == "quantized" else 4 * D + 4
    return dict(bytes=sum(lens) * H * per + sum(new) * H * G * D * 4, flops=4 * G * D * H * seen)
