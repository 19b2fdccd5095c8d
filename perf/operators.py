"""What is measured of the paged-serving operators: block tables and slot maps, writes through a slot map, page summaries,
attention over selected pages, four-bit pages and the attention that reads them.

Every kind of case has a plain form (elementary torch operations, 32 bits, 64 where a choice between near values hangs on
it) and the calls a user's program makes of the library.  Shapes: D = 128 throughout, pools [n_pages, H, page, D], block
tables int32 [batch, blocks], query head j reads KV head j // G.
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
        # one decoding step of the serving mix: 64 sequences grow by one token, a few of them into a new page
        dict(name="tables-step", kind="tables", batch=64, page=64, lo=4096, hi=65536, turnover=False),
        # a busy scheduler step: prompts arrive, sequences finish, others were just compressed to a quarter
        dict(name="tables-turnover", kind="tables", batch=512, page=32, lo=1, hi=32768, turnover=True),
        # the new keys and values of that decoding step, taken out of a fused projection's output
        dict(name="write-step", kind="write", tokens=64, heads=8, page=64, fused=True, spread=True, dtype="bf16"),
        # a compressed prompt, degrees and all, from its slab into its pages
        dict(name="write-prompt", kind="write", tokens=29999, heads=8, page=64, fused=False, spread=False, dtype="bf16"),
        # after a decoding step only each sequence's last page has a new summary
        dict(name="summaries-step", kind="summaries", batch=64, heads=8, page=64, lo=4096, hi=16384, last=True),
        # after a prefill every page gets one
        dict(name="summaries-prompt", kind="summaries", batch=5, heads=8, page=64, lo=8191, hi=32768, last=False),
        # one long conversation: 4096 of 131072 tokens are read
        dict(name="sparse-one", kind="sparse", batch=1, heads=8, group=4, page=64, lo=131072, hi=131072, select=64, first=1, last=2),
        # a serving batch, ragged: 32 pages of each sequence are read
        dict(name="sparse-batch", kind="sparse", batch=32, heads=8, group=4, page=64, lo=4096, hi=65536, select=32, first=1, last=2),
        # a decoded window that goes into four-bit pages, and back for clustering
        dict(name="quantize-window", kind="quantize", tokens=64, heads=8, page=64, dtype="f32"),
        # a compressed prompt into four-bit pages, and back
        dict(name="quantize-prompt", kind="quantize", tokens=32749, heads=8, page=64, dtype="bf16"),
        # one sequence's decode step over four-bit pages
        dict(name="quantized-one", kind="quantized", batch=1, heads=8, group=4, page=64, lo=16416, hi=16416),
        # the batch-32 decode workload over four-bit pages, ragged
        dict(name="quantized-batch", kind="quantized", batch=32, heads=8, group=4, page=64, lo=4097, hi=16384),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tables", "write", "summaries", "sparse", "quantize", "quantized"])
    page, heads, group = rng.choice([32, 64, 128, 256]), rng.choice([1, 2, 3, 4, 8]), rng.randint(1, 8)
    if kind == "tables":
        hi = _log_uniform(rng, 64, 32768)
        return dict(kind=kind, batch=_log_uniform(rng, 1, 512), page=page, lo=_log_uniform(rng, 1, hi), hi=hi, turnover=rng.random() < 0.5)
    if kind == "write":
        tokens = _log_uniform(rng, 1, 29999)
        return dict(kind=kind, tokens=tokens, heads=heads, page=page, fused=rng.random() < 0.5,
                    spread=tokens <= 512 and rng.random() < 0.5, dtype="bf16" if heads == 8 else rng.choice(["bf16", "f32"]))
    if kind == "quantize":
        return dict(kind=kind, tokens=_log_uniform(rng, 1, 32749), heads=heads, page=page, dtype="bf16" if heads == 8 else rng.choice(["bf16", "f32"]))
    batch = _log_uniform(rng, 1, 32)
    if kind == "summaries":
        batch = min(batch, 5)
        hi = _log_uniform(rng, 33, 32768)
        return dict(kind=kind, batch=batch, heads=heads, page=page, lo=_log_uniform(rng, 1, hi), hi=hi, last=rng.random() < 0.5)
    if kind == "sparse":
        batch, hi = min(batch, 128 // group), _log_uniform(rng, 64, 32768)
        first, last = rng.randint(0, 2), rng.randint(1, 3)
        most = max(first + last, 2048 // page)
        return dict(kind=kind, batch=batch, heads=heads, group=group, page=page, lo=_log_uniform(rng, 1, hi), hi=hi,
                    select=_log_uniform(rng, first + last, most), first=first, last=last)
    batch, hi = min(batch, 128 // group), _log_uniform(rng, 1, 8192)
    return dict(kind=kind, batch=batch, heads=heads, group=group, page=page, lo=_log_uniform(rng, 1, hi), hi=hi)


def _lens(case):
    """The batch's lengths: a matter of the case, not of the seed, and its bounds are among them."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    lens = [_log_uniform(rng, case["lo"], case["hi"]) for _ in range(case["batch"])]
    lens[0] = case["hi"]
    if len(lens) > 1:
        lens[-1] = case["lo"]
    return lens


def _old_and_new(case):
    lens = _lens(case)
    if not case["turnover"]:
        return lens, [n + 1 for n in lens]
    old, new = [], []
    for i, n in enumerate(lens):
        a, b = [(n, 0), (n, (n + 3) // 4), (n, n + 1), (0, n)][i % 4]
        old.append(a)
        new.append(b)
    return old, new


def _blocks(n, page):
    return (n + page - 1) // page


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _tables(lens, page, extra, seed):
    """Block tables over a permuted pool, and the pool's size."""
    need = [_blocks(n, page) for n in lens]
    n_pages = sum(need) + extra
    perm = torch.randperm(n_pages, generator=_gen(seed), device=DEV).to(torch.int32)
    width = max(max(need), 1)
    at = torch.tensor([sum(need[:b]) for b in range(len(lens))], device=DEV)
    i = torch.arange(width, device=DEV)
    mine = i < torch.tensor(need, device=DEV)[:, None]
    table = torch.where(mine, perm[torch.where(mine, at[:, None] + i, 0)], torch.zeros((), dtype=torch.int32, device=DEV))
    return table.contiguous(), n_pages, perm


def _views(table, lens):
    """ckv_paged_view: the address of a sequence's row of the table, and its length."""
    return torch.tensor([[table.data_ptr() + 4 * table.stride(0) * b, n] for b, n in enumerate(lens)], dtype=torch.int64, device=DEV)


def _degrees(shape, g):
    """Cluster degrees as two ratio-1 rounds leave them: mostly 1 to 7."""
    return torch.randint(1, 8, shape, generator=g, device=DEV, dtype=torch.int32)


def prepare(case, seed):
    g = _gen(1000003 * (seed + 1) + 17)
    kind, page = case["kind"], case["page"]
    st = dict(case=case)
    if kind == "tables":
        old, new = _old_and_new(case)
        width = max(max(_blocks(n, page) for n in old + new), 1)
        table, _, _ = _tables(old, page, 0, seed)
        used = sum(_blocks(n, page) for n in old)
        take = sum(max(0, _blocks(n, page) - _blocks(o, page)) for o, n in zip(old, new))
        n_pages = used + take + 5
        perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        full = torch.full((len(old), width), -1, dtype=torch.int32, device=DEV)
        mine = torch.arange(table.shape[1], device=DEV) < torch.tensor([_blocks(n, page) for n in old], device=DEV)[:, None]
        full[:, :table.shape[1]] = torch.where(mine, perm[table.long()], -1)
        ring = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        head = n_pages // 3
        at = (head + torch.arange(n_pages - used, device=DEV)) % n_pages
        ring[at] = perm[used:]
        grow = [max(0, n - o) for o, n in zip(old, new)]
        i64 = dict(dtype=torch.int64, device=DEV)
        st.update(lens=torch.tensor(old, **i64), new_lens=torch.tensor(new, **i64), table=full, ring=ring,
                  ring_state=torch.tensor([head, n_pages - used], **i64), slots=torch.full((sum(grow) + 3,), -7, **i64),
                  slot_begin=torch.full((len(old) + 1,), -7, **i64), lens_out=torch.full((len(old),), -7, **i64),
                  ring_state_out=torch.full((2,), -7, **i64), status=torch.full((1,), -7, dtype=torch.int32, device=DEV),
                  views=torch.zeros((len(old), 2), **i64), free=n_pages - used, taken=take,
                  given=sum(max(0, _blocks(o, page) - _blocks(n, page)) for o, n in zip(old, new)), grown=sum(grow))
        return st
    if kind in ("write", "quantize"):
        n, H = case["tokens"], case["heads"]
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}[case["dtype"]]
        table, n_pages, perm = _tables([n], page, 9, seed)
        if kind == "write" and case["spread"]:  # one token each of `tokens` sequences, anywhere in their last pages
            n_pages = n + 9
            perm = torch.randperm(n_pages, generator=g, device=DEV)
            slots = perm[:n] * page + torch.randint(0, page, (n,), generator=g, device=DEV)
        else:
            pos = torch.arange(n, device=DEV)
            slots = table[0, pos // page].long() * page + pos % page
        if kind == "write" and case["fused"]:  # rows of a fused q, k, v projection
            qkv = torch.randn((n, 6 * H, D), generator=g, device=DEV, dtype=dt)
            k, v = qkv[:, 4 * H:5 * H], qkv[:, 5 * H:]
        else:  # a slab [H, n, D] of a compressed cache
            k, v = (torch.randn((H, n, D), generator=g, device=DEV, dtype=dt).transpose(0, 1) for _ in range(2))
        if kind == "quantize":  # a few channels of real keys are many times larger than the rest
            k[..., torch.randint(0, D, (4,), generator=g, device=DEV)] *= 8
        st.update(slots=slots.contiguous(), k=k, v=v, deg=_degrees((H, n), g).t(), table=table, n=n)
        if kind == "write":
            st["slots"][-1:] = -1 if n > 1 else st["slots"][-1:]  # a padded batch ends in slots that are nobody's
            st.update(k_pages=torch.zeros((n_pages, H, page, D), dtype=dt, device=DEV), v_pages=torch.zeros((n_pages, H, page, D), dtype=dt, device=DEV),
                      deg_pages=torch.zeros((n_pages, H, page), dtype=torch.int32, device=DEV),
                      logdeg_pages=torch.zeros((n_pages, H, page), dtype=torch.float32, device=DEV))
        else:
            st.update(pool=_empty_pool(n_pages, H, page), k_out=torch.zeros((H, n, D), dtype=dt, device=DEV),
                      v_out=torch.zeros((H, n, D), dtype=dt, device=DEV), deg_out=torch.zeros((H, n), dtype=torch.int32, device=DEV),
                      logdeg_out=torch.zeros((H, n), dtype=torch.float32, device=DEV))
        return st
    lens, H = _lens(case), case["heads"]
    table, n_pages, _ = _tables(lens, page, 9, seed)
    st.update(table=table, lens=torch.tensor(lens, dtype=torch.int64, device=DEV), longest=max(lens), views=_views(table, lens))
    deg = _degrees((n_pages, H, page), g)
    if kind == "quantized":
        codes = [torch.randint(0, 256, (n_pages, H, page, D // 2), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        scales = [torch.randint(123, 127, (n_pages, H, page, D // 32), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        st["pool"] = [codes[0], codes[1], scales[0], scales[1], deg, torch.log(deg.float())]
    else:
        # keys of one page resemble each other: a centre for each page and head, and noise around it
        k = torch.randn((n_pages, H, page, D), generator=g, device=DEV, dtype=torch.bfloat16)
        centre = torch.randn((n_pages, H, 1, D), generator=g, device=DEV, dtype=torch.bfloat16)
        k.mul_(0.6).add_(centre, alpha=0.8)
        st.update(k_pages=k, deg_pages=deg)
        if kind == "summaries":
            st.update(c_pages=torch.zeros((n_pages, H, D), dtype=torch.bfloat16, device=DEV), clog_pages=torch.zeros((n_pages, H), dtype=torch.float32, device=DEV))
            begin = [n - 1 if case["last"] else 0 for n in lens]
            st.update(begin=torch.tensor(begin, dtype=torch.int64, device=DEV), most=max(_blocks(n, page) - b // page for n, b in zip(lens, begin)))
            return st
        c = (centre[:, :, 0].float() * 0.8 + 0.1 * torch.randn((n_pages, H, D), generator=g, device=DEV)).bfloat16()
        st.update(v_pages=torch.randn((n_pages, H, page, D), generator=g, device=DEV, dtype=torch.bfloat16), logdeg_pages=torch.log(deg.float()),
                  c_pages=c, clog_pages=torch.log(deg.sum(2).float()),
                  selected=torch.full((len(lens), H, case["select"]), -7, dtype=torch.int32, device=DEV))
    q = torch.randn((len(lens), H * case["group"], D), generator=g, device=DEV, dtype=torch.bfloat16)
    st.update(q=q, out=torch.zeros_like(q))
    if kind == "quantized":
        st["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    return st


def _empty_pool(n_pages, H, page):
    u8 = dict(dtype=torch.uint8, device=DEV)
    return [torch.zeros((n_pages, H, page, D // 2), **u8), torch.zeros((n_pages, H, page, D // 2), **u8), torch.zeros((n_pages, H, page, D // 32), **u8),
            torch.zeros((n_pages, H, page, D // 32), **u8), torch.zeros((n_pages, H, page), dtype=torch.int32, device=DEV),
            torch.zeros((n_pages, H, page), dtype=torch.float32, device=DEV)]


def run(state):
    kind = state["case"]["kind"]
    return {"tables": _run_tables, "write": _run_write, "summaries": _run_summaries, "sparse": _run_sparse, "quantize": _run_quantize,
            "quantized": _run_quantized}[kind](state)


# ---- block tables and slot maps

def _run_tables(st):
    page, table, ring = st["case"]["page"], st["table"], st["ring"]
    if own:
        from paper_2506_11418_b200 import binding as b
        b.pages_resize(st["lens"], st["new_lens"], table, ring, st["ring_state"], st["slots"], st["slot_begin"], st["lens_out"],
                       st["ring_state_out"], st["status"], page, st["views"])
        return dict(table=table, ring=ring, ring_state=st["ring_state_out"], slots=st["slots"], slot_begin=st["slot_begin"],
                    lens=st["lens_out"], status=st["status"])
    old, new = st["lens"], st["new_lens"]
    have, want = (old + page - 1) // page, (new + page - 1) // page
    take, give, grow = (want - have).clamp(min=0), (have - want).clamp(min=0), (new - old).clamp(min=0)
    rows = torch.arange(old.numel(), device=DEV)
    head, count = st["ring_state"][0], st["ring_state"][1]
    # pages given back, in the order of the sequences, behind the free ones
    b = torch.repeat_interleave(rows, give, output_size=st["given"])
    given = table[b, want[b] + torch.arange(st["given"], device=DEV) - (give.cumsum(0) - give)[b]]
    supply = torch.cat([ring[(head + torch.arange(st["free"], device=DEV)) % ring.numel()], given])
    ring[(head + count + torch.arange(st["given"], device=DEV)) % ring.numel()] = given
    # pages taken, in the same order, from the front
    b = torch.repeat_interleave(rows, take, output_size=st["taken"])
    table[b, have[b] + torch.arange(st["taken"], device=DEV) - (take.cumsum(0) - take)[b]] = supply[:st["taken"]]
    begin = torch.cat([torch.zeros_like(old[:1]), grow.cumsum(0)])
    b = torch.repeat_interleave(rows, grow, output_size=st["grown"])
    pos = old[b] + torch.arange(st["grown"], device=DEV) - begin[b]
    slots = torch.full_like(st["slots"], -1)
    slots[:st["grown"]] = table[b, pos // page].long() * page + pos % page
    state = torch.stack([(head + st["taken"]) % ring.numel(), count + st["given"] - st["taken"]])
    return dict(table=table, ring=ring, ring_state=state, slots=slots, slot_begin=begin, lens=new.clone(), status=torch.zeros_like(st["status"]))


# ---- writes through a slot map

def _run_write(st):
    if own:
        from paper_2506_11418_b200 import binding as b
        b.pages_write(st["slots"], st["k"], st["v"], st["k_pages"], st["v_pages"], st["deg_pages"], st["logdeg_pages"], st["deg"])
    else:
        page, mine = st["case"]["page"], st["slots"] >= 0
        s = st["slots"][mine]
        p, o = s // page, s % page
        st["k_pages"][p, :, o] = st["k"][mine]
        st["v_pages"][p, :, o] = st["v"][mine]
        st["deg_pages"][p, :, o] = st["deg"][mine]
        st["logdeg_pages"][p, :, o] = torch.log(st["deg"][mine].float())
    return [st["k_pages"], st["v_pages"], st["deg_pages"], st["logdeg_pages"]]


# ---- page summaries: the degree-weighted mean key of a page, and the logarithm of its degrees' sum

def _run_summaries(st):
    if own:
        from paper_2506_11418_b200 import binding as b
        b.pages_summarize(st["views"], st["k_pages"], st["deg_pages"], st["c_pages"], st["clog_pages"], st["most"], st["begin"])
    else:
        page = st["case"]["page"]
        blk = st["begin"][:, None] // page + torch.arange(st["most"], device=DEV)
        left = st["lens"][:, None] - blk * page                       # tokens of the sequence from this page on
        mine = left > 0
        p = st["table"].gather(1, torch.where(mine, blk, 0))[mine].long()
        held = torch.arange(page, device=DEV) < left[mine][:, None]
        w = (st["deg_pages"][p] * held[:, None]).float()
        total = w.sum(2)
        st["c_pages"][p] = ((st["k_pages"][p].float() * w[..., None]).sum(2) / total[..., None]).bfloat16()
        st["clog_pages"][p] = torch.log(total)
    return [st["c_pages"], st["clog_pages"]]


# ---- attention over the pages that their summaries select

def _run_sparse(st):
    case = st["case"]
    page, H, G = case["page"], case["heads"], case["group"]
    if own:
        from paper_2506_11418_b200 import binding as b
        b.pages_select(st["views"], st["c_pages"], st["clog_pages"], page, G, st["q"], SCALE, st["longest"], st["selected"], case["first"],
                       case["last"])
        b.decode_attn_selected(st["views"], st["k_pages"], st["v_pages"], st["logdeg_pages"], st["selected"], H, G, st["q"], st["out"], SCALE)
        return dict(selected=st["selected"], out=st["out"])
    lens, q = st["lens"], st["q"].view(-1, H, G, D)
    n = (lens + page - 1) // page
    blk = torch.arange(st["table"].shape[1], device=DEV)
    pages = st["table"].long()
    # scores in 64 bits: a selection must not hang on the order of a sum
    score = (st["c_pages"][pages].double().transpose(1, 2) @ q.double().transpose(2, 3) * SCALE).amax(3) + st["clog_pages"][pages].double().transpose(1, 2)
    always = (blk < case["first"]) | ((blk >= n[:, None] - case["last"]) & (blk < n[:, None]))
    score = torch.where(always[:, None], math.inf, score)
    score = torch.where((blk < n[:, None])[:, None], score, -math.inf)
    best = torch.sort(score, dim=2, descending=True, stable=True).indices[:, :, :case["select"]]
    best = torch.nn.functional.pad(best, (0, case["select"] - best.shape[2]), value=blk.numel())
    best = torch.where(torch.arange(case["select"], device=DEV) < n[:, None, None], best, blk.numel()).sort(2).values
    listed_ = best < blk.numel()
    at = torch.where(listed_, best, 0)
    p, h = pages[torch.arange(lens.numel(), device=DEV)[:, None, None], at], torch.arange(H, device=DEV)[None, :, None]
    held = listed_[..., None] & (at[..., None] * page + torch.arange(page, device=DEV) < lens[:, None, None, None])
    s = (st["k_pages"][p, h].float().flatten(2, 3) @ q.float().transpose(2, 3)) * SCALE + st["logdeg_pages"][p, h].flatten(2, 3)[..., None]
    out = _weighted(s, held.flatten(2, 3), st["v_pages"][p, h].float().flatten(2, 3))
    return dict(selected=torch.where(listed_, best, -1).int(), out=out.reshape(st["q"].shape).bfloat16())


def _weighted(s, held, v):
    """softmax over the tokens that are held, times the values: s [.., tokens, G], v [.., tokens, D] -> [.., G, D]."""
    s = torch.where(held[..., None], s, -math.inf)
    w = torch.exp(s - s.amax(-2, keepdim=True))
    return (w / w.sum(-2, keepdim=True)).transpose(-1, -2) @ torch.where(held[..., None], v, 0.0)


# ---- four-bit pages: rows in groups of 32 that share a power of two

def _run_quantize(st):
    if own:
        from paper_2506_11418_b200 import binding as b
        pool = b.QuantPool(*st["pool"])
        b.pages_quantize(st["slots"], st["k"], st["v"], pool, st["deg"])
        b.pages_dequantize(st["table"][0], st["n"], pool, st["k_out"], st["v_out"], st["deg_out"], st["logdeg_out"])
        return [st["k_out"], st["v_out"], st["deg_out"], st["logdeg_out"]]
    deg = st["deg"].t().contiguous()
    return [_four_bits(st["k"]), _four_bits(st["v"]), deg, torch.log(deg.float())]


def _four_bits(x):
    """The values that x [n, H, D] becomes, as a slab [H, n, D] of its type: the shared power of two is that of the group's
    largest magnitude over 4, elements go to the nearest level (ties to the even code) and end at 6."""
    y = x.transpose(0, 1).float().unflatten(2, (D // 32, 32))
    e = (torch.frexp(y.abs().amax(3, keepdim=True)).exponent - 3).clamp(-127, 125)
    m = torch.ldexp(y.abs(), -e)
    lv = torch.tensor(LEVELS, device=DEV)
    code = (m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)
    return (torch.sign(y) * torch.ldexp(lv[code], e)).flatten(2).to(x.dtype)


def _run_quantized(st):
    case = st["case"]
    H, G, page = case["heads"], case["group"], case["page"]
    if own:
        from paper_2506_11418_b200 import binding as b
        b.decode_attn_quantized(st["views"], b.QuantPool(*st["pool"]), H, G, st["q"], st["out"], SCALE, st["longest"], st["workspace"])
        return st["out"]
    pages = st["table"].long()
    k = _from_codes(st["pool"][0], st["pool"][2], pages, _KEY_BYTE)
    q = st["q"].view(-1, H, G, D).float()
    s = (k @ q.transpose(2, 3)) * SCALE + st["pool"][5][pages].transpose(1, 2).flatten(2, 3)[..., None]
    del k
    held = torch.arange(s.shape[2], device=DEV) < st["lens"][:, None, None]
    out = _weighted(s, held, _from_codes(st["pool"][1], st["pool"][3], pages, _VALUE_BYTE))
    return out.reshape(st["q"].shape).bfloat16()


def _from_codes(codes, scales, pages, byte_of):
    """The rows of a batch's pages in 32 bits: [batch, H, tokens, D]."""
    c = codes[pages].transpose(1, 2).flatten(2, 3)[..., byte_of]
    odd = torch.arange(D, device=DEV) % 2 == 1
    c = torch.where(odd, c >> 4, c & 15).long()
    lv = torch.tensor(LEVELS + [-x for x in LEVELS], device=DEV)
    e = scales[pages].transpose(1, 2).flatten(2, 3).int() - 127
    return lv[c] * torch.ldexp(torch.ones((), device=DEV), e).repeat_interleave(32, 3)


# ---- 64 bits, each operator from its definition

def exact(case, seed):
    st = prepare(case, seed)
    kind, page = case["kind"], case["page"]
    if kind == "tables":
        old, new = st["lens"].tolist(), st["new_lens"].tolist()
        table, ring = st["table"].cpu().numpy(), st["ring"].cpu().numpy()
        head, count = st["ring_state"].tolist()
        slots, begin = [], [0]
        for b in range(len(old)):                                     # sequences give first
            for i in range(_blocks(new[b], page), _blocks(old[b], page)):
                ring[(head + count) % len(ring)] = table[b, i]
                count += 1
        for b in range(len(old)):                                     # and then take
            for i in range(_blocks(old[b], page), _blocks(new[b], page)):
                table[b, i] = ring[head]
                head, count = (head + 1) % len(ring), count - 1
            pos = np.arange(old[b], max(old[b], new[b]))
            slots.append(table[b, pos // page].astype(np.int64) * page + pos % page)
            begin.append(begin[-1] + len(pos))
        slots = np.concatenate(slots + [np.full(st["slots"].numel() - begin[-1], -1, np.int64)])
        t = torch.from_numpy
        return dict(table=t(table), ring=t(ring), ring_state=torch.tensor([head, count]), slots=t(slots), slot_begin=torch.tensor(begin),
                    lens=torch.tensor(new), status=torch.zeros(1, dtype=torch.int32))
    if kind == "write":
        kept = (st["slots"] >= 0).nonzero()[:, 0]
        at = st["slots"][kept]                                        # row s of a pool laid out [n_pages * page, H, ..] is slot s
        new = [st["k"].double(), st["v"].double(), st["deg"], torch.log(st["deg"].double())]
        out = []
        for pool, rows in zip((st["k_pages"].double(), st["v_pages"].double(), st["deg_pages"], st["logdeg_pages"].double()), new):
            flat = pool.transpose(1, 2).flatten(0, 1)
            out.append(flat.index_copy(0, at, rows[kept]).unflatten(0, (-1, page)).transpose(1, 2).contiguous())
        return out
    if kind == "quantize":
        def nearest(x):
            y = x.double().transpose(0, 1).reshape(case["heads"], -1, D // 32, 32)
            out = torch.empty_like(y)
            lv = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
            even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=DEV)    # of two equally near levels the even code
            for a in range(0, y.shape[1], 4096):
                z = y[:, a:a + 4096]
                top = z.abs().amax(3, keepdim=True)
                e = torch.where(top > 0, torch.floor(torch.log2(top.clamp(min=1e-300))) - 2, -127.0).clamp(-127, 125)
                e = torch.where(2.0 ** (e + 3) <= top, e + 1, torch.where((2.0 ** (e + 2) > top) & (e > -127), e - 1, e))
                m = (z.abs() / 2.0 ** e).clamp(max=6.0)
                near = (m[..., None] - lv[even_first]).abs().argmin(-1)
                out[:, a:a + 4096] = torch.sign(z) * lv[even_first][near] * 2.0 ** e
            return out.reshape(case["heads"], -1, D)
        deg = st["deg"].t().contiguous()
        return [nearest(st["k"]), nearest(st["v"]), deg, torch.log(deg.double())]
    lens = st["lens"].tolist()
    if kind == "summaries":
        c, lg = st["c_pages"].double(), st["clog_pages"].double()
        for b, n in enumerate(lens):
            for i in range(st["begin"][b].item() // page, _blocks(n, page)):
                p, m = st["table"][b, i].item(), min(page, n - i * page)
                d = st["deg_pages"][p, :, :m].double()
                c[p] = torch.einsum("hm,hmd->hd", d, st["k_pages"][p, :, :m].double()) / d.sum(1, keepdim=True)
                lg[p] = torch.log(d.sum(1))
        return [c, lg]
    H, G = case["heads"], case["group"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    chosen = torch.full((len(lens), H, case.get("select", 1)), -1, dtype=torch.int32)
    lv = torch.tensor(LEVELS + [-x for x in LEVELS], dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        p = st["table"][b, :_blocks(n, page)].long()
        for h in range(H):
            q = st["q"][b, h * G:(h + 1) * G].double()
            if kind == "sparse":
                score = (torch.einsum("gd,nd->gn", q, st["c_pages"][p, h].double()) * SCALE).max(0).values + st["clog_pages"][p, h].double()
                rank = sorted(range(len(p)), key=lambda i, s=score.tolist(): (not (i < case["first"] or i >= len(p) - case["last"]), -s[i], i))
                best = sorted(rank[:case["select"]])
                chosen[b, h, :len(best)] = torch.tensor(best, dtype=torch.int32)
                pos = (torch.tensor(best, device=DEV)[:, None] * page + torch.arange(page, device=DEV)).flatten()
                pos = pos[pos < n]
                k, v, lg = (st[x][p[pos // page], h, pos % page].double() for x in ("k_pages", "v_pages", "logdeg_pages"))
            else:
                pos = torch.arange(n, device=DEV)
                at = (p[pos // page], h, pos % page)
                rows = []
                for c, e, byte_of in ((st["pool"][0], st["pool"][2], _KEY_BYTE), (st["pool"][1], st["pool"][3], _VALUE_BYTE)):
                    c, rank = c[at][:, byte_of].long(), torch.arange(D, device=DEV)
                    rows.append(lv[(c >> (4 * (rank % 2))) % 16] * 2.0 ** (e[at].double()[:, rank // 32] - 127))
                k, v, lg = rows[0], rows[1], st["pool"][5][at].double()
            w = torch.softmax(torch.einsum("gd,nd->gn", q, k) * SCALE + lg, 1)
            out[b, h * G:(h + 1) * G] = w @ v
    return dict(selected=chosen, out=out) if kind == "sparse" else out


def work(case):
    """Every input read once, every output written once; products of the plain definitions."""
    kind, page = case["kind"], case["page"]
    if kind == "tables":
        old, new = _old_and_new(case)
        grow = sum(max(0, n - o) for o, n in zip(old, new))
        moved = sum(abs(_blocks(n, page) - _blocks(o, page)) for o, n in zip(old, new))
        return dict(bytes=8 * grow + 8 * moved + len(old) * (8 * 4 + 16) + 40, flops=0)
    if kind in ("write", "quantize"):
        rows, es = case["tokens"] * case["heads"], 2 if case["dtype"] == "bf16" else 4
        if kind == "write":
            return dict(bytes=8 * case["tokens"] + rows * (4 * D * es + 12), flops=0)
        # read, written as codes, scales, degrees; read again, written as values
        return dict(bytes=8 * case["tokens"] + rows * (4 * D * es + 2 * 2 * (D // 2 + D // 32) + 4 + 8 + 8 + 8), flops=0)
    lens, H = _lens(case), case["heads"]
    if kind == "summaries":
        rows = sum(n - ((n - 1) // page * page if case["last"] else 0) for n in lens) * H
        pages = sum(1 if case["last"] else _blocks(n, page) for n in lens) * H
        return dict(bytes=rows * (2 * D + 4) + pages * (2 * D + 4), flops=2 * rows * D)
    G, Q = case["group"], len(lens) * H * case["group"] * D * 2
    if kind == "sparse":
        pages = sum(_blocks(n, page) for n in lens) * H
        rows = sum(min(n, case["select"] * page) for n in lens) * H
        return dict(bytes=pages * (2 * D + 4) + rows * (4 * D + 4) + 2 * Q + 4 * len(lens) * H * case["select"], flops=2 * G * D * (pages + 2 * rows))
    rows = sum(lens) * H
    return dict(bytes=rows * (2 * (D // 2 + D // 32) + 4) + 2 * Q, flops=4 * G * D * rows)
