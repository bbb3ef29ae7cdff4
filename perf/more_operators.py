"""The serving operators on a paged latent cache, measured: attention of one new token per sequence over the pages, rows put into pages and
read back, pages reserved (allocated, and copied where they are shared), sequences forked and freed, the pool compacted.

Pool: keys and values [n_pages, kv heads, P, head size]; refs[p] counts the sequences that hold page p (0: free); row r of sequence b is
place r % P of page table[b, r // P]; an entry of the table is -1 where there is no page."""
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one user, a short context, the head layout of the 16k prefill: what counts is how long the call takes to get going
        {"name": "attend_1x1k", "op": "attend", "B": 1, "S": 1024, "P": 64, "hq": 8, "hk": 2, "dh": 128, "ragged": False},
        # the decode benchmark's batch and context
        {"name": "attend_32x16k", "op": "attend", "B": 32, "S": 16384, "P": 64, "hq": 8, "hk": 2, "dh": 128, "ragged": False},
        # one long context in small pages, the training configuration's heads
        {"name": "attend_1x128k", "op": "attend", "B": 1, "S": 131072, "P": 16, "hq": 8, "hk": 2, "dh": 64, "ragged": False},
        # users at different points, one of them with nothing cached yet, large heads, pages that end inside every tile
        {"name": "attend_13x5001_ragged", "op": "attend", "B": 13, "S": 5001, "P": 40, "hq": 4, "hk": 1, "dh": 256, "ragged": True},
        # the keys and values of one decode step's tokens
        {"name": "append_32x1", "op": "append", "B": 32, "S": 1000, "P": 64, "n": 1, "hk": 2, "dh": 128},
        # a prompt's keys and values handed over from the prefill
        {"name": "append_1x16k", "op": "append", "B": 1, "S": 16500, "P": 64, "n": 16384, "hk": 2, "dh": 128},
        # before a decode step of beams that were forked a step ago: every beam but one of each request gets its own last page
        {"name": "reserve_32x1", "op": "reserve", "B": 32, "S": 1000, "P": 64, "share": 4, "n": 1, "all": False, "hk": 2, "dh": 128},
        # continuations of one prompt that are to be changed from the first row on: pages of their own for all of it
        {"name": "reserve_8x16k_own", "op": "reserve", "B": 8, "S": 16384, "P": 64, "share": 8, "n": 16384, "all": True, "hk": 2, "dh": 128},
        # a step of beam search: 8 requests with 4 beams each take over one another's pages, then some end and some go back a few tokens
        {"name": "fork_beams_32x1k", "op": "fork", "B": 32, "S": 1000, "P": 64, "kind": "beams", "group": 4, "hk": 2, "dh": 128},
        # 8 prompts of 16k tokens with 31 continuations each, in small pages; half of the continuations end at once
        {"name": "fork_256x16k", "op": "fork", "B": 256, "S": 16384, "P": 16, "kind": "samples", "group": 32, "hk": 2, "dh": 32},
        # a small pool after a few sequences have gone
        {"name": "compact_24x700", "op": "compact", "B": 24, "S": 700, "P": 16, "gone": 0.25, "hk": 2, "dh": 64},
        # a pool of a gigabyte of which half has been freed
        {"name": "compact_64x16k_half", "op": "compact", "B": 64, "S": 16384, "P": 64, "gone": 0.5, "hk": 2, "dh": 128},
    ]


HEADS = [(8, 2, 128), (8, 2, 64), (16, 4, 64), (4, 4, 32), (4, 1, 256), (8, 1, 64), (16, 1, 128), (4, 2, 128)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "reserve", "fork", "compact"])
    hq, hk, dh = rng.choice(HEADS)
    P = rng.choice([16, 32, 64, 128, rng.randint(1, 200)])
    B = _log(rng, 1, 64)
    most = 32 * 16384 * 2 * 128 // (B * hk * dh)            # rows of a sequence that keep the case within the largest listed one
    if op == "attend":
        return {"op": op, "B": B, "S": _log(rng, 1, min(131072, most)), "P": P, "hq": hq, "hk": hk, "dh": dh, "ragged": rng.random() < 0.6}
    S = _log(rng, 1, max(1, min(16384, most // 4, P * 1024)))
    if op == "append":
        n = max(1, min(S // 4, 16384 // B))
        return {"op": op, "B": B, "S": n + rng.randint(0, 300), "P": P, "n": n, "hk": hk, "dh": dh}
    if op == "reserve":
        full = rng.random() < 0.3
        return {"op": op, "B": B, "S": S, "P": P, "share": rng.randint(1, 8), "n": S if full else rng.randint(1, 40), "all": full, "hk": hk, "dh": dh}
    if op == "fork":
        return {"op": op, "B": B, "S": S, "P": P, "kind": rng.choice(["beams", "samples"]), "group": rng.randint(2, 8), "hk": 2, "dh": 32}
    return {"op": op, "B": B, "S": S, "P": P, "gone": round(rng.uniform(0.1, 0.9), 3), "hk": hk, "dh": dh}


def _lens(case):
    """Cached rows of each sequence: all full, or spread down from the full one with one empty sequence among three or more."""
    B, S = case["B"], case["S"]
    if not case.get("ragged"):
        return [S] * B
    lens = [max(0, S * (B - b) // B - (b % 3)) for b in range(B)]
    if B >= 3:
        lens[B // 2] = 0
    return lens


def _held(case):
    """Tokens that each sequence holds before a reservation, fork or compaction; members of a group that shares pages have the same."""
    B, S = case["B"], case["S"]
    if case["op"] == "reserve":
        return [S if case["all"] else max(1, S - 37 * (b // case["share"])) for b in range(B)]
    if case["op"] == "fork":
        held = [max(1, S - 13 * (b // case["group"])) for b in range(B)]
        return held if case["kind"] == "beams" else [n if b % case["group"] == 0 else 0 for b, n in enumerate(held)]
    return [max(1, S - 5 * b) for b in range(B)]


def _up(n, P):
    return -(-n // P)


def _window(case):
    """(first page index, behind the last) of a reservation, for each sequence."""
    out = []
    for n in _held(case):
        first = 0 if case["all"] else n
        out.append((first // case["P"], _up(first + case["n"], case["P"])))
    return out


def _copies(case):
    """Pages that a reservation has to copy: those of the window that the group shares, for all of the group but its last."""
    B, share, n = case["B"], case["share"], 0
    for b, (held, (i0, i1)) in enumerate(zip(_held(case), _window(case))):
        if b % share != share - 1 and b != B - 1:
            n += max(0, min(i1, _up(held, case["P"])) - i0)
    return n


def work(case):
    if case["op"] == "attend":
        rows = sum(_lens(case))
        return {"bytes": rows * case["hk"] * case["dh"] * 4 + 4 * sum(_up(n, case["P"]) for n in _lens(case)) + 4 * case["B"] * case["hq"] * (case["dh"] + 1),
                "flops": 4 * rows * case["hq"] * case["dh"]}
    page = 4 * case["hk"] * case["P"] * case["dh"]               # keys and values of a page
    if case["op"] == "append":
        rows = case["B"] * case["n"] * case["hk"]
        return {"bytes": rows * 12 * case["dh"], "flops": rows * case["dh"]}
    if case["op"] == "reserve":
        entries = sum(b - a for a, b in _window(case))
        return {"bytes": 2 * page * _copies(case) + 16 * entries, "flops": entries}
    if case["op"] == "fork":
        entries = sum(_up(n, case["P"]) for n in _held(case)) * (1 if case["kind"] == "beams" else case["group"])
        return {"bytes": 24 * entries, "flops": 2 * entries}
    held = sum(_up(n, case["P"]) for n in _held(case))
    left = held * (1 - case["gone"])
    return {"bytes": int(2 * page * left * case["gone"]) + 8 * held, "flops": held}


# ---------------------------------------------------------------------------------------------------------- inputs of a case
def _handle(hq, hk, dh):
    from paper_2510_04476_b200.binding import CCA
    return CCA(d_model=hq * dh, n_q_heads=hq, n_kv_heads=hk, head_dim=dh)


def _pool(gen, n_pages, P, B, max_pages, hk, dh):
    """The pool's tensors; what says who holds which page (refs, table, len) lies in one buffer."""
    meta = torch.zeros(n_pages + B * max_pages + B, dtype=torch.int32, device="cuda")
    pages = {"refs": meta[:n_pages], "table": meta[n_pages:n_pages + B * max_pages].view(B, max_pages), "len": meta[n_pages + B * max_pages:]}
    pages["table"].fill_(-1)
    for name in ("k", "v"):
        pages[name] = torch.empty(n_pages, hk, P, dh, dtype=torch.bfloat16, device="cuda")
        for part in pages[name].split(max(1, (1 << 26) // (hk * P * dh))):
            part.normal_(generator=gen)
    return pages, meta


def _give(pages, order, counts, group=1):
    """counts[b] pages for sequence b, taken from `order`; the members of a group have the same ones."""
    at = 0
    table = torch.full(pages["table"].shape, -1, dtype=torch.int32)
    order = order.cpu().int()
    for b, n in enumerate(counts):
        if b % group == 0:
            row = order[at:at + n]
            at += n
        table[b, :n] = row
    pages["table"].copy_(table)
    _recount(pages)


def _recount(pages):
    entries = pages["table"].flatten().long()
    there = entries >= 0
    pages["refs"].zero_().index_add_(0, entries.clamp_min(0), there.int())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    B, S, P, hk, dh, op = case["B"], case["S"], case["P"], case["hk"], case["dh"], case["op"]
    st = {"case": case}
    if op == "attend":
        lens, hq = _lens(case), case["hq"]
        counts = [_up(n, P) for n in lens]
        n_pages = sum(counts) + max(8, sum(counts) // 16)       # a few are free
        pages, meta = _pool(gen, n_pages, P, B, max(1, _up(S, P)), hk, dh)
        # normalised queries and keys, as the block makes them; the keys' temperatures differ by head
        st["q"] = torch.nn.functional.normalize(normal(B, hq, dh), dim=-1).mul(math.sqrt(dh)).bfloat16()
        beta = torch.linspace(0.7, 1.5, hk, device="cuda").view(1, hk, 1, 1)
        for part in pages["k"].split(max(1, (1 << 24) // (hk * P * dh))):
            part.copy_(torch.nn.functional.normalize(part.float(), dim=-1) * (math.sqrt(dh) * beta))
        _give(pages, torch.randperm(n_pages, generator=gen, device="cuda"), counts)
        pages["len"].copy_(torch.tensor(lens, dtype=torch.int32))
        if own:
            st["cca"] = _handle(hq, hk, dh)
            st["ws"] = st["cca"].alloc_paged_workspace(B, S)
    elif op == "append":
        counts = [_up(S, P)] * B
        n_pages = sum(counts) + 8
        pages, meta = _pool(gen, n_pages, P, B, counts[0], hk, dh)
        _give(pages, torch.randperm(n_pages, generator=gen, device="cuda"), counts)
        pages["len"].copy_(torch.randint(0, S - case["n"] + 1, (B,), generator=gen, device="cuda"))
        st["k"], st["v"] = normal(B, case["n"], hk, dh).bfloat16(), normal(B, case["n"], hk, dh).bfloat16()
        if own:
            st["cca"] = _handle(hk, hk, dh)
    elif op == "reserve":
        held = _held(case)
        counts = [_up(n, P) for n in held]
        wide = max(b for _, b in _window(case))
        distinct = sum(counts[::case["share"]])
        n_pages = distinct + sum(b - a for a, b in _window(case)) + 16
        pages, meta = _pool(gen, n_pages, P, B, max(wide, max(counts)), hk, dh)
        _give(pages, torch.randperm(n_pages, generator=gen, device="cuda"), counts, case["share"])
        pages["len"].copy_(torch.tensor(held, dtype=torch.int32))
        st["first"] = torch.zeros(B, dtype=torch.int32, device="cuda") if case["all"] else None
        st["width"] = max(b - a for a, b in _window(case))
    elif op == "fork":
        held, group = _held(case), case["group"]
        counts = [_up(n, P) for n in held]
        n_pages = sum(counts) + 8
        pages, meta = _pool(gen, n_pages, P, B, max(counts) + 2, hk, dh)
        _give(pages, torch.randperm(n_pages, generator=gen, device="cuda"), counts)
        pages["len"].copy_(torch.tensor(held, dtype=torch.int32))
        base = torch.arange(B, device="cuda") // group * group
        if case["kind"] == "beams":           # every beam goes on from one of its request's, some from themselves
            size = (B - base).clamp_max(group)
            st["child"] = torch.arange(B, dtype=torch.int32, device="cuda")
            st["parent"] = (base + (torch.rand(B, generator=gen, device="cuda") * size).long().minimum(size - 1)).int()
        else:
            st["child"] = torch.tensor([b for b in range(B) if b % group] or [0], dtype=torch.int32, device="cuda")
            st["parent"] = base.int()[st["child"].long()]
        luck = torch.rand(B, generator=gen, device="cuda")
        keep = torch.where(luck < 0.25, torch.randint(0, S + 1, (B,), generator=gen, device="cuda").int(), -1)
        st["keep"] = torch.where(luck > (0.5 if case["kind"] == "samples" else 0.8), 0, keep).int()
    else:
        held = _held(case)
        counts = [_up(n, P) for n in held]
        n_pages = sum(counts)
        pages, meta = _pool(gen, n_pages, P, B, max(counts), hk, dh)
        _give(pages, torch.randperm(n_pages, generator=gen, device="cuda"), counts)
        pages["len"].copy_(torch.tensor(held, dtype=torch.int32))
        gone = torch.rand(pages["table"].shape, generator=gen, device="cuda") < case["gone"]          # what other sequences held
        pages["table"].masked_fill_(gone, -1)
        _recount(pages)
    if own and "cca" not in st:
        st["cca"] = _handle(hk, hk, dh)
        st["ws"] = st["cca"].alloc_pages_workspace(n_pages, B, pages["table"].shape[1])
    st["pages"], st["meta"] = pages, meta
    st["meta0"] = meta.clone()
    return st


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(st):
    return {"attend": _attend, "append": _append, "reserve": _reserve, "fork": _fork, "compact": _compact}[st["case"]["op"]](st)


def _attend(st):
    """The new tokens' queries over the cached rows."""
    q, pages, case = st["q"], st["pages"], st["case"]
    if own:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        return {"o": st["cca"].paged_attention(q, pages, case["S"], st["ws"], lse=lse), "lse": lse}
    hk, dh = case["hk"], case["dh"]
    at = pages["table"].long().clamp_min(0)
    k, v = (pages[n][at].transpose(1, 2).flatten(2, 3) for n in ("k", "v"))                   # [B, hk, rows, dh]
    s = q.float().unflatten(1, (hk, -1)) @ k.float().transpose(-1, -2) / math.sqrt(dh)        # [B, hk, g, rows]
    there = torch.arange(s.shape[-1], device=q.device) < pages["len"].view(-1, 1, 1, 1)
    s = s.masked_fill(~there, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    e = torch.exp(s - top)
    total = e.sum(-1, keepdim=True)
    o = e @ v.float().masked_fill(~there.transpose(-1, -2), 0.0) / total.clamp_min(1e-30)
    return {"o": o.flatten(1, 2).bfloat16(), "lse": (top + total.log()).flatten(1)}


def _append(st):
    """New rows into the pages, and what the pages now hold in their places."""
    pages, case = st["pages"], st["case"]
    if own:
        st["cca"].paged_append(pages, st["k"], st["v"])
        k, v = st["cca"].paged_read(pages, case["n"])
        return {"k": k, "v": v}
    P = case["P"]
    row = (pages["len"].view(-1, 1) + torch.arange(case["n"], device="cuda")).long()          # [B, n]
    page, place = pages["table"].long().gather(1, row // P), row % P
    for name in ("k", "v"):
        pages[name][page, :, place] = st[name]
    return {name: pages[name][page, :, place] for name in ("k", "v")}


def _reserve(st):
    """Pages for the rows behind each sequence's, or for all of its rows, that it holds alone."""
    pages, case = st["pages"], st["case"]
    st["meta"].copy_(st["meta0"])            # as the steps before left it
    if own:
        st["cca"].pages_reserve(pages, case["n"], st["ws"], first=st["first"])
        return pages
    P, refs, table = case["P"], pages["refs"], pages["table"]
    B, wide = table.shape
    first = pages["len"] if st["first"] is None else st["first"]
    i0, i1 = first // P, (first + case["n"] + P - 1) // P
    at = i0.view(-1, 1) + torch.arange(st["width"], device="cuda")                            # [B, width] page indexes
    inside = at < i1.view(-1, 1)
    at = at.clamp_max(wide - 1).long()
    entry = table.gather(1, at)
    page = entry.long().clamp_min(0)
    shared = inside & (entry >= 0) & (refs[page] > 1)
    flat, seq = page.flatten(), torch.arange(B, dtype=torch.int32, device="cuda").view(-1, 1).expand_as(page)
    asked = torch.zeros_like(refs).index_add_(0, flat, shared.flatten().int())
    last = torch.full_like(refs, -1).scatter_reduce_(0, flat, torch.where(shared, seq, -1).flatten(), "amax")
    keeps = (asked[page] == refs[page]) & (last[page] == seq)
    need = inside & ((entry < 0) | (shared & ~keeps))
    fits = need.sum() <= (refs == 0).sum()
    free = (refs != 0).int().sort(stable=True).indices                                       # the free pages, ascending, then the others
    new = free[(need.flatten().cumsum(0) - 1).clamp_min(0)].view_as(page)
    take, copy = need & fits, shared & ~keeps & fits
    still = refs.argmax()                                                                    # a held page, written onto itself where nothing is copied
    to, source = torch.where(copy, new, still), torch.where(copy, page, still)
    rows = torch.arange(B, device="cuda").view(-1, 1).expand_as(at)
    spare = torch.cat([table, table[:, :1]], 1)                                              # a column for what is not inside
    spare[rows, torch.where(take, at, wide)] = new.int()
    table.copy_(spare[:, :wide])
    for name in ("k", "v"):
        pages[name][to.flatten()] = pages[name][source.flatten()]
    refs.index_add_(0, flat, -copy.flatten().int())
    refs.index_add_(0, new.flatten(), take.flatten().int())
    return pages


def _fork(st):
    """Children take over their parents' pages; then some sequences are freed and some lose their last tokens."""
    pages, case = st["pages"], st["case"]
    st["meta"].copy_(st["meta0"])
    if own:
        st["cca"].pages_fork(pages, st["parent"], st["child"], st["ws"])
        st["cca"].pages_free(pages, st["keep"])
        return {n: pages[n] for n in ("refs", "table", "len")}
    P, refs, table, length = case["P"], pages["refs"], pages["table"], pages["len"]
    parent, child = st["parent"].long(), st["child"].long()
    index = torch.arange(table.shape[1], device="cuda")
    held = (length[parent] + P - 1) // P
    rows = torch.where(index < held.view(-1, 1), table[parent], -1)
    rows = torch.where((parent == child).view(-1, 1), table[child], rows)
    old = table[child]
    refs.index_add_(0, rows.long().clamp_min(0).flatten(), (rows >= 0).int().flatten())
    refs.index_add_(0, old.long().clamp_min(0).flatten(), -(old >= 0).int().flatten())
    lens = length[parent]
    table[child] = rows
    length[child] = lens
    keep = st["keep"]
    goes = (keep >= 0).view(-1, 1) & (index >= ((keep.minimum(length) + P - 1) // P).view(-1, 1)) & (table >= 0)
    refs.index_add_(0, table.long().clamp_min(0).flatten(), -goes.int().flatten())
    table.masked_fill_(goes, -1)
    length.copy_(torch.where(keep >= 0, keep.minimum(length), length))
    return {n: pages[n] for n in ("refs", "table", "len")}


def _compact(st):
    """All held pages to the front of the pool."""
    pages, case = st["pages"], st["case"]
    st["meta"].copy_(st["meta0"])
    if own:
        return {**pages, "used": st["cca"].pages_compact(pages, st["ws"])}
    refs, table = pages["refs"], pages["table"]
    n = refs.numel()
    page = torch.arange(n, device="cuda")
    held = refs > 0
    used = held.sum()
    hole, comes = ~held & (page < used), held & (page >= used)
    first = (~comes).int().sort(stable=True).indices                                         # the pages that come, ascending, before the others
    source = torch.where(hole, first[(hole.cumsum(0) - 1).clamp_min(0)], page)
    holes = (~hole).int().sort(stable=True).indices
    place = torch.where(comes, holes[(comes.cumsum(0) - 1).clamp_min(0)], page)
    for name in ("k", "v"):
        pages[name].copy_(pages[name][source])
    refs.copy_(torch.where(page < used, refs[source], 0))
    table.copy_(torch.where(table >= 0, place[table.long().clamp_min(0)].int(), table))
    return {**pages, "used": used.int().view(1)}


# -------------------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    pages, P = st["pages"], case["P"]
    if case["op"] == "append":
        return {"k": st["k"].double(), "v": st["v"].double()}
    if case["op"] in ("reserve", "compact"):
        return _moved(case, st)
    if case["op"] == "fork":
        return _passed_on(case, st)
    g, dh = case["hq"] // case["hk"], case["dh"]
    o = torch.zeros(case["B"], case["hq"], dh, dtype=torch.float64, device="cuda")
    lse = torch.full((case["B"], case["hq"]), float("-inf"), dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(case)):
        for h in range(case["hk"] if n else 0):
            own_pages = pages["table"][b, :_up(n, P)].long()
            k, v = (pages[x][own_pages, h].reshape(-1, dh)[:n].double() for x in ("k", "v"))
            s = torch.einsum("gd,rd->gr", st["q"][b, h * g:(h + 1) * g].double(), k) / math.sqrt(dh)
            o[b, h * g:(h + 1) * g] = torch.einsum("gr,rd->gd", torch.softmax(s, dim=1), v)
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(s, dim=1)
    return {"o": o, "lse": lse}


def _passed_on(case, st):
    """Who holds what after a fork and the freeing, sequence by sequence."""
    P, table, lens = case["P"], st["pages"]["table"].tolist(), st["pages"]["len"].tolist()
    before = [(row[:_up(n, P)], n) for row, n in zip(table, lens)]
    now = list(before)
    for parent, child in zip(st["parent"].tolist(), st["child"].tolist()):
        now[child] = before[parent]
    refs = [0] * st["pages"]["refs"].numel()
    for b, keep in enumerate(st["keep"].tolist()):
        row, n = now[b]
        n = n if keep < 0 else min(n, keep)
        row = row[:_up(n, P)]
        table[b], lens[b] = row + [-1] * (len(table[b]) - len(row)), n
        for page in row:
            refs[page] += 1
    return {"refs": torch.tensor(refs), "table": torch.tensor(table), "len": torch.tensor(lens)}


def _moved(case, st):
    """Where each page's numbers come from, page by page; the numbers themselves are moved as they are."""
    pages, P = st["pages"], case["P"]
    refs, table = pages["refs"].tolist(), pages["table"].tolist()
    source = list(range(len(refs)))
    if case["op"] == "compact":
        held = [p for p, n in enumerate(refs) if n > 0]
        for to, page in zip([p for p in range(len(held)) if refs[p] == 0], [p for p in held if p >= len(held)]):
            source[to] = page
    else:
        free = iter([p for p, n in enumerate(refs) if n == 0])
        window = _window(case)
        holders = {}
        for b, (i0, i1) in enumerate(window):
            for i in range(i0, i1):
                holders.setdefault(table[b][i], []).append(b)
        for b, (i0, i1) in enumerate(window):
            for i in range(i0, i1):
                page = table[b][i]
                if page < 0:
                    next(free)
                elif refs[page] > 1 and not (len(holders[page]) == refs[page] and holders[page][-1] == b):
                    source[next(free)] = page
    at = torch.tensor(source, device="cuda")
    out = {"refs": None, "table": None, "len": None, **{n: pages[n][at].double() for n in ("k", "v")}}
    return {**out, "used": None} if case["op"] == "compact" else out
