"""The serving operators on 4-bit data, measured: attention over a latent cache held in 4 bits, rows put into that cache, eviction from
it by accumulated attention weight, and matrix-vector products with 4-bit weights.

Format (cache rows and weight rows alike): groups of 32 channels share a scale s = bf16(max|x| / 7); a channel is
c * s with a whole number c = clamp(rint(x / s), -7, 7)."""
import math

import torch

own = False

ROW_GROUP = 32


# ------------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one user, a short context, the head layout of the 16k prefill: what counts is how long the calls take to get going
        {"name": "attend_1x1k", "op": "attend", "B": 1, "S": 1024, "hq": 8, "hk": 2, "dh": 128, "ragged": False},
        # the decode benchmark's batch and context
        {"name": "attend_32x16k", "op": "attend", "B": 32, "S": 16384, "hq": 8, "hk": 2, "dh": 128, "ragged": False},
        # one long context, the training configuration's heads
        {"name": "attend_1x128k", "op": "attend", "B": 1, "S": 131072, "hq": 8, "hk": 2, "dh": 64, "ragged": False},
        # a batch of users at different points, an odd capacity, one of them with nothing cached yet, large heads
        {"name": "attend_13x5001_ragged", "op": "attend", "B": 13, "S": 5001, "hq": 4, "hk": 1, "dh": 256, "ragged": True},
        # the keys and values of one decode step's tokens
        {"name": "append_32x1", "op": "append", "B": 32, "n": 1, "S": 1000, "hk": 2, "dh": 128},
        # a prompt's keys and values handed over from the prefill
        {"name": "append_1x16k", "op": "append", "B": 1, "n": 16384, "S": 16500, "hk": 2, "dh": 128},
        # a cache at its bound: every step one row of each head has to go
        {"name": "evict_32x4k_by_1", "op": "evict", "B": 32, "S": 4097, "hk": 2, "dh": 128, "keep": 4096, "recent": 256},
        # a prompt cut down to half its rows before decoding begins
        {"name": "evict_32x16k_to_half", "op": "evict", "B": 32, "S": 16384, "hk": 2, "dh": 128, "keep": 8192, "recent": 512},
        # down-projection of the 16k prefill configuration (queries, keys and values stacked), one token
        {"name": "linear_1x1536x4096", "op": "linear", "M": 1, "N": 1536, "K": 4096, "out": "float32"},
        # its up-projection for the decode benchmark's batch
        {"name": "linear_32x4096x1024", "op": "linear", "M": 32, "N": 4096, "K": 1024, "out": "bfloat16"},
        # a wide layer, few tokens, an odd number of them and of rows
        {"name": "linear_5x16383x8192", "op": "linear", "M": 5, "N": 16383, "K": 8192, "out": "bfloat16"},
        # a fuller batch
        {"name": "linear_64x8192x8192", "op": "linear", "M": 64, "N": 8192, "K": 8192, "out": "bfloat16"},
    ]


HEADS = [(8, 2, 128), (8, 2, 64), (16, 4, 64), (4, 4, 32), (4, 1, 256), (8, 1, 64), (16, 1, 128), (4, 2, 128)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "evict", "linear", "linear"])
    if op == "linear":
        return {"op": op, "M": rng.randint(1, 64), "N": _log(rng, 64, 8192), "K": 32 * _log(rng, 2, 256), "out": rng.choice(["bfloat16", "float32"])}
    hq, hk, dh = rng.choice(HEADS)
    B = _log(rng, 1, 32)
    most = 32 * 16384 * 2 * 128 // (B * hk * dh)            # rows of a sequence that keep the case within the largest listed one
    S = _log(rng, 1, min(131072, most))
    if op == "attend":
        return {"op": op, "B": B, "S": S, "hq": hq, "hk": hk, "dh": dh, "ragged": rng.random() < 0.6}
    if op == "append":
        n = max(1, min(S // 4, 16384 // B))
        return {"op": op, "B": B, "n": n, "S": n + rng.randint(0, 300), "hk": hk, "dh": dh}
    S = max(2, min(S, 32768))
    keep = rng.randint(1, S)
    return {"op": op, "B": B, "S": S, "hk": hk, "dh": dh, "keep": keep, "recent": rng.randint(0, keep // 2)}


def _lens(case):
    """Cached rows of each sequence: all full, or spread down from the full one with one empty sequence among three or more."""
    B, S = case["B"], case["S"]
    if not case.get("ragged"):
        return [S] * B
    lens = [max(0, S * (B - b) // B - (b % 3)) for b in range(B)]
    if B >= 3:
        lens[B // 2] = 0
    return lens


def _row_bytes(dh):
    return 2 * (dh // 2 + dh // 16)          # key and value: codes and scales


def work(case):
    if case["op"] == "attend":
        rows = sum(_lens(case))
        return {"bytes": rows * case["hk"] * (_row_bytes(case["dh"]) + 8) + 4 * case["B"] * case["hq"] * case["dh"],
                "flops": 4 * rows * case["hq"] * case["dh"]}
    if case["op"] == "append":
        rows = case["B"] * case["n"] * case["hk"]
        return {"bytes": rows * (4 * case["dh"] + _row_bytes(case["dh"]) + 8 + 8 * case["dh"]), "flops": 6 * rows * case["dh"]}
    if case["op"] == "evict":
        S, keep, recent = case["S"], case["keep"], case["recent"]
        tail = S - keep
        late = min(recent, tail)
        moved = late + (tail - late) * (keep - recent) / max(1, S - recent)   # expected: rows behind `keep` that stay
        heads = case["B"] * case["hk"]
        return {"bytes": heads * (8 * S + moved * (2 * _row_bytes(case["dh"]) + 8)), "flops": heads * S}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": N * K // 2 + N * K // 16 + 2 * M * K + (4 if case["out"] == "float32" else 2) * M * N, "flops": 2 * M * N * K}


# ---------------------------------------------------------------------------------------------------------- inputs of a case
def _quantise(x):
    """Codes (fp32 holding whole numbers) and scales (bf16) of x [..., d]."""
    g = x.float().unflatten(-1, (-1, ROW_GROUP))
    s = (g.abs().amax(-1, keepdim=True) / 7).bfloat16()
    c = torch.where(s > 0, (g / s.float()).round().clamp(-7, 7), torch.zeros_like(g))
    return c.flatten(-2), s.squeeze(-1)


def _pack(c):
    """Whole numbers -7..7 [..., d] as bytes [..., d / 2], two in a byte in sign and magnitude, in the order the cache keeps them."""
    d = c.shape[-1]
    block = min(d, 128)
    c = c.to(torch.int32).unflatten(-1, (d // block, block // 32, 8, 2, 2))
    sign, mag = (c < 0).int(), c.abs()
    byte = (sign[..., 0, :] << 7) | mag[..., 0, :] | (sign[..., 1, :] << 6) | (mag[..., 1, :] << 3)
    return byte.transpose(-3, -2).flatten(-4).to(torch.uint8)


def _handle(hq, hk, dh):
    from paper_2510_04476_b200.binding import CCA
    return CCA(d_model=hq * dh, n_q_heads=hq, n_kv_heads=hk, head_dim=dh)


def _empty_cache(B, S, hk, dh):
    """A cache's tensors; what counts up while it is used (weight, position, len) lies in one buffer."""
    n = B * hk * S
    meta = torch.zeros(2 * n + B, dtype=torch.int32, device="cuda")
    cache = {"weight": meta[:n].view(torch.float32).view(B, hk, S), "position": meta[n:2 * n].view(B, hk, S), "len": meta[2 * n:]}
    for name in ("k", "v"):
        cache[name + "_codes"] = torch.zeros(B, hk, S, dh // 2, dtype=torch.uint8, device="cuda")
        cache[name + "_scales"] = torch.zeros(B, hk, S, dh // 32, dtype=torch.bfloat16, device="cuda")
    return cache, meta


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    st = {"case": case}
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = normal(M, K).bfloat16()
        codes, scales = _quantise((0.02 * normal(N, K)).bfloat16())
        st["codes"], st["scales"] = codes.to(torch.int8), scales
        # laid out once: 16 rows by 128 columns in a tile, what is behind the last row and column is zero
        n16, k128 = (N + 15) // 16, (K + 127) // 128
        wide = torch.zeros(n16 * 16, k128 * 128, device="cuda")
        wide[:N, :K] = codes
        sw = torch.zeros(n16 * 16, k128 * 4, dtype=torch.bfloat16, device="cuda")
        sw[:N, :K // 32] = scales
        st["packed"] = {"codes": _pack(wide.view(n16 * 16, k128, 128)).view(n16, 16, k128, 64).transpose(1, 2).contiguous(),
                        "scales": sw.view(n16, 16, k128, 4).transpose(1, 2).contiguous(), "N": N, "K": K}
        if own:
            st["cca"] = _handle(4, 4, 64)
        return st

    B, S, hk, dh = case["B"], case["S"], case["hk"], case["dh"]
    cache, meta = _empty_cache(B, S, hk, dh)
    st["cache"], st["meta"] = cache, meta
    if case["op"] == "append":
        st["k"], st["v"] = normal(B, case["n"], hk, dh).bfloat16(), normal(B, case["n"], hk, dh).bfloat16()
        cache["len"].copy_(torch.randint(0, S - case["n"] + 1, (B,), generator=gen, device="cuda"))
        cache["weight"].fill_(0.5)           # what earlier rows left behind in these places
        st["position"] = cache["len"] * 3 + 5
        if own:
            st["cca"] = _handle(hk, hk, dh)
        return st

    if case["op"] == "evict":
        for name in ("k", "v"):      # rows are moved as they are: any bytes will do
            cache[name + "_codes"].copy_(torch.randint(0, 256, cache[name + "_codes"].shape, generator=gen, device="cuda", dtype=torch.uint8))
            cache[name + "_scales"].copy_(normal(*cache[name + "_scales"].shape).abs())
        cache["weight"].copy_((1.5 * normal(B, hk, S)).exp())          # a few rows hold most of the weight
        # earlier evictions have mixed the first rows, the later ones came in order
        mixed = 3 * S // 4
        cache["position"].copy_(torch.arange(S, device="cuda", dtype=torch.int32).expand(B, hk, S))
        cache["position"][..., :mixed] = torch.rand(B, hk, mixed, generator=gen, device="cuda").argsort(-1).int()
        cache["len"].fill_(S)
        st["next"] = torch.full((B,), S, dtype=torch.int32, device="cuda")
        st["meta0"] = meta.clone()
        if own:
            st["cca"] = _handle(hk, hk, dh)
            st["ws"] = st["cca"].alloc_qcache_workspace(B, S)
        return st

    hq = case["hq"]
    # normalised queries and keys, as the block makes them: logits of unit variance; the keys' scales differ by head
    st["q"] = torch.nn.functional.normalize(normal(B, hq, dh), dim=-1).mul(math.sqrt(dh)).bfloat16()
    codes, scales = [], []
    for name in ("k", "v"):
        x = normal(B, hk, S, dh)
        if name == "k":
            x = torch.nn.functional.normalize(x, dim=-1).mul_(math.sqrt(dh)).mul_(torch.linspace(0.7, 1.5, hk, device="cuda").view(1, hk, 1, 1))
        c, s = _quantise(x.bfloat16())
        cache[name + "_codes"].copy_(_pack(c))
        cache[name + "_scales"].copy_(s)
        codes.append(c.to(torch.int8))
        scales.append(s)
    st["codes"], st["scales"] = codes, scales
    cache["weight"].copy_(torch.rand(B, hk, S, generator=gen, device="cuda"))
    cache["len"].copy_(torch.tensor(_lens(case), dtype=torch.int32, device="cuda"))
    if own:
        st["cca"] = _handle(hq, hk, dh)
        st["ws"] = st["cca"].alloc_qcache_workspace(B, S)
    return st


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(st):
    return {"attend": _attend, "append": _append, "evict": _evict, "linear": _linear}[st["case"]["op"]](st)


def _values(codes, scales):
    return (codes.float().unflatten(-1, (-1, ROW_GROUP)) * scales.float().unsqueeze(-1)).flatten(-2)


def _attend(st):
    """The new tokens' queries over the cached rows; every row's weight grows by what it was given."""
    q, cache, case = st["q"], st["cache"], st["case"]
    if own:
        o = st["cca"].qcache_attention(q, cache, case["S"], st["ws"])
        return {"o": o, "weight": cache["weight"]}
    hk, dh, S = case["hk"], case["dh"], case["S"]
    k, v = (_values(c, s) for c, s in zip(st["codes"], st["scales"]))
    s = q.float().unflatten(1, (hk, -1)) @ k.transpose(-1, -2) / math.sqrt(dh)                # [B, hk, g, S]
    there = torch.arange(S, device=q.device) < cache["len"].view(-1, 1, 1, 1)
    s = s.masked_fill(~there, float("-inf"))
    e = torch.exp(s - s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)).masked_fill(~there, 0.0)
    p = e / e.sum(-1, keepdim=True).clamp_min(1e-30)
    cache["weight"] += p.sum(2)
    return {"o": (p @ v).flatten(1, 2).bfloat16(), "weight": cache["weight"]}


def _append(st):
    """New rows into the cache, and the values that it now holds for them."""
    cache, case = st["cache"], st["case"]
    if own:
        st["cca"].qcache_append(cache, st["k"], st["v"], st["position"])
        k, v = st["cca"].qcache_read(cache, case["n"])
        return {"k": k, "v": v, "weight": cache["weight"], "position": cache["position"]}
    n, hk, dev = case["n"], case["hk"], st["k"].device
    row = (cache["len"].view(-1, 1) + torch.arange(n, device=dev)).long()                  # [B, n]
    at = row.unsqueeze(1).expand(-1, hk, -1)
    got = []
    for name in ("k", "v"):
        c, s = _quantise(st[name].transpose(1, 2))                                            # [B, hk, n, dh]
        codes, scales = cache[name + "_codes"], cache[name + "_scales"]
        codes.scatter_(2, at.unsqueeze(-1).expand(-1, -1, -1, codes.shape[-1]), _pack(c))
        scales.scatter_(2, at.unsqueeze(-1).expand(-1, -1, -1, scales.shape[-1]), s)
        got.append(_values(c, s).transpose(1, 2).contiguous())
    cache["weight"].scatter_(2, at, torch.zeros_like(at, dtype=torch.float32))
    cache["position"].scatter_(2, at, (st["position"].view(-1, 1, 1) + torch.arange(n, device=dev, dtype=torch.int32)).expand(-1, hk, -1).int())
    return {"k": got[0], "v": got[1], "weight": cache["weight"], "position": cache["position"]}


def _evict(st):
    """Every head down to its `keep` rows: the newest ones and those with the most weight. A row behind `keep` that stays moves into the
    place of one that goes, both in ascending order. Rows are moved as they are, so their bytes come back whole."""
    cache, case = st["cache"], st["case"]
    st["meta"].copy_(st["meta0"])            # weights, positions and lengths as the steps before left them
    if own:
        st["cca"].qcache_evict(cache, case["keep"], case["recent"], st["next"], case["S"], st["ws"])
        return cache
    S, keep = case["S"], case["keep"]
    weight, position, length = cache["weight"], cache["position"], cache["len"]
    row = torch.arange(S, device=weight.device)
    there = row < length.view(-1, 1, 1)
    late = position >= (st["next"] - case["recent"]).view(-1, 1, 1)
    key = weight.masked_fill(late, float("inf")).masked_fill(~there, float("-inf"))
    order = key.sort(dim=-1, descending=True, stable=True).indices
    stays = torch.zeros_like(there.expand_as(key)).scatter(2, order[..., :keep], True) | (length <= keep).view(-1, 1, 1)
    hole, comes = ~stays & (row < keep), stays & (row >= keep) & there & (length > keep).view(-1, 1, 1)
    first = (~comes).long().sort(dim=-1, stable=True).indices                                # rows that come, ascending, before the others
    source = torch.where(hole, first.gather(2, (hole.long().cumsum(-1) - 1).clamp_min(0)), row)
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        t = cache[name]
        t.copy_(t.gather(2, source.unsqueeze(-1).expand_as(t)))
    weight.copy_(weight.gather(2, source))
    position.copy_(position.gather(2, source))
    length.clamp_(max=keep)
    return cache


def _linear(st):
    """Tokens through a layer with 4-bit weights."""
    dtype = getattr(torch, st["case"]["out"])
    if own:
        return st["cca"].qlinear(st["packed"], st["x"], out_dtype=dtype)
    return (st["x"].float() @ _values(st["codes"], st["scales"]).t()).to(dtype)


# -------------------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "linear":
        w = st["codes"].double() * st["scales"].double().repeat_interleave(ROW_GROUP, 1)
        return torch.einsum("mk,nk->mn", st["x"].double(), w)
    cache = st["cache"]
    if case["op"] == "append":
        out = {"weight": torch.full_like(cache["weight"], 0.5, dtype=torch.float64), "position": None}
        for b, first in enumerate(cache["len"].tolist()):
            out["weight"][b, :, first:first + case["n"]] = 0
        for name in ("k", "v"):
            x = st[name].double().view(*st[name].shape[:-1], -1, ROW_GROUP)
            scale = (x.abs().max(-1, keepdim=True).values / 7).to(torch.bfloat16).double()
            out[name] = (torch.clamp(torch.round(x / scale.clamp_min(1e-300)), -7, 7) * scale).view(st[name].shape)
        return out
    if case["op"] == "evict":
        weight, position = cache["weight"].double().cpu().numpy(), cache["position"].cpu().numpy()
        S, keep, recent = case["S"], case["keep"], case["recent"]
        if keep < S:
            for b in range(weight.shape[0]):
                for h in range(weight.shape[1]):
                    w, p = weight[b, h], position[b, h]
                    rank = sorted(range(S), key=lambda r: (p[r] < S - recent, -w[r] if p[r] < S - recent else 0.0, r))[:keep]
                    stay = set(rank)
                    holes = [r for r in range(keep) if r not in stay]
                    w[holes] = w[sorted(r for r in rank if r >= keep)]
        return {"weight": torch.from_numpy(weight), "position": None, "len": None, "k_codes": None, "v_codes": None, "k_scales": None, "v_scales": None}
    lens, g, dh = _lens(case), case["hq"] // case["hk"], case["dh"]
    o = torch.zeros(case["B"], case["hq"], dh, dtype=torch.float64, device="cuda")
    weight = cache["weight"].double()
    for b, n in enumerate(lens):
        for h in range(case["hk"] if n else 0):
            k, v = (c[b, h, :n].double() * s[b, h, :n].double().repeat_interleave(ROW_GROUP, 1) for c, s in zip(st["codes"], st["scales"]))
            p = torch.softmax(torch.einsum("gd,rd->gr", st["q"][b, h * g:(h + 1) * g].double(), k) / math.sqrt(dh), dim=1)
            o[b, h * g:(h + 1) * g] = torch.einsum("gr,rd->gd", p, v)
            weight[b, h, :n] += p.sum(0)
    return {"o": o, "weight": weight}
