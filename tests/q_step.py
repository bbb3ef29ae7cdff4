"""One decode step on 4-bit weights and a 4-bit cache against the fp64 oracle, from the same cached rows on both sides.  Nothing of a test
runner is needed here."""
import torch

from oracle import cca_oracle as O
from oracle import q_oracle as Q
from tests.util import check_close


def dequantised(w):
    """The block's weights as the 4-bit format holds them."""
    return {n: Q.values(*Q.quantise(t)) if n in ("w_qk", "w_v1", "w_v2", "w_o") else t for n, t in w.items()}


def cached_rows(state, n):
    """The first n cached keys and values, [B, n, h_k, d_h] F64 each, decoded from the cache's bytes."""
    rows = []
    for x in ("k", "v"):
        codes, scales = (state["cache"][x + part][:, :, :n].contiguous() for part in ("_codes", "_scales"))
        rows.append(Q.values(Q.unpack(codes), scales.cpu()).transpose(1, 2))
    return rows


def check_step(cca, cfg, weights64, state, ref_state, x, max_len, workspace, packed):
    """One step on both sides.  The new row's codes are within half a step of the oracle's key and value (plus 1e-2 + 1e-2 |ref| for the
    arithmetic before the rounding); output and weights are those of attention over the rows that the GPU cached.  Advances `state`."""
    cache = state["cache"]
    n = int(cache["len"][0])
    before = cached_rows(state, n)
    ref_state["k"], ref_state["v"] = before
    weight = cache["weight"].clone()
    out = cca.decode_step_q(packed, x.cuda(), state, max_len, workspace)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    O.decode_step(cfg, weights64, ref_state, x)
    after = cached_rows(state, n + 1)
    for name, old, new in zip("kv", before, after):
        assert torch.equal(new[:, :n], old), name
        step = cache[name + "_scales"][:, :, n].cpu().double().repeat_interleave(Q.GROUP, -1)
        want = ref_state[name][:, n]
        assert ((new[:, n] - want).abs() <= step / 2 + 1e-2 + 1e-2 * want.abs()).all(), name
    o, p = Q.attention(ref_state["q_last"], *(r.transpose(1, 2) for r in after), [n + 1] * x.shape[0], cfg.g)
    check_close("out", out, o.reshape(x.shape[0], -1) @ weights64["w_o"].t())
    weight[:, :, n] = 0                                # a new row starts from nothing
    check_close("weight", (cache["weight"] - weight)[:, :, :n + 1].cpu(), p.reshape(p.shape[0], cfg.n_kv_heads, cfg.g, -1).sum(2))
    state["pos"] += 1
    cache["len"] += 1
