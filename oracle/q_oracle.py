"""fp64 CPU oracle of the 4-bit cache and the 4-bit weights (definitions of include/cca.h, "Cache and weights in 4 bits").

TEST INFRASTRUCTURE ONLY, like cca_oracle.py: plain definitions, one loop per index where that is the clearest, nothing shared with
the CUDA path.  Codes are whole numbers in int64, scales the bf16 numbers widened exactly.

Pins: tests/test_q_oracle.py.
"""
from __future__ import annotations

import math

import torch

F64 = torch.float64
GROUP = 32


def quantise(x):
    """(codes int64 [..., d], scales F64 [..., d / 32]) of a bf16 tensor.  The division is the definition's: fp32, to nearest."""
    g = x.detach().cpu().float().reshape(*x.shape[:-1], -1, GROUP)
    amax = g.abs().amax(-1)
    finite = torch.isfinite(amax)
    s = (amax / 7.0).to(torch.bfloat16).float()
    s = torch.where(s < torch.finfo(torch.float32).tiny, torch.zeros_like(s), s)
    s = torch.where(finite, s, torch.full_like(s, float("nan")))
    c = torch.where((s > 0)[..., None], (g / s[..., None]).round().clamp(-7, 7), torch.zeros_like(g))
    return c.to(torch.int64).reshape(x.shape), s.to(F64)


def values(codes, scales):
    return codes.to(F64) * scales.to(F64).repeat_interleave(GROUP, -1)


def _places(d):
    """For every channel of a row: (byte, shift of the sign bit, shift of the magnitude)."""
    block = min(d, 128)
    G = block // GROUP
    place = {}
    for blk in range(d // block):
        for i in range(8):
            for grp in range(G):
                for j in range(2):
                    byte = blk * (block // 2) + 2 * G * i + 2 * grp + j
                    ch = blk * block + 32 * grp + 4 * i + j
                    place[ch] = (byte, 7, 0)
                    place[ch + 2] = (byte, 6, 3)
    return [place[c] for c in range(d)]


def pack(codes):
    """Rows of codes [..., d] as bytes [..., d / 2]."""
    d = codes.shape[-1]
    out = torch.zeros(*codes.shape[:-1], d // 2, dtype=torch.int64)
    for c, (byte, s, m) in enumerate(_places(d)):
        out[..., byte] |= ((codes[..., c] < 0).to(torch.int64) << s) | (codes[..., c].abs() << m)
    return out.to(torch.uint8)


def unpack(rows):
    """pack backwards."""
    d = 2 * rows.shape[-1]
    rows = rows.cpu().to(torch.int64)
    out = torch.zeros(*rows.shape[:-1], d, dtype=torch.int64)
    for c, (byte, s, m) in enumerate(_places(d)):
        mag = (rows[..., byte] >> m) & 7
        out[..., c] = torch.where((rows[..., byte] >> s) & 1 == 1, -mag, mag)
    return out


def unpack_tiles(codes, scales, N, K):
    """(codes int64 [N, K], scales F64 [N, K / 32]) of a weight matrix's tiles."""
    n16, k128 = codes.shape[:2]
    c = unpack(codes).permute(0, 2, 1, 3).reshape(n16 * 16, k128 * 128)
    s = scales.cpu().to(F64).permute(0, 2, 1, 3).reshape(n16 * 16, k128 * 4)
    return c, s


def attention(q, k, v, lens, g):
    """q [B, h_q, d], k, v [B, h_k, R, d] -> (o [B, h_q, d], p [B, h_q, R]) over each sequence's first lens[b] rows; a sequence
    without rows gives zeros."""
    B, hq, d = q.shape
    o = torch.zeros(B, hq, d, dtype=F64)
    p = torch.zeros(B, hq, k.shape[2], dtype=F64)
    for b in range(B):
        n = int(lens[b])
        for i in range(hq if n else 0):
            s = (k[b, i // g, :n].to(F64) @ q[b, i].to(F64)) / math.sqrt(d)
            p[b, i, :n] = torch.softmax(s, 0)
            o[b, i] = p[b, i, :n] @ v[b, i // g, :n].to(F64)
    return o, p


def evict(weight, position, n, keep, recent, next_position):
    """One head's rows: list of (from, to) moves, ascending, for n cached rows."""
    if n <= keep:
        return []

    def order(r):
        w = float(weight[r])
        late = int(position[r]) >= int(next_position) - recent
        return (not late, 0.0 if late else (math.inf if math.isnan(w) else -w), not late and math.isnan(w), r)
    stay = set(sorted(range(n), key=order)[:keep])
    go = [r for r in range(keep) if r not in stay]
    come = sorted(r for r in stay if r >= keep)
    assert len(go) == len(come)
    return list(zip(come, go))
