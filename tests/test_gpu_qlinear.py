"""Products with 4-bit weights, and the decode step on them, against the fp64 oracle.

Tolerance of a product: the codes are exact operands and every product of one with a bf16 number is exact in fp32; an output is a sum of 32
products per group, one scaling per group, and a chain of at most K / 256 + 1 groups per warp and 8 warps, each add off by at
most 2^-23 of the terms' magnitudes (adds may truncate): |err| <= 2^-23 (K / 256 + 48) sum |x w|, plus 2^-8 |y| for a bf16 output.

From 9 tokens on the products of 512 columns are a chain of 64 adds on the tensor cores (two exact parts of each weight, 16 products an
add), each off by at most 2^-23 of the sum so far, which after i adds has i / 64 of the chunk's sum |x w| (terms of one distribution): 33 times
2^-23 of that in all.  The K / 512 chunks and 8 ranks are added in fp32, 2^-24 of the sum |x w| an add:
|err| <= 2^-23 (33 + K / 1024 + 4) sum |x w|, below the bound above."""
import pytest
import torch

from oracle import cca_oracle as O
from oracle import q_oracle as Q
from paper_2510_04476_b200 import synth
from tests.util import check_close, oracle_cfg, to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cca():
    from paper_2510_04476_b200.binding import CCA
    h = CCA(d_model=256, n_q_heads=4, n_kv_heads=4, head_dim=64)
    yield h
    h.close()


def _weights(N, K, seed):
    gen = torch.Generator().manual_seed(seed)
    w = (0.05 * torch.randn(N, K, generator=gen) * torch.exp(torch.randn(N, 1, generator=gen))).bfloat16()
    return w, gen


def _check(y, x, w64, K):
    x = x.double()
    ref, mag = x @ w64.t(), x.abs() @ w64.abs().t()
    tol = 2.0 ** -23 * (K / 256 + 48) * mag + 1e-35
    if y.dtype is torch.bfloat16:
        tol = tol + 2.0 ** -8 * ref.abs()
    err = (y.cpu().double() - ref).abs()
    assert y.shape == ref.shape and (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("N,K", [(1, 32), (15, 96), (16, 128), (17, 160), (64, 256), (100, 1056), (33, 4096)])
def test_pack(cca, N, K):
    w, _ = _weights(N, K, N + K)
    w[0, 0] = 0
    packed = cca.qlinear_pack(w.cuda())
    c, s = Q.unpack_tiles(packed["codes"], packed["scales"], N, K)
    cr, sr = Q.quantise(w)
    assert torch.equal(c[:N, :K], cr) and torch.equal(s[:N, :K // 32], sr)
    assert not c[N:].any() and not c[:, K:].any() and not s[N:].any() and not s[:, K // 32:].any()


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 130])
@pytest.mark.parametrize("N,K", [(1, 32), (17, 160), (96, 1024), (250, 4128)])
def test_product(cca, M, N, K):
    w, gen = _weights(N, K, N + K)
    packed = cca.qlinear_pack(w.cuda())
    w64 = Q.values(*Q.quantise(w))
    x = torch.randn(M, K, generator=gen).bfloat16()
    for dtype in (torch.float32, torch.bfloat16):
        _check(cca.qlinear(packed, x.cuda(), out_dtype=dtype), x, w64, K)
    assert cca.last_status() == 0


@pytest.mark.parametrize("M,N,K", [(1, 1536, 4096), (32, 4096, 1024), (5, 4095, 8192), (64, 2050, 8192)])
def test_product_of_a_layer(cca, M, N, K):
    w, gen = _weights(N, K, 5)
    packed = cca.qlinear_pack(w.cuda())
    x = torch.randn(M, K, generator=gen).bfloat16()
    y = cca.qlinear(packed, x.cuda(), out_dtype=torch.float32)
    _check(y, x, Q.values(*Q.quantise(w)), K)
    assert torch.equal(y, cca.qlinear(packed, x.cuda(), out_dtype=torch.float32))


@pytest.mark.parametrize("M", [1, 5, 8, 9])
@pytest.mark.parametrize("N,K", [(9473, 32), (9500, 160), (9487, 1024), (10001, 2080), (9600, 3136), (9472, 5120), (9473, 8192), (9473, 8224)])
def test_product_of_many_rows(cca, M, N, K):
    """Many rows and long inner dimensions, ragged ends."""
    w, gen = _weights(N, K, N + K)
    packed = cca.qlinear_pack(w.cuda())
    x = torch.randn(M, K, generator=gen).bfloat16()
    w64 = Q.values(*Q.quantise(w))
    for dtype in (torch.float32, torch.bfloat16):
        _check(cca.qlinear(packed, x.cuda(), out_dtype=dtype), x, w64, K)


@pytest.mark.parametrize("scale", [1e-12, 1e12])
def test_product_of_small_and_large_inputs(cca, scale):
    w, gen = _weights(64, 512, 6)
    packed = cca.qlinear_pack(w.cuda())
    x = (scale * torch.randn(3, 512, generator=gen)).bfloat16()
    _check(cca.qlinear(packed, x.cuda(), out_dtype=torch.float32), x, Q.values(*Q.quantise(w)), 512)


@pytest.mark.parametrize("M", [3, 9, 40])
def test_product_without_the_tensor_core_kernels(cca, M):
    w, gen = _weights(100, 1056, 8)
    packed = cca.qlinear_pack(w.cuda())
    x = torch.randn(M, 1056, generator=gen).bfloat16()
    before = cca.set_impl(0)
    try:
        _check(cca.qlinear(packed, x.cuda(), out_dtype=torch.float32), x, Q.values(*Q.quantise(w)), 1056)
    finally:
        cca.set_impl(before)


@pytest.mark.parametrize("M,N,K", [(9, 150, 32768), (64, 40, 65536), (33, 9500, 8192)])
def test_product_of_numbers_of_one_sign_in_long_rows(cca, M, N, K):
    """Every add of a chain is cut off to the same side: the bound of chunks of 64 adds, with 8 more for terms that are not all alike."""
    gen = torch.Generator().manual_seed(K)
    w = (0.05 * torch.rand(N, K, generator=gen)).bfloat16()
    x = torch.rand(M, K, generator=gen).bfloat16()
    y = cca.qlinear(cca.qlinear_pack(w.cuda()), x.cuda(), out_dtype=torch.float32).cpu().double()
    ref = x.double() @ Q.values(*Q.quantise(w)).t()
    assert ((y - ref).abs() <= 2.0 ** -23 * (45 + K / 1024) * ref).all(), float(((y - ref).abs() / ref).max() * 2 ** 23)
    assert cca.last_status() == 0


def test_product_of_more_rows_than_a_grid_dimension_has_blocks(cca):
    N, K, M = 65535 * 128 + 1, 32, 9
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.randn(N, K, generator=gen, device="cuda").bfloat16()
    x = torch.randn(M, K, generator=gen, device="cuda").bfloat16()
    y = cca.qlinear(cca.qlinear_pack(w), x, out_dtype=torch.float32)
    for part in (slice(0, 200), slice(N - 200, N)):
        _check(y[:, part], x.cpu(), Q.values(*Q.quantise(w[part].cpu())), K)
    assert cca.last_status() == 0


def test_a_nan_input_touches_its_own_token_alone(cca):
    w, gen = _weights(40, 160, 6)
    packed = cca.qlinear_pack(w.cuda())
    x = torch.randn(9, 160, generator=gen).bfloat16()
    x[3, 100] = float("nan")
    y = cca.qlinear(packed, x.cuda(), out_dtype=torch.float32)
    assert torch.isnan(y[3]).all() and torch.isfinite(y[[0, 1, 2, 4, 5, 6, 7, 8]]).all()


def test_given_output_and_refusals(cca):
    from paper_2510_04476_b200.binding import CcaError
    w, gen = _weights(24, 64, 7)
    packed = cca.qlinear_pack(w.cuda())
    x = torch.randn(2, 64, generator=gen).bfloat16().cuda()
    out = torch.empty(2, 24, dtype=torch.float32, device="cuda")
    assert cca.qlinear(packed, x, out=out) is out
    assert torch.equal(out, cca.qlinear(packed, x, out_dtype=torch.float32))
    for bad in (lambda: cca.qlinear(packed, x[:, :32].contiguous()), lambda: cca.qlinear(packed, x.float()), lambda: cca.qlinear(packed, x.cpu()),
                lambda: cca.qlinear(packed, x, out=out[:1]), lambda: cca.qlinear(packed, x, out_dtype=torch.float16),
                lambda: cca.qlinear({**packed, "N": 40}, x), lambda: cca.qlinear(packed, x[:0]),
                lambda: cca.qlinear_pack(w[:, :48].contiguous().cuda()), lambda: cca.qlinear_pack(w.float().cuda())):
        with pytest.raises(CcaError):
            bad()


# ------------------------------------------------------------------------------------------------ the decode step
def S_(name, B, S, E, hq, hk, dh, **kw):
    return synth.Shape(name, B, S, E, hq, hk, dh, seed=sum(map(ord, name)) % 1000, **kw)


def _dequantised(w):
    return {n: Q.values(*Q.quantise(t)) if n in ("w_qk", "w_v1", "w_v2", "w_o") else t for n, t in w.items()}


def _rows(cca, state, n):
    """The first n cached rows as the oracle keeps them, [B, n, hk, dh] F64, decoded from the cache's bytes."""
    return [Q.values(Q.unpack(state["cache"][x + "_codes"][:, :, :n].contiguous()),
                     state["cache"][x + "_scales"][:, :, :n].contiguous().cpu()).transpose(1, 2) for x in ("k", "v")]


def _check_step(cca, cfg, wd, state, ostate, x, max_len, ws, packed):
    """One step on both sides from the same cached rows.  The new row: its codes are within half a step of the oracle's key and value
    (plus 1e-2 + 1e-2 |ref| for the arithmetic before the rounding); the output: from the row that the GPU cached."""
    n = int(state["cache"]["len"][0])
    k0, v0 = _rows(cca, state, n)
    ostate["k"], ostate["v"] = k0, v0
    weight = state["cache"]["weight"].clone()
    out = cca.decode_step_q(packed, x.cuda(), state, max_len, ws)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    O.decode_step(cfg, wd, ostate, x)
    k1, v1 = _rows(cca, state, n + 1)
    assert torch.equal(k1[:, :n], k0) and torch.equal(v1[:, :n], v0)
    for got, ref, name in ((k1[:, n], ostate["k"][:, n], "k"), (v1[:, n], ostate["v"][:, n], "v")):
        step = state["cache"][name + "_scales"][:, :, n].cpu().double().repeat_interleave(32, -1)
        assert ((got - ref).abs() <= step / 2 + 1e-2 + 1e-2 * ref.abs()).all(), name
    o, p = Q.attention(ostate["q_last"], k1.transpose(1, 2), v1.transpose(1, 2), [n + 1] * x.shape[0], cfg.g)
    ref = o.reshape(x.shape[0], -1) @ wd["w_o"].t()
    check_close("out", out, ref)
    weight[:, :, n] = 0                              # a new row starts from nothing
    grown = (state["cache"]["weight"] - weight)[:, :, :n + 1].cpu()
    check_close("weight", grown, p.reshape(p.shape[0], cfg.n_kv_heads, cfg.g, -1).sum(2))
    state["pos"] += 1
    state["cache"]["len"] += 1


STEPS = [
    S_("q_dh32", 3, 12, 256, 4, 2, 32),
    S_("q_dh64_g4", 2, 20, 512, 8, 2, 64),
    S_("q_dh128_g4", 2, 17, 1024, 4, 1, 128),
    S_("q_dh256_g2", 2, 9, 1024, 4, 2, 256),
    S_("q_dh256_g16", 1, 6, 4096, 16, 1, 256),
    S_("q_mha", 2, 9, 256, 4, 4, 64, flags=0),
    S_("q_g16", 1, 9, 1024, 16, 1, 64),
    S_("q_k3_k4", 2, 9, 512, 8, 2, 64, k_seq=3, k_ch=4),
    S_("q_k1_k1", 2, 5, 512, 8, 2, 64, k_seq=1, k_ch=1),
    S_("q_no_shift", 2, 5, 512, 8, 2, 64, flags=63 & ~8),
    S_("q_no_conv2", 2, 5, 512, 8, 2, 64, flags=63 & ~2),
    S_("q_batch_over_32", 37, 4, 256, 4, 2, 64),
    S_("q_wide", 2, 3, 4096, 32, 32, 128),
]


@pytest.mark.parametrize("sh", STEPS, ids=lambda s: s.name)
def test_decode_step_from_an_empty_cache(sh):
    from paper_2510_04476_b200.binding import CCA
    t = synth.make_inputs(sh, want_dout=False)
    cfg, dev, wd = oracle_cfg(sh), to_device(t), _dequantised(t)
    cca = CCA.from_shape(sh)
    packed = cca.pack_weights_q(dev)
    S_max = sh.S + 2
    state, ostate = cca.new_decode_state_q(sh.B, S_max), O.decode_init(cfg, sh.B)
    ws = cca.alloc_decode_workspace_q(sh.B, S_max)
    ws.fill_(255)
    for tok in range(sh.S):
        _check_step(cca, cfg, wd, state, ostate, t["x"][:, tok], tok + 1, ws, packed)
    if state["qk0_hist"].numel():
        check_close("qk0_hist", state["qk0_hist"], ostate["qk0_hist"])
    assert torch.equal(state["x_prev"].cpu(), t["x"][:, sh.S - 1])
    assert not state["cache"]["k_codes"][:, :, sh.S:].any()
    cca.close()


def test_prefill_then_decode_with_eviction():
    """All of it together: a prompt through the forward, its keys and values into the 4-bit cache, decode steps on 4-bit weights that
    gather weights, eviction down to a bound after every step; the position runs past the cache's capacity."""
    from paper_2510_04476_b200.binding import CCA
    sh = S_("q_together", 2, 400, 512, 8, 2, 64)
    S0, keep, S_max = 380, 100, 384
    t = synth.make_inputs(sh, want_dout=False)
    cfg, dev, wd = oracle_cfg(sh), to_device(t), _dequantised(t)
    cca = CCA.from_shape(sh)
    packed = cca.pack_weights_q(dev)
    x0 = dev["x"][:, :S0].contiguous()
    ws0 = cca.alloc_workspace(sh.B, S0, False)
    cca.forward(dev, x0, ws0)
    state = cca.new_decode_state_q(sh.B, S_max)
    cca.decode_state_from_prefill_q(x0, ws0, state)
    state["pos"].fill_(S0)
    state["cache"]["len"].fill_(S0)
    _, I = O.forward(cfg, t, t["x"][:, :S0])
    for name in ("k", "v"):
        got = Q.values(Q.unpack(state["cache"][name + "_codes"][:, :, :S0].contiguous()), state["cache"][name + "_scales"][:, :, :S0].contiguous().cpu())
        step = state["cache"][name + "_scales"][:, :, :S0].cpu().double().repeat_interleave(32, -1)
        ref = I[name].transpose(1, 2)
        assert ((got - ref).abs() <= step / 2 + 1e-2 + 1e-2 * ref.abs()).all()
    ostate = O.decode_state_after_prefill(cfg, I, S0)
    ws = cca.alloc_decode_workspace_q(sh.B, S_max)
    qws = cca.alloc_qcache_workspace(sh.B, S_max)
    for tok in range(S0, sh.S):
        if tok == S0:                        # the history went through bf16 weights in the prefill on both sides
            check_close("qk0_hist", state["qk0_hist"], ostate["qk0_hist"])
        _check_step(cca, cfg, wd, state, ostate, t["x"][:, tok], S_max, ws, packed)
        cca.qcache_evict(state["cache"], keep, 16, state["pos"], S_max, qws)
        assert state["cache"]["len"].tolist() == [keep, keep]
    assert int(state["pos"][0]) > S_max
    late = state["cache"]["position"][:, :, :keep].sort(-1).values[..., -16:].cpu()
    assert torch.equal(late, torch.arange(sh.S - 16, sh.S, dtype=torch.int32).expand_as(late))
    cca.close()


def test_decode_step_in_a_graph_and_a_sequence_that_is_full():
    from paper_2510_04476_b200.binding import CCA
    sh = S_("q_graph", 3, 6, 512, 8, 2, 64)
    t = synth.make_inputs(sh, want_dout=False)
    dev = to_device(t)
    cca = CCA.from_shape(sh)
    packed = cca.pack_weights_q(dev)
    xs = [dev["x"][:, i].contiguous() for i in range(sh.S)]
    ws = cca.alloc_decode_workspace_q(sh.B, 8)

    def fresh():
        s = cca.new_decode_state_q(sh.B, 8)
        for i in range(3):
            cca.decode_step_q(packed, xs[i], s, 8, ws)
            s["pos"] += 1
            s["cache"]["len"] += 1
        return s

    a, b = fresh(), fresh()
    x, out = xs[3].clone(), torch.empty_like(xs[3])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cca.decode_step_q(packed, x, a, 8, ws, out=out)
        a["pos"] += 1
        a["cache"]["len"] += 1
    for i in (3, 4, 5):
        x.copy_(xs[i])
        g.replay()
        want = cca.decode_step_q(packed, xs[i], b, 8, ws)
        b["pos"] += 1
        b["cache"]["len"] += 1
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    for n in a["cache"]:
        assert torch.equal(a["cache"][n], b["cache"][n]), n
    assert cca.last_status() == 0
    # the second sequence is full, the third has no position: nothing of theirs is written
    b["cache"]["len"].copy_(torch.tensor([6, 8, 6], dtype=torch.int32))
    b["pos"].copy_(torch.tensor([6, 8, -1], dtype=torch.int32))
    before = {n: v.clone() for n, v in {**b["cache"], "h": b["qk0_hist"], "x": b["x_prev"]}.items()}
    cca.decode_step_q(packed, xs[0], b, 8, ws)
    torch.cuda.synchronize()
    assert cca.last_status() == 121
    for n, v in {**b["cache"], "h": b["qk0_hist"], "x": b["x_prev"]}.items():
        assert torch.equal(v[1:], before[n][1:]), n
    assert torch.equal(b["x_prev"][0], xs[0][0])
    cca.close()


def test_decode_step_refusals():
    from paper_2510_04476_b200.binding import CCA, CcaError
    sh = S_("q_args", 2, 4, 256, 4, 2, 64)
    dev = to_device(synth.make_inputs(sh, want_dout=False))
    cca = CCA.from_shape(sh)
    packed = cca.pack_weights_q(dev)
    state = cca.new_decode_state_q(2, 8)
    ws = cca.alloc_decode_workspace_q(2, 8)
    x = dev["x"][:, 0].contiguous()
    nc = CCA.from_shape(sh.replace(causal=0))
    for bad in (lambda: cca.decode_step_q(packed, x, state, 9, ws), lambda: cca.decode_step_q(packed, x, state, 8, ws[:400]),
                lambda: cca.decode_step_q(packed, x[:1], state, 8, ws), lambda: cca.decode_step_q({**packed, "w_o": packed["w_vp"]}, x, state, 8, ws),
                lambda: cca.decode_step_q({**packed, "temp": None}, x, state, 8, ws),
                lambda: cca.decode_step_q({**packed, "conv1_w": packed["conv0_w"]}, x, state, 8, ws),
                lambda: nc.decode_step_q(packed, x, state, 8, ws),
                lambda: cca.decode_state_from_prefill_q(dev["x"], ws[:1000], state)):
        with pytest.raises(CcaError):
            bad()
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    nc.close()
    cca.close()
