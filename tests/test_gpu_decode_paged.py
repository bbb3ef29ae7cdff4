"""The decode step on a cache in pages, and a run of all that belongs to it: a prefill into pages, its sequence forked, steps that go
different ways, sequences freed, the pool compacted under them.  Tolerance as everywhere: max |err| <= 1e-2 + 1e-2 |ref|."""
import pytest
import torch

from oracle import cca_oracle as O
from paper_2510_04476_b200 import synth
from tests.test_gpu_pages import ints
from tests.util import check_close, oracle_cfg, to_device

pytestmark = pytest.mark.gpu


def S_(name, B, S, E, hq, hk, dh, **kw):
    return synth.Shape(name, B, S, E, hq, hk, dh, seed=sum(map(ord, name)) % 1000, **kw)


def _cca(sh):
    from paper_2510_04476_b200.binding import CCA
    return CCA.from_shape(sh)


SHAPES = [S_("pg_dh32", 3, 20, 256, 4, 2, 32), S_("pg_dh64_g4", 2, 40, 512, 8, 2, 64), S_("pg_dh128_g4", 2, 33, 1024, 4, 1, 128),
          S_("pg_mha", 2, 17, 256, 4, 4, 64, flags=0), S_("pg_g16", 1, 37, 1024, 16, 1, 64), S_("pg_k3_k4", 2, 15, 512, 8, 2, 64, k_seq=3, k_ch=4),
          S_("pg_k1_k1", 2, 9, 512, 8, 2, 64, k_seq=1, k_ch=1), S_("pg_no_norm", 2, 9, 512, 8, 2, 64, flags=63 & ~16),
          S_("pg_no_conv2", 2, 9, 512, 8, 2, 64, flags=63 & ~2), S_("pg_dh256_g2", 2, 25, 1024, 4, 2, 256), S_("pg_dh256_g9", 1, 18, 9 * 256, 9, 1, 256)]


@pytest.mark.parametrize("sh", SHAPES, ids=lambda s: s.name)
@pytest.mark.parametrize("size", [1, 7, 16])
def test_steps_from_nothing_match_the_oracle(sh, size):
    t = synth.make_inputs(sh, want_dout=False)
    cfg, dev, cca = oracle_cfg(sh), to_device(t), _cca(sh)
    wide = -(-sh.S // size)
    st = cca.new_decode_state_paged(sh.B * wide + 1, size, sh.B, wide)
    pages = st["pages"]
    ws, pws = cca.alloc_decode_workspace_paged(sh.B, sh.S), cca.alloc_pages_workspace(sh.B * wide + 1, sh.B, wide)
    ws.fill_(255)
    ost = O.decode_init(cfg, sh.B)
    for tok in range(sh.S):
        ref = O.decode_step(cfg, t, ost, t["x"][:, tok])
        cca.pages_reserve(pages, 1, pws)
        out = cca.decode_step_paged(dev, dev["x"][:, tok].contiguous(), st, sh.S, ws)
        pages["len"] += 1
        check_close(f"out[{tok}]", out, ref)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    k, v = cca.paged_read(pages, sh.S, ints([0] * sh.B))
    check_close("k", k.reshape(ost["k"].shape), ost["k"])
    check_close("v", v.reshape(ost["v"].shape), ost["v"])
    if st["qk0_hist"].numel():
        check_close("qk0_hist", st["qk0_hist"], ost["qk0_hist"])
    assert torch.equal(st["x_prev"].cpu(), t["x"][:, sh.S - 1])
    cca.close()


@pytest.mark.parametrize("dh,hk,hq,size", [(64, 2, 8, 16), (128, 2, 8, 64)])
def test_a_prompt_forked_and_continued(dh, hk, hq, size):
    """One prompt of S0 tokens and four continuations of it that differ: each follows the oracle's forward of its own sequence, while the
    prompt's pages are shared, the last one is copied, a sequence goes, and the pool is compacted between steps."""
    S0, n = 299, 6
    sh = S_(f"pg_fork{dh}", 1, S0 + n, hq * dh, hq, hk, dh)
    t = synth.make_inputs(sh, want_dout=False)
    cfg, cca = oracle_cfg(sh), _cca(sh)
    dev = to_device(t)
    gen = torch.Generator().manual_seed(4)
    x = t["x"].repeat(4, 1, 1)
    x[1:, S0:] = torch.randn(3, n, sh.d_model, generator=gen).bfloat16()
    refs = [O.forward_rows(cfg, t, x[b:b + 1], list(range(S0, S0 + n)))[0][0] for b in range(4)]
    wide = -(-(S0 + n) // size)
    n_pages, B = 3 * wide, 5
    st = cca.new_decode_state_paged(n_pages, size, B, wide)
    pages = st["pages"]
    pws, dws = cca.alloc_pages_workspace(n_pages, B, wide), cca.alloc_decode_workspace_paged(B, S0 + n)
    # the prompt goes to sequence 2
    one = slice(2, 3)
    mine = {"pages": {**pages, "table": pages["table"][one], "len": pages["len"][one]}, "qk0_hist": st["qk0_hist"][one], "x_prev": st["x_prev"][one]}
    ws = cca.alloc_workspace(1, S0, False)
    prompt = dev["x"][:, :S0].contiguous()
    cca.forward(dev, prompt, ws)
    cca.pages_reserve(mine["pages"], S0, pws)
    cca.decode_state_from_prefill_paged(prompt, ws, mine)
    pages["len"][2] = S0
    pages["len"][3] = -1                                       # not in use
    # forked to 0, 1 and 4
    cca.pages_fork(pages, ints(2, 2, 2), ints(0, 1, 4), pws)
    for name in ("qk0_hist", "x_prev"):
        st[name][[0, 1, 4]] = st[name][[2, 2, 2]].clone()
    who = {0: 0, 1: 1, 2: 2, 4: 3}                             # sequence -> continuation
    assert int((pages["refs"] > 0).sum()) == -(-S0 // size)
    for i in range(n):
        if i == 3:                                             # 0 ends, and the pool is compacted
            cca.pages_free(pages, ints(0, -1, -1, -1, -1))
            pages["len"][0] = -1
            del who[0]
            used = cca.pages_compact(pages, pws)
            assert used.tolist() == [int((pages["refs"] > 0).sum())] and not pages["refs"][int(used):].any()
        step = torch.zeros(B, sh.d_model, dtype=torch.bfloat16)
        for b, c in who.items():
            step[b] = x[c, S0 + i]
        cca.pages_reserve(pages, 1, pws)
        out = cca.decode_step_paged(dev, step.cuda(), st, S0 + n, dws)
        torch.cuda.synchronize()
        assert cca.last_status() == 0                          # the sequences that are not in use are skipped
        for b, c in who.items():
            check_close(f"out[{b}, {i}]", out[b], refs[c][i])
            pages["len"][b] += 1
    assert pages["len"].tolist() == [-1, S0 + n, S0 + n, -1, S0 + n]
    assert int((pages["refs"] > 0).sum()) < 3 * -(-S0 // size)
    cca.close()


def test_a_sequence_without_a_page_of_its_own_is_skipped():
    sh = S_("pg_skip", 4, 3, 256, 4, 2, 64)
    t = synth.make_inputs(sh, want_dout=False)
    dev, cca = to_device(t), _cca(sh)
    st = cca.new_decode_state_paged(9, 4, 4, 2)
    pages, ws = st["pages"], cca.alloc_decode_workspace_paged(4, 8)
    pages["table"].copy_(torch.tensor([[0, -1], [1, -1], [2, 3], [-1, -1]]))
    pages["refs"].copy_(ints(1, 2, 1, 1, 0, 0, 0, 0, 0))       # page 1 is held by others too
    pages["len"].copy_(ints(2, 2, 8, 1))                       # 2: full, 3: nothing there
    before = {n: (pages[n] if n in pages else st[n]).clone() for n in ("k", "v", "qk0_hist", "x_prev")}
    cca.decode_step_paged(dev, dev["x"][:, 0].contiguous(), st, 8, ws)
    torch.cuda.synchronize()
    assert cca.last_status() == 122
    for n in ("k", "v"):
        changed = (pages[n] != before[n]).flatten(2).any(-1).any(-1)
        assert changed.tolist() == [True] + [False] * 8, n
    for n in ("qk0_hist", "x_prev"):
        assert not torch.equal(st[n][0], before[n][0]) and torch.equal(st[n][1:], before[n][1:]), n
    cca.close()


def test_captured_steps():
    """Reservation and step in one graph, replayed while the sequences grow: the same as calls one by one."""
    sh = S_("pg_graph", 2, 12, 512, 8, 2, 64)
    t = synth.make_inputs(sh, want_dout=False)
    dev, cca = to_device(t), _cca(sh)
    outs = []
    for captured in (False, True):
        st = cca.new_decode_state_paged(8, 4, 2, 4)
        pages, ws, pws = st["pages"], cca.alloc_decode_workspace_paged(2, 16), cca.alloc_pages_workspace(8, 2, 4)
        x, out = torch.empty(2, 512, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 512, dtype=torch.bfloat16, device="cuda")

        def step():
            cca.pages_reserve(pages, 1, pws)
            cca.decode_step_paged(dev, x, st, 16, ws, out=out)
            pages["len"].add_(1)
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
        got = []
        for tok in range(sh.S):
            x.copy_(dev["x"][:, tok])
            g.replay() if captured else step()
            got.append(out.clone())
        torch.cuda.synchronize()
        assert cca.last_status() == 0 and pages["len"].tolist() == [12, 12]
        outs.append(torch.stack(got))
    assert torch.equal(*outs)
    cca.close()


def test_refusals():
    from paper_2510_04476_b200.binding import CcaError
    sh = S_("pg_refuse", 2, 3, 256, 4, 2, 64)
    t = synth.make_inputs(sh, want_dout=False)
    dev, cca = to_device(t), _cca(sh)
    st = cca.new_decode_state_paged(9, 4, 2, 2)
    ws = cca.alloc_decode_workspace_paged(2, 8)
    x = dev["x"][:, 0].contiguous()
    pre = cca.alloc_workspace(2, 3, False)
    for match, call in [
        ("invalid", lambda: cca.decode_step_paged(dev, x, st, 9, ws)),
        ("invalid", lambda: cca.decode_step_paged(dev, x, st, 0, ws)),
        ("workspace too small", lambda: cca.decode_step_paged(dev, x, st, 8, ws[:1000])),
        ("x: wants", lambda: cca.decode_step_paged(dev, x[:1], st, 8, ws)),
        ("x_prev", lambda: cca.decode_step_paged(dev, x, {n: v for n, v in st.items() if n != "x_prev"}, 8, ws)),
        ("w_o", lambda: cca.decode_step_paged({**dev, "w_o": None}, x, st, 8, ws)),
        ("invalid", lambda: cca.decode_step_paged({**dev, "temp": None}, x, st, 8, ws)),
        ("out: wants", lambda: cca.decode_step_paged(dev, x, st, 8, ws, out=x[:1])),
        ("workspace too small", lambda: cca.decode_state_from_prefill_paged(dev["x"], pre[:1000], st)),
        ("invalid", lambda: cca.decode_state_from_prefill_paged(torch.zeros(2, 9, 256, dtype=torch.bfloat16, device="cuda"), pre, st)),
    ]:
        with pytest.raises(CcaError, match=match):
            call()
    assert cca.last_status() == 0
    cca.close()
