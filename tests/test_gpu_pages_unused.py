"""Sequences that are not in use (a negative length) in the calls that go by the length: rows read back, and what a prefill hands over."""
import pytest
import torch

from oracle import pages_oracle as P
from tests.test_gpu_decode_paged import S_, _cca
from tests.test_gpu_pages import bits, filled, ints, make
from tests.util import to_device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 2, 40])
def test_read_by_length_gives_zeros(n):
    cca = make(2, 64)
    pages = filled(cca, 30, 8, 5, 6)
    ws = cca.alloc_pages_workspace(30, 5, 6)
    cca.pages_reserve(pages, 48, ws)
    pages["len"].copy_(ints(0, -1, 5, -30, 47))
    pool = P.Pool.of(pages)
    for _ in range(3):                                         # whatever the new tensors held
        torch.full((1 << 22,), 7.0, device="cuda")
        got = cca.paged_read(pages, n)
        for g, w in zip(got, pool.read(n)):
            assert torch.equal(bits(g), bits(w))
        assert not got[0][1].any() and not got[1][1].any() and not got[0][3].any() and not got[1][3].any()
    first = [0, -1, 5, -30, 47]                                # by a start of its own the same sequences are read as they are
    for g, w in zip(cca.paged_read(pages, n, ints(first)), pool.read(n, first)):
        assert torch.equal(bits(g), bits(w))
    assert cca.last_status() == 0
    cca.close()

@pytest.mark.parametrize("k_seq,k_ch,S", [(2, 2, 33), (4, 4, 5), (4, 4, 20), (3, 4, 1), (1, 1, 9)])
def test_prefill_leaves_them_as_they_are(k_seq, k_ch, S):
    """The others get what the slab's hand-over gives; nothing of a sequence that is not in use is written."""
    sh = S_("pg_unused", 4, S, 256, 4, 2, 64, k_seq=k_seq, k_ch=k_ch)
    from paper_2510_04476_b200 import synth
    dev, cca = to_device(synth.make_inputs(sh, want_dout=False)), _cca(sh)
    ws = cca.alloc_workspace(4, S, False)
    cca.forward(dev, dev["x"], ws)
    slab = cca.new_decode_state(4, S)
    cca.decode_state_from_prefill(dev["x"], ws, slab)
    st = cca.new_decode_state_paged(60, 4, 4, 12)
    pages = st["pages"]
    cca.pages_reserve(pages, S, cca.alloc_pages_workspace(60, 4, 12))
    pages["len"].copy_(ints(0, -1, 0, -9))
    for name in ("qk0_hist", "x_prev"):
        st[name].fill_(3.0)
    for name in ("k", "v"):
        pages[name].fill_(5.0)
    cca.decode_state_from_prefill_paged(dev["x"], ws, st)
    torch.cuda.synchronize()
    assert cca.last_status() == 0
    for name in ("qk0_hist", "x_prev"):
        assert torch.equal(st[name][::2], slab[name][::2]), name
        assert bool((st[name][1::2] == 3.0).all()), name
    k, v = cca.paged_read(pages, S, ints(0, 0, 0, 0))
    for got, name in ((k, "k_cache"), (v, "v_cache")):
        assert torch.equal(got.flatten(2)[::2], slab[name][::2]), name
        assert bool((got[1::2] == 5.0).all()), name
    cca.close()


def test_prefill_of_one_slot_among_others_and_in_a_graph():
    """A slice of the state, captured: the slot's own rows and history alone change, at every replay."""
    sh = S_("pg_unused_one", 1, 17, 512, 8, 2, 64, k_seq=3, k_ch=2)
    from paper_2510_04476_b200 import synth
    dev, cca = to_device(synth.make_inputs(sh, want_dout=False)), _cca(sh)
    ws = cca.alloc_workspace(1, 17, False)
    cca.forward(dev, dev["x"], ws)
    st = cca.new_decode_state_paged(20, 4, 3, 6)
    one = {"pages": {**st["pages"], "table": st["pages"]["table"][1:2], "len": st["pages"]["len"][1:2]},
           "qk0_hist": st["qk0_hist"][1:2], "x_prev": st["x_prev"][1:2]}
    cca.pages_reserve(one["pages"], 17, cca.alloc_pages_workspace(20, 1, 6))
    cca.decode_state_from_prefill_paged(dev["x"], ws, one)
    want = {n: st[n].clone() for n in ("qk0_hist", "x_prev")}
    assert bool(want["x_prev"][1].any()) and not want["x_prev"][::2].any() and not want["qk0_hist"][::2].any()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cca.decode_state_from_prefill_paged(dev["x"], ws, one)
    for length in (0, -1, 0):
        st["pages"]["len"][1] = length
        for n in want:
            st[n].fill_(2.0)
        g.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(st[n][1], want[n][1] if length == 0 else torch.full_like(want[n][1], 2.0))
            assert bool((st[n][::2] == 2.0).all())
    assert cca.last_status() == 0
    cca.close()
