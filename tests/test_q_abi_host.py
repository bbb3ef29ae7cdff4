"""CPU checks of the 4-bit entry points: sizes and refusals that need no device."""
import ctypes as C

import pytest
import torch

from paper_2510_04476_b200 import binding
from tests.test_abi_host import host_handle


@pytest.fixture()
def host():
    lib = binding.load_library()
    rc, h = host_handle(lib)
    assert rc == 0
    yield lib, h
    lib.cca_destroy(h)


@pytest.mark.parametrize("N,K,code", [(1, 32, 0), (16, 128, 0), (17, 160, 0), (0, 32, 1), (16, 0, 1), (16, 31, 2), (16, 48, 2),
                                       ((1 << 24) + 1, 32, 2), (16, (1 << 20) + 32, 2)])
def test_qlinear_sizes(N, K, code):
    lib = binding.load_library()
    c, s = C.c_size_t(), C.c_size_t()
    assert lib.cca_qlinear_sizes(N, K, C.byref(c), C.byref(s)) == code
    if code == 0:
        tiles = -(-N // 16) * -(-K // 128)
        assert (c.value, s.value) == (tiles * 1024, tiles * 128)
    assert lib.cca_qlinear_sizes(16, 32, None, C.byref(s)) == 1


def test_workspace_sizes(host):
    lib, h = host
    n = C.c_size_t()
    for fn in (lib.cca_qcache_workspace_size, lib.cca_decode_workspace_size_q):
        assert fn(h, 0, 128, C.byref(n)) == 1
        assert fn(h, 1, 0, C.byref(n)) == 1
        assert fn(h, 1, 128, None) == 1
        assert fn(None, 1, 128, C.byref(n)) == 1
        assert fn(h, 65536, 1, C.byref(n)) == 2
        assert fn(h, 1, (1 << 24) + 1, C.byref(n)) == 2
        assert fn(h, 1024, 1 << 21, C.byref(n)) == 2
        last = 0
        for max_len in (1, 63, 64, 65, 1000, 1 << 20):
            assert fn(h, 3, max_len, C.byref(n)) == 0
            assert n.value >= last
            last = n.value


def test_host_only_handle_refuses_compute(host):
    lib, h = host
    cache, w, qw, s = binding.cca_qcache(), binding.cca_qlinear_weights(), binding.cca_q_weights(), binding.cca_q_decode_state()
    one = C.c_void_p(256)                       # a pointer that is never followed: the handle has no device
    for n in ("k_codes", "v_codes", "k_scales", "v_scales", "len"):
        setattr(cache, n, 256)
    cache.S_max = 16
    assert lib.cca_qcache_append(h, one, one, None, None, C.byref(cache), 1, 1, None) == 1
    assert lib.cca_qcache_read(h, C.byref(cache), None, one, one, 1, 1, None) == 1
    assert lib.cca_qcache_attention(h, one, one, C.byref(cache), 16, 0, one, 1 << 30, 1, None) == 1
    assert lib.cca_qcache_evict(h, C.byref(cache), 1, 0, one, 16, one, 1 << 30, 1, None) == 1
    assert lib.cca_qlinear_pack(h, one, C.byref(w), None) == 1
    assert lib.cca_qlinear(h, C.byref(w), one, one, 0, 1, None) == 1
    assert lib.cca_decode_step_q(h, C.byref(qw), one, one, C.byref(s), 16, one, 1 << 30, 1, None) == 1
    assert lib.cca_decode_state_from_prefill_q(h, one, one, 1 << 30, 1, 1, C.byref(s), None) == 1


def test_extension_refuses_what_does_not_fit():
    """The marshalling extension on CPU tensors: every argument is refused by name, nothing reaches the library."""
    binding.load_library()
    from paper_2510_04476_b200 import _bind as b
    h = b.new_handle(0, 256, 4, 2, 64, 2, 2, 0)
    w = {"codes": torch.zeros(2, 1, 16, 64, dtype=torch.uint8), "scales": torch.zeros(2, 1, 16, 4, dtype=torch.bfloat16), "N": 24, "K": 64}
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    cache = {"len": torch.zeros(1, dtype=torch.int32), "k_codes": torch.zeros(1, 2, 8, 32, dtype=torch.uint8)}
    for match, call in (("N", lambda: b.qlinear(h, {}, x, None, torch.bfloat16)),
                        ("codes: wants a contiguous Byte tensor .* on cuda:0, got .* on cpu", lambda: b.qlinear(h, w, x, None, torch.bfloat16)),
                        ("dict", lambda: b.qlinear(h, 5, x, None, torch.bfloat16)),
                        ("k_codes", lambda: b.qcache_attention(h, x, cache, 8, x, None, None)),
                        ("len: wants a tensor", lambda: b.qcache_evict(h, {}, 1, 0, x, 8, x)),
                        ("cache", lambda: b.decode_step_q(h, {}, x, {}, 8, x, None)),
                        ("w: wants two", lambda: b.qlinear_pack(h, x[0]))):
        with pytest.raises(binding.CcaError, match=match):
            call()
    with pytest.raises(TypeError):
        b.qlinear(h)
    with pytest.raises(ValueError):
        b.qlinear(3, w, x, None, torch.bfloat16)           # no handle
