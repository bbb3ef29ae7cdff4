"""CPU checks of the entry points on pages: sizes and refusals that need no device."""
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


@pytest.mark.parametrize("n_pages,max_pages,B,code", [(1, 1, 1, 0), (1000, 64, 33, 0), (0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (-1, 1, 1, 1),
                                                       (1, 1, 65536, 2), (1, (1 << 24) + 1, 1, 2), (1, 1 << 24, 65, 2), (1 << 31, 1, 1, 2),
                                                       (1 << 62, 1, 1, 2), (1, 1 << 62, 1, 2)])
def test_pages_workspace_sizes(host, n_pages, max_pages, B, code):
    lib, h = host
    n = C.c_size_t()
    assert lib.cca_pages_workspace_size(h, n_pages, max_pages, B, C.byref(n)) == code
    assert lib.cca_pages_workspace_size(h, n_pages, max_pages, B, None) == 1
    assert lib.cca_pages_workspace_size(None, n_pages, max_pages, B, C.byref(n)) == 1
    if code == 0:
        assert n.value >= 4 * max(5 * n_pages + B, B * max_pages + B)


def test_attention_and_step_workspace_sizes(host):
    lib, h = host
    n = C.c_size_t()
    for fn in (lib.cca_paged_workspace_size, lib.cca_decode_workspace_size_paged):
        assert fn(h, 0, 128, C.byref(n)) == 1
        assert fn(h, 1, 0, C.byref(n)) == 1
        assert fn(h, 1, 128, None) == 1
        assert fn(None, 1, 128, C.byref(n)) == 1
        assert fn(h, 65536, 1, C.byref(n)) == 2
        assert fn(h, 1, (1 << 24) + 1, C.byref(n)) == 2
        for B in (1, 3, 200):                              # never falls with the length or the batch
            last = 0
            for max_len in (1, 63, 64, 65, 1000, 16384, 1 << 20):
                assert fn(h, B, max_len, C.byref(n)) == 0
                assert n.value >= last
                last = n.value
        sizes = []
        for B in range(1, 300):
            assert fn(h, B, 4096, C.byref(n)) == 0
            sizes.append(n.value)
        assert sizes == sorted(sizes)


def test_host_only_handle_refuses_compute(host):
    lib, h = host
    pages, w, s = binding.cca_pages(), binding.cca_weights(), binding.cca_paged_decode_state()
    one = C.c_void_p(256)                                  # a pointer that is never followed: the handle has no device
    for n in ("k", "v", "refs", "table", "len"):
        setattr(pages, n, 256)
    pages.n_pages = pages.page_size = pages.max_pages = 16
    s.pages = pages
    p = C.byref(pages)
    assert lib.cca_pages_reserve(h, p, 1, None, None, one, 1 << 30, 1, None) == 1
    assert lib.cca_pages_fork(h, p, one, one, 1, one, 1 << 30, 1, None) == 1
    assert lib.cca_pages_free(h, p, one, 1, None) == 1
    assert lib.cca_pages_compact(h, p, one, one, 1 << 30, 1, None) == 1
    assert lib.cca_paged_append(h, one, one, None, p, 1, 1, None) == 1
    assert lib.cca_paged_read(h, p, None, one, one, 1, 1, None) == 1
    assert lib.cca_paged_attention(h, one, one, None, p, 16, one, 1 << 30, 1, None) == 1
    assert lib.cca_decode_step_paged(h, C.byref(w), one, one, C.byref(s), 16, one, 1 << 30, 1, None) == 1
    assert lib.cca_decode_state_from_prefill_paged(h, one, one, 1 << 30, 1, 1, C.byref(s), None) == 1


def test_extension_refuses_what_does_not_fit():
    """The marshalling extension on CPU tensors: every argument is refused by name, nothing reaches the library."""
    binding.load_library()
    from paper_2510_04476_b200 import _bind as b
    h = b.new_handle(0, 256, 4, 2, 64, 2, 2, 0)
    pages = {"k": torch.zeros(4, 2, 8, 64, dtype=torch.bfloat16), "table": torch.zeros(1, 4, dtype=torch.int32)}
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    for match, call in (("k: wants a tensor", lambda: b.pages_free(h, {}, x)),
                        ("table: wants a tensor", lambda: b.pages_free(h, {"k": x}, x)),
                        ("four dimensions", lambda: b.pages_free(h, {**pages, "k": x}, x)),
                        ("two", lambda: b.pages_free(h, {**pages, "table": x[0]}, x)),
                        ("k: wants a contiguous BFloat16 tensor of shape .4, 2, 8, 64. on cuda:0, got .* on cpu", lambda: b.pages_reserve(h, pages, 1, x, None, None)),
                        ("dict", lambda: b.paged_append(h, 5, x, x, None)),
                        ("pages", lambda: b.decode_step_paged(h, {}, x, {}, 8, x, None)),
                        ("pages", lambda: b.decode_state_from_prefill_paged(h, x, x, {}))):
        with pytest.raises(binding.CcaError, match=match):
            call()
    for call in (b.pages_reserve, b.pages_fork, b.pages_free, b.pages_compact, b.paged_append, b.paged_read, b.paged_attention,
                 b.decode_step_paged, b.decode_state_from_prefill_paged):
        with pytest.raises(TypeError):
            call(h)
