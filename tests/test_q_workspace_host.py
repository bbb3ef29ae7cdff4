"""Workspace sizes on the CPU: one for caches of at most max_len rows serves every shorter call, and every smaller batch."""
import ctypes as C
import itertools

import pytest

from paper_2510_04476_b200 import binding

SHAPES = [(8, 2, 128), (8, 2, 64), (4, 1, 256), (4, 4, 32), (64, 1, 64), (24, 2, 128)]


def _handle(lib, hq, hk, dh):
    cfg = binding.cca_config(hq * dh, hq, hk, dh, 1, 2, 2, 1, 63, 10000.0)
    h = C.c_void_p()
    assert lib.cca_init(C.byref(cfg), -1, C.byref(h)) == 0
    return h


def _sizes(fn, h, B, lengths):
    n, out = C.c_size_t(), []
    ref = C.byref(n)
    for max_len in lengths:
        assert fn(h, B, max_len, ref) == 0
        out.append(n.value)
    return out


@pytest.mark.parametrize("hq,hk,dh", SHAPES)
@pytest.mark.parametrize("name", ["cca_qcache_workspace_size", "cca_decode_workspace_size_q"])
def test_size_never_falls_with_the_length(name, hq, hk, dh):
    lib = binding.load_library()
    h = _handle(lib, hq, hk, dh)
    for B in (1, 2, 3, 4, 32, 150):
        sizes = _sizes(getattr(lib, name), h, B, range(1, 20000 if B < 5 else 6000))
        fell = [i + 1 for i, (a, b) in enumerate(itertools.pairwise(sizes)) if b < a]
        assert not fell, (B, fell[:4])
    lib.cca_destroy(h)


@pytest.mark.parametrize("hq,hk,dh", SHAPES)
@pytest.mark.parametrize("name", ["cca_qcache_workspace_size", "cca_decode_workspace_size_q"])
def test_size_never_falls_with_the_batch(name, hq, hk, dh):
    lib = binding.load_library()
    h = _handle(lib, hq, hk, dh)
    for max_len in (1, 64, 1000, 8192, 16385, 1 << 20):
        sizes = [_sizes(getattr(lib, name), h, B, [max_len])[0] for B in range(1, 200)]
        assert sizes == sorted(sizes), max_len
    lib.cca_destroy(h)


@pytest.mark.parametrize("hq,hk,dh", SHAPES)
def test_size_of_the_bf16_step_never_falls(hq, hk, dh):
    lib = binding.load_library()
    h = _handle(lib, hq, hk, dh)
    for B in (1, 2, 3, 4, 32, 150):
        sizes = _sizes(lib.cca_decode_workspace_size, h, B, range(1, 20000 if B < 5 else 6000))
        assert sizes == sorted(sizes), B
    for max_len in (1, 64, 1000, 8192, 16385, 1 << 20):
        sizes = [_sizes(lib.cca_decode_workspace_size, h, B, [max_len])[0] for B in range(1, 200)]
        assert sizes == sorted(sizes), max_len
    lib.cca_destroy(h)
