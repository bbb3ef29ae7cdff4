"""Products with 4-bit weights of small and large size, at every token count around the change of kernel.

The bound is the products' own, 2^-23 (K / 256 + 48) sum |x w| for fp32 outputs, with nothing absolute beside it: within the stated range no
intermediate number leaves fp32's normal range."""
import pytest
import torch

from oracle import q_oracle as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cca():
    from paper_2510_04476_b200.binding import CCA
    h = CCA(d_model=256, n_q_heads=4, n_kv_heads=4, head_dim=64)
    yield h
    h.close()


@pytest.mark.parametrize("M", [1, 8, 9, 40])
@pytest.mark.parametrize("w_exp,x_exp", [(w, x) for w in (-86, -80, -73, -60, -40, 0, 20) for x in (-28, 0, 20, 50) if w + x >= -88])
def test_product_of_weights_of_any_size(cca, M, w_exp, x_exp):
    N, K = 70, 1056
    gen = torch.Generator().manual_seed(M - w_exp)
    w = (2.0 ** w_exp * torch.randn(N, K, generator=gen).clamp(-8, 8)).bfloat16()
    x = (2.0 ** x_exp * torch.randn(M, K, generator=gen)).bfloat16()
    y = cca.qlinear(cca.qlinear_pack(w.cuda()), x.cuda(), out_dtype=torch.float32).cpu().double()
    w64 = Q.values(*Q.quantise(w))
    ref, mag = x.double() @ w64.t(), x.double().abs() @ w64.abs().t()
    assert float(mag.min()) > 2.0 ** -96
    err = (y - ref).abs() / mag
    assert float(err.max()) <= 2.0 ** -23 * (K / 256 + 48), float(err.max() * 2 ** 23)
    assert cca.last_status() == 0


@pytest.mark.parametrize("N,K", [(1000, 1024), (2368, 4096), (2369, 4096), (2368, 4128), (4736, 2048), (4737, 2048), (4736, 2080), (1180, 4096)])
@pytest.mark.parametrize("M", [8, 9, 32, 33, 64, 65, 97])
def test_product_on_both_sides_of_the_change_of_kernel(cca, M, N, K):
    """16 x 148 and 32 x 148 rows, 4096 columns in all: where one kernel takes over from the other."""
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    w = (0.05 * torch.randn(N, K, generator=gen, device="cuda")).bfloat16()
    x = torch.randn(M, K, generator=gen, device="cuda").bfloat16()
    y = cca.qlinear(cca.qlinear_pack(w), x, out_dtype=torch.float32).double()
    w64 = Q.values(*Q.quantise(w)).cuda()
    ref, mag = x.double() @ w64.t(), x.double().abs() @ w64.abs().t()
    assert ((y - ref).abs() <= 2.0 ** -23 * (K / 256 + 48) * mag).all(), float(((y - ref).abs() / mag).max() * 2 ** 23)
    assert cca.last_status() == 0
