"""Every kernel of the 8-bit product on the GPU, at products that are listed by the kernel that they take (the host tests ask for it)."""
import pytest
import torch

import paper_2605_27003_amd as svdq
from tests.int8_products import PRODUCTS
from tests.test_gpu_int8 import BF16, F32, I8, Guarded, check_grouped, check_product, experts_of, loads_of, offsets_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,E", [call for calls in PRODUCTS.values() for call in calls])
def test_product_of_each_kernel(M, N, K, E):
    """Against 64 bits, in memory that no call may change beside its outputs; grouped: ragged and empty experts, rows in front and behind that no expert owns."""
    g = torch.Generator("cuda").manual_seed(M + N + K + E)
    lead = (E,) if E else ()
    codes = lambda *shape: torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=I8)
    q, qw = codes(M, K), codes(*lead, N, K)
    s, sw = 0.01 + torch.rand(M, generator=g, device="cuda"), 0.01 + torch.rand((*lead, N), generator=g, device="cuda")
    bias = 100.0 * torch.randn((*lead, N), generator=g, device="cuda")
    owned = slice(None)
    if E:
        first, behind = min(3, M // 4), min(5, M // 4)
        offsets = offsets_of(loads_of(M + E, M - first - behind, E, empty=0.2), first)
        owned = experts_of(offsets, M) >= 0
        assert int(owned.sum()) == M - first - behind
    for dtype in (BF16, F32):
        y = Guarded(M, N, dtype, ld=N + 8 if N % 8 == 0 else N)
        if E:
            svdq.linear_w8a8_grouped(q, s, offsets, qw, sw, bias, out=y.t)
            check_grouped(y.t, q, s, offsets, qw, sw, bias)
        else:
            svdq.linear_w8a8(q, s, qw, sw, bias, out=y.t)
            check_product(y.t, q, s, qw, sw, bias)
        assert y.intact(owned)


@pytest.mark.parametrize("N,K", [(515, 1040), (2048, 5120), (5120, 2048)])
def test_a_row_is_the_same_bits_in_every_kernel(N, K):
    """Alone, among a few and among thousands, dense and grouped: the sums are exact and what follows rounds alike, so a batch's size changes no row."""
    M = 6000
    g = torch.Generator("cuda").manual_seed(K)
    q, qw = (torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=I8) for shape in ((M, K), (N, K)))
    s, sw, bias = 0.01 + torch.rand(M, generator=g, device="cuda"), 0.01 + torch.rand(N, generator=g, device="cuda"), 100.0 * torch.randn(N, generator=g, device="cuda")
    for dtype, bits in ((BF16, torch.int16), (F32, torch.int32)):
        want = svdq.linear_w8a8(q, s, qw, sw, bias, out_dtype=dtype).view(bits)
        for m in (1, 9, 24, 40, 70, 130, 300, 600, 1100, 2305, 4000):
            assert torch.equal(svdq.linear_w8a8(q[-m:], s[-m:], qw, sw, bias, out_dtype=dtype).view(bits), want[-m:]), m
        for m in (5, 200, 3000):
            got = svdq.linear_w8a8_grouped(q[:m], s[:m], offsets_of([m // 3, m - m // 3]), qw.expand(2, N, K).contiguous(), sw.expand(2, N).contiguous(), bias.expand(2, N).contiguous(), out_dtype=dtype)
            assert torch.equal(got.view(bits), want[:m]), m
