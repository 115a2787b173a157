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
