"""The 8-bit quantise pass where there are many rows: a wave's team walks several of them, with the next row's values, its expert, token and ratio at hand."""
import numpy as np
import pytest
import torch

import paper_2605_27003_amd as svdq
from tests.test_gpu_int8 import BF16, F32, I8, I32, Guarded, check_quantised, experts_of, loads_of, offsets_of, quantise64

pytestmark = pytest.mark.gpu

# Rows past every number of blocks that rows are dealt to one at a time, and no multiple of what a team then walks, for each count of waves a row and of chunks
# a lane: K up to 512, 1024, 1536, 2048 (a wave a row), 4096, 5120 (two), 8192, 10240, 14336 (four), 16384, 32768 (sixteen).
MANY = [(17001, 496), (17001, 1024), (16999, 1040), (16999, 1536), (17003, 1552), (16999, 2048), (9001, 2064), (9001, 4096), (8999, 4112), (9001, 5120), (5003, 5136), (4999, 8192),
        (5003, 8208), (4999, 10240), (5003, 10256), (4999, 13824), (4099, 14352), (4099, 16384), (2999, 16400), (2999, 32768)]


def activations(seed, M, K):
    """Rows of different sizes, a NaN and an infinity among them, in memory with a longer row stride."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((M, K + 8), generator=g, device="cuda") * torch.exp(torch.randn((M, 1), generator=g, device="cuda"))
    x[M // 2, K - 1], x[M // 3, 0], x[M - 1] = float("nan"), float("inf"), 0.0
    return x.to(BF16)[:, :K]


@pytest.mark.parametrize("M,K", MANY)
@pytest.mark.parametrize("gelu", [False, True])
def test_many_rows(M, K, gelu):
    x = activations(K, M, K)
    il = 0.5 + torch.rand(K, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    v = svdq.debug_gelu(x.contiguous()) if gelu else x
    for smooth in (il, None):
        qg, sg = Guarded(M, K, I8), Guarded(M, 1, F32)
        svdq.quantize_act_int8(x, smooth, 0.9, gelu=gelu, out=(qg.t, sg.t[:, 0]))
        check_quantised(qg.t, sg.t[:, 0], *quantise64(v, smooth, 0.9))
        assert qg.intact() and sg.intact()


@pytest.mark.parametrize("M,K", MANY)
@pytest.mark.parametrize("E", [3, 700])
@pytest.mark.parametrize("gelu", [False, True])
def test_many_grouped_rows(M, K, E, gelu):
    """Few experts, and so many that a team's rows are several experts', with empty ones between: each row with its expert's smoothing vector, its own token
    (some of them none) and its own ratio; rows that no expert owns in front and behind."""
    tokens = M // 3
    x = activations(K, tokens, K)
    g = torch.Generator("cuda").manual_seed(M)
    il, rho = 0.5 + torch.rand((E, K), generator=g, device="cuda"), 0.3 + 0.7 * torch.rand(M, generator=g, device="cuda")
    rows = torch.from_numpy(np.random.default_rng(3).integers(-1, tokens + 1, M)).to(I32).cuda()
    offsets = offsets_of(loads_of(M, M - 12, E), 5)
    e = experts_of(offsets, M)
    owned = e >= 0
    assert int(owned.sum()) == M - 12
    v = torch.cat([svdq.debug_gelu(x.contiguous()) if gelu else x, torch.zeros((1, K), dtype=BF16, device="cuda")])
    v = v[torch.where((rows < 0) | (rows >= tokens), torch.full_like(rows, tokens), rows).long()]
    qg, sg = Guarded(M, K, I8), Guarded(M, 1, F32)
    svdq.quantize_act_int8_grouped(x, offsets, il, rho, rows=rows, gelu=gelu, out=(qg.t, sg.t[:, 0]))
    q, s = quantise64(v, il[e.clamp_min(0)], rho)
    check_quantised(qg.t[owned], sg.t[owned, 0], q[owned], s[owned])
    assert qg.intact(owned) and sg.intact(owned)
    if not gelu:                                                      # of x's own rows, with one ratio and no smoothing
        x = activations(K + 1, M, K)
        qg, sg = Guarded(M, K, I8), Guarded(M, 1, F32)
        svdq.quantize_act_int8_grouped(x, offsets, None, 0.7, out=(qg.t, sg.t[:, 0]))
        q, s = quantise64(x, None, 0.7)
        check_quantised(qg.t[owned], sg.t[owned, 0], q[owned], s[owned])
        assert qg.intact(owned) and sg.intact(owned)


def test_runs_of_as_many_rows_as_there_are():
    """Sixteen rows a team, the most, and more blocks than rows are otherwise dealt to; dense and grouped."""
    M, K, E = 140_003, 272, 900
    x = activations(5, M, K)
    check_quantised(*svdq.quantize_act_int8(x, None, 0.8), *quantise64(x, None, 0.8))
    il, rho = 0.5 + torch.rand((E, K), device="cuda"), 0.3 + 0.7 * torch.rand(M, device="cuda")
    rows = torch.randperm(M, device="cuda").to(I32)
    offsets = offsets_of(loads_of(1, M, E))
    check_quantised(*svdq.quantize_act_int8_grouped(x, offsets, il, rho, rows=rows), *quantise64(x[rows.long()], il[experts_of(offsets, M)], rho))


@pytest.mark.parametrize("M,N,K,E,gelu", [(5003, 1300, 5120, 0, False), (26300, 640, 5120, 0, True), (17001, 515, 1552, 0, True), (9001, 1300, 5120, 2, False), (9001, 648, 4112, 3, True),
                                          (5003, 768, 2048, 128, False), (4999, 515, 13824, 2, True)])
def test_layers_of_many_rows_are_their_two_halves(M, N, K, E, gelu):
    """Bit for bit, with rows given in another order where the layer is grouped; and x as its own output where its rows are as long."""
    g = torch.Generator("cuda").manual_seed(M + K)
    lead = (E,) if E else ()
    qw = torch.randint(-127, 128, (*lead, N, K), generator=g, device="cuda", dtype=I8)
    sw, bias = 0.001 * torch.rand((*lead, N), generator=g, device="cuda"), torch.randn((*lead, N), generator=g, device="cuda")
    il, x = 0.5 + torch.rand((*lead, K), generator=g, device="cuda"), activations(K, M, K)
    if E:
        rho, rows, offsets = 0.3 + 0.7 * torch.rand(M, generator=g, device="cuda"), torch.randperm(M, generator=g, device="cuda").to(I32), offsets_of(loads_of(M, M, E))
        layer = svdq.W8A8Experts(il, qw, sw, bias)
        qx, sx = svdq.quantize_act_int8_grouped(x, offsets, il, rho, rows=rows, gelu=gelu)
        want, call = svdq.linear_w8a8_grouped(qx, sx, offsets, qw, sw, bias), lambda **kw: layer.forward(x, offsets, rho, rows=rows, gelu=gelu, **kw)
    else:
        layer = svdq.W8A8Linear(il, qw, sw, bias)
        qx, sx = svdq.quantize_act_int8(x, il, 0.9, gelu=gelu)
        want, call = svdq.linear_w8a8(qx, sx, qw, sw, bias), lambda **kw: layer.forward(x, 0.9, gelu=gelu, **kw)
    y = Guarded(M, N, BF16, ld=N + 8)
    assert torch.equal(call().view(torch.int16), want.view(torch.int16))
    call(out=y.t)
    assert torch.equal(y.t.contiguous().view(torch.int16), want.view(torch.int16)) and y.intact()
    assert torch.equal(call(out=x[:, :N]).contiguous().view(torch.int16), want.view(torch.int16))
