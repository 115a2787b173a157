"""The 8-bit layer on the GPU against its definition: codes and scales from binary32 operations emulated in 64 bits, products in
64 bits (exact: K 128^2 < 2^53)."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import paper_2605_27003_amd as svdq
from paper_2605_27003_amd import binding

pytestmark = pytest.mark.gpu
F32, F64, BF16, I8, I32 = torch.float32, torch.float64, torch.bfloat16, torch.int8, torch.int32


def rand(seed, *shape, scale=1.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape, dtype=np.float32) * np.float32(scale)).cuda()


def codes(seed, *shape, low=-127, high=127):
    return torch.from_numpy(np.random.default_rng(seed).integers(low, high, shape, dtype=np.int8, endpoint=True)).cuda()


def r32(t):
    return t.to(F32).to(F64)


def quantise64(x, il, rho):
    """(codes f64, scales f64) of x [M, K] by the definition, every operation rounded to binary32; il [K], [M, K] or None, rho a number or [M]."""
    v = x.to(F64)
    if il is not None:
        v = r32(v * il.to(F64))
    rho = torch.as_tensor(rho, dtype=F32, device=x.device).to(F64)
    a = v.abs().amax(dim=1)
    bad = ~(v.isfinite().all(dim=1)) | torch.isnan(rho)
    s = r32(r32(rho * a) / 127.0)
    none = ~bad & (s < 2.0 ** -126)
    s = torch.where(none | bad, torch.ones_like(s), s)
    q = torch.round(r32(v * r32(1.0 / s)[:, None])).clamp(-127, 127)
    zero = (none | bad)[:, None]
    return torch.where(zero, torch.zeros_like(q), q), torch.where(bad, torch.full_like(s, float("nan")), torch.where(none, torch.zeros_like(s), s))


def check_quantised(qx, sx, q, s):
    assert torch.equal(qx.to(F64), q)
    assert torch.equal(torch.isnan(sx), torch.isnan(s)) and torch.equal(torch.nan_to_num(sx.to(F64), nan=-1.0), torch.nan_to_num(s, nan=-1.0))


def check_product(y, q, s, qw, sw, bias):
    """|error| of (float(sum) s) sw + bias: three binary32 roundings of the product, one of the sum (2^-24 each, their products
    far below the fourth power's slack), half a step of the output's type (bf16 2^-8, of a value up to that much larger)."""
    p = (q.to(F64) @ qw.to(F64).t()) * s.to(F64)[:, None] * sw.to(F64)
    want = p + (0.0 if bias is None else bias.to(F64))
    bound = 4 * 2.0 ** -24 * p.abs() + 2 * 2.0 ** -24 * want.abs()
    if y.dtype == BF16:
        bound = bound * 1.01 + 2.0 ** -8 * want.abs()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(y), nan)
    off = torch.where(nan, torch.zeros_like(want), (y.to(F64) - want).abs() - bound)
    assert off.max().item() <= 1e-37, off.max().item()


class Guarded:
    """A [rows, cols] view in the middle of memory that no call may change, with row stride ld and the first element `lead` elements in."""

    def __init__(self, rows, cols, dtype, ld=None, lead=64):
        self.ld, self.lead, self.rows, self.cols = ld or cols, lead, rows, cols
        n = lead + rows * self.ld + 4096
        self.flat = torch.full((n,), 77, dtype=dtype, device="cuda")
        self.t = self.flat[lead:lead + rows * self.ld].view(rows, self.ld)[:, :cols]

    def intact(self, written=None):
        """Nothing changed but the rows `written` (all of them by default)."""
        seen = self.flat.clone()
        body = seen[self.lead:self.lead + self.rows * self.ld].view(self.rows, self.ld)
        body[slice(None) if written is None else written, :self.cols] = 77
        return bool((seen == 77).all())


@pytest.mark.parametrize("M,K", [(1, 16), (3, 48), (5, 512), (2, 528), (70, 1024), (9, 1040), (4, 2064), (33, 4096), (19, 5120), (6, 8176), (3, 13824), (2, 16400), (3, 32768)])
@pytest.mark.parametrize("smooth", [False, True])
def test_codes_and_scales(M, K, smooth):
    x = (rand(K + M, M, K + 24) * torch.exp(rand(K, M, 1))).to(BF16)[:, :K]
    il = 0.5 + rand(K + 1, K).abs() if smooth else None
    for rho in (1.0, 0.8, 0.013):
        qx, sx = svdq.quantize_act_int8(x, il, rho)
        check_quantised(qx, sx, *quantise64(x, il, rho))


def test_every_tie_and_every_step():
    """x / s on whole numbers and halves: the scale is 1 (the row's maximum is 127), ties go to the even code."""
    v = torch.arange(-254, 255, dtype=F32) / 2
    x = torch.zeros((2, 512))
    x[0, :509] = v
    x[1, :509] = -v
    x = x.to(BF16).cuda()
    qx, sx = svdq.quantize_act_int8(x)
    assert sx.tolist() == [1.0, 1.0] and torch.equal(qx[0, :509].cpu().float(), torch.round(v)) and torch.equal(qx[1], -qx[0])


@pytest.mark.parametrize("K", [64, 5120])
def test_rows_of_special_values(K):
    """Each alone in its row: zeros, the smallest subnormals, the largest finite values, infinities, NaN, and an overflow by smoothing."""
    x = rand(3, 12, K).to(BF16)
    x[1] = 0
    x[2] = 1e-39
    x[3] = torch.where(x[3] > 0, 1e-37, -2e-37)
    x[4, K // 2] = float("inf")
    x[5, 1] = float("-inf")
    x[6, K - 1] = float("nan")
    x[7] = torch.where(x[7] > 0, 3.3e38, -3.3e38)
    x[8, 0], x[9, 0] = 1e38, -0.0
    x[10] = -0.0
    il = torch.ones(K, device="cuda")
    il[0] = 100.0
    for smoothing in (None, il):
        qx, sx = svdq.quantize_act_int8(x, smoothing, 0.9)
        q, s = quantise64(x, smoothing, 0.9)
        check_quantised(qx, sx, q, s)
    qw, sw = codes(5, 96, K), rand(6, 96).abs()
    check_product(svdq.linear_w8a8(qx, sx, qw, sw, out_dtype=F32), q, s, qw, sw, None)


def test_gelu_in_front():
    x = (rand(8, 37, 1552) * 2).to(BF16)
    il = 0.5 + rand(9, 1552).abs()
    qx, sx = svdq.quantize_act_int8(x, il, 0.9, gelu=True)
    check_quantised(qx, sx, *quantise64(svdq.debug_gelu(x), il, 0.9))
    lin = svdq.W8A8Linear(il, codes(10, 200, 1552), rand(11, 200).abs(), rand(12, 200))
    assert torch.equal(lin.forward(x, 0.9, gelu=True), svdq.linear_w8a8(qx, sx, lin.qw, lin.sw, lin.bias))


@pytest.mark.parametrize("M,K", [(262200, 512), (140000, 1008), (70001, 2048), (33000, 4112), (20000, 8192), (9800, 13824), (5000, 32768)])
def test_gelu_of_many_tokens(M, K):
    """Where there are many the activation comes from a table: the same codes, and on every bf16 value, NaN rows and all."""
    x = torch.randn((M, K), generator=torch.Generator("cuda").manual_seed(K), device="cuda", dtype=BF16) * 2
    every = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(BF16).cuda()
    every = every[every.isfinite()][:65024 // K * K if K < 65024 else K].view(-1, K)
    x[-len(every):] = every
    x[5, 3] = float("nan")
    qx, sx = svdq.quantize_act_int8(x, None, 0.9, gelu=True)
    for rows in (slice(0, 40), slice(M // 2, M // 2 + 40), slice(M - len(every) - 3, M)):
        check_quantised(qx[rows], sx[rows], *quantise64(svdq.debug_gelu(x[rows]), None, 0.9))
        few = svdq.quantize_act_int8(x[rows].contiguous(), None, 0.9, gelu=True)          # without the table
        assert torch.equal(few[0], qx[rows]) and torch.equal(few[1].view(I32), sx[rows].view(I32))


SHAPES = [(1, 1, 16), (1, 129, 128), (3, 5, 144), (2, 5120, 5120), (7, 1000, 13824), (16, 512, 4096), (17, 640, 1040), (33, 100, 16), (64, 64, 64), (65, 72, 80), (100, 4999, 272),
          (128, 128, 128), (129, 257, 272), (200, 300, 4112), (300, 2048, 2048), (513, 771, 400), (1000, 1000, 1008), (2305, 515, 512), (4097, 2560, 640), (1, 30720, 160), (40, 8, 32768),
          # several rounds of the largest tiles, K of two stages and more, whole and not
          (17000, 2048, 256), (20001, 2100, 272), (30000, 1290, 640), (9000, 5120, 384)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_product(M, N, K, dtype):
    q, s, qw, sw, bias = codes(M, M, K), 0.01 + rand(1, M).abs(), codes(N, N, K), 0.01 + rand(2, N).abs(), rand(3, N, scale=100.0)
    check_product(svdq.linear_w8a8(q, s, qw, sw, bias, out_dtype=dtype), q, s, qw, sw, bias)
    check_product(svdq.linear_w8a8(q, s, qw, sw, out_dtype=dtype), q, s, qw, sw, None)


@pytest.mark.parametrize("M,N", [(5, 70), (150, 200), (600, 300)])
def test_extreme_codes(M, N):
    """Sums as large as they get, of both signs; -128, which the quantise pass does not make, is an ordinary weight and code."""
    K, one = 32768, torch.ones(max(M, N), device="cuda")
    for a, b in ((127, 127), (-128, -128), (127, -128)):
        q, qw = torch.full((M, K), a, dtype=I8, device="cuda"), torch.full((N, K), b, dtype=I8, device="cuda")
        assert bool((svdq.linear_w8a8(q, one[:M], qw, one[:N], out_dtype=F32) == float(a * b * K)).all())


@pytest.mark.parametrize("M,N,K", [(1, 33, 64), (20, 120, 144), (131, 260, 272), (520, 1027, 256)])
@pytest.mark.parametrize("dtype,ld,lead", [(BF16, 8, 64), (BF16, 1, 64), (BF16, 8, 3), (F32, 4, 64), (F32, 3, 65)])
def test_outputs_in_the_middle_of_memory(M, N, K, dtype, ld, lead):
    """Row strides and starts that allow 16-byte stores and that do not; nothing beside the outputs changes."""
    q, s, qw, sw, bias = codes(1, M, K), rand(1, M).abs(), codes(2, N, K), rand(2, N).abs(), rand(3, N)
    y = Guarded(M, N, dtype, ld=(N + ld - 1) // ld * ld + ld, lead=lead)
    assert svdq.linear_w8a8(q, s, qw, sw, bias, out=y.t) is y.t
    check_product(y.t, q, s, qw, sw, bias)
    assert y.intact()
    qg, sg = Guarded(M, K, I8), Guarded(1, M, F32, lead=65)
    x = rand(4, M, K).to(BF16)
    svdq.quantize_act_int8(x, out=(qg.t, sg.t[0]))
    check_quantised(qg.t, sg.t[0], *quantise64(x, None, 1.0))
    assert qg.intact() and sg.intact()


def loads_of(seed, M, E, empty=0.4):
    rng = np.random.default_rng(seed)
    share = rng.random(E) ** 3 * (rng.random(E) > empty) + 1e-12
    return np.random.default_rng(seed + 1).multinomial(M, share / share.sum())


def offsets_of(loads, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(loads)]), dtype=I32).cuda()


def experts_of(offsets, M):
    """Expert of every row, -1 for those of none."""
    e = torch.searchsorted(offsets.to(torch.int64), torch.arange(M, device="cuda"), right=True) - 1
    return torch.where((e < 0) | (e >= offsets.numel() - 1), torch.full_like(e, -1), e)


def check_grouped(y, q, s, offsets, qw, sw, bias):
    o = offsets.tolist()
    for e, (a, b) in enumerate(zip(o, o[1:])):
        if b > a:
            check_product(y[a:b], q[a:b], s[a:b], qw[e], sw[e], None if bias is None else bias[e])


@pytest.mark.parametrize("M,E,N,K", [(1, 1, 16, 16), (1, 64, 200, 256), (5, 3, 33, 48), (32, 128, 320, 512), (60, 7, 130, 272), (64, 1, 128, 128), (300, 2, 257, 400), (700, 65, 100, 144),
                                     (1000, 9, 1030, 640), (2500, 3, 520, 1040), (4096, 1024, 24, 32), (9000, 5, 768, 512), (20000, 3, 2100, 400), (18000, 64, 3000, 256), (18000, 65, 3000, 128)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_grouped_product(M, E, N, K, dtype):
    """Ragged and empty experts; rows in front of the first and behind the last expert stay as they were."""
    q, s, qw, sw, bias = codes(1, M, K), 0.1 + rand(1, M).abs(), codes(2, E, N, K), 0.1 + rand(2, E, N).abs(), rand(3, E, N, scale=50.0)
    for first, behind in ((0, 0), (min(3, M - 1), min(5, M - 1 - min(3, M - 1)))):
        loads = loads_of(M + E, M - first - behind, E)
        offsets = offsets_of(loads, first)
        y = Guarded(M, N, dtype, ld=N + 8)
        svdq.linear_w8a8_grouped(q, s, offsets, qw, sw, bias, out=y.t)
        check_grouped(y.t, q, s, offsets, qw, sw, bias)
        owned = experts_of(offsets, M) >= 0
        assert y.intact(owned) and bool((y.t[~owned] == 77).all())
    check_grouped(svdq.linear_w8a8_grouped(q, s, offsets, qw, sw, out_dtype=dtype), q, s, offsets, qw, sw, None)


@pytest.mark.parametrize("M,E,K,tokens", [(1, 1, 16, 1), (7, 3, 528, 4), (64, 130, 1024, 64), (333, 5, 2064, 100), (50, 2, 5120, 7), (20, 3, 16400, 9)])
def test_grouped_codes_and_scales(M, E, K, tokens):
    """Gathered rows (some tokens many times), a smoothing vector for each expert, a ratio for each row."""
    x = rand(1, tokens, K + 8).to(BF16)[:, :K]
    il, rho = 0.5 + rand(2, E, K).abs(), 0.3 + 0.7 * torch.rand(M, generator=torch.Generator().manual_seed(M)).cuda()
    rows = torch.from_numpy(np.random.default_rng(3).integers(0, tokens, M)).to(I32).cuda()
    first = min(2, M - 1)
    offsets = offsets_of(loads_of(M, M - first, E), first)
    e = experts_of(offsets, M)
    owned = e >= 0
    for smooth, ratio in itertools.product((il, None), (rho, 0.7)):
        qg, sg = Guarded(M, K, I8), Guarded(M, 1, F32)
        svdq.quantize_act_int8_grouped(x, offsets, smooth, ratio, rows=rows, out=(qg.t, sg.t[:, 0]))
        q, s = quantise64(x[rows.long()], None if smooth is None else il[e.clamp_min(0)], ratio)
        check_quantised(qg.t[owned], sg.t[owned, 0], q[owned], s[owned])
        assert qg.intact(owned) and sg.intact(owned)
    if tokens >= M:
        qx, sx = svdq.quantize_act_int8_grouped(x[:M], offsets, il)
        q, s = quantise64(x[:M], il[e.clamp_min(0)], 1.0)
        check_quantised(qx[owned], sx[owned], q[owned], s[owned])


def test_row_ratios_and_rows_that_make_no_sense():
    """A row number outside x is a row of zeros; a ratio that is not positive gives scale 0, a NaN scale NaN."""
    x, K = rand(1, 6, 272).to(BF16), 272
    rows = torch.tensor([0, -1, 6, 5, 1 << 30, -(1 << 31), 2, 2], dtype=I32).cuda()
    rho = torch.tensor([1.0, 1.0, 0.5, -0.5, 1.0, 1.0, float("nan"), 0.0]).cuda()
    offsets = torch.tensor([0, 3, 8], dtype=I32).cuda()
    qx, sx = svdq.quantize_act_int8_grouped(x, offsets, rho=rho, rows=rows)
    token = torch.cat([x, torch.zeros((1, K), dtype=BF16, device="cuda")])[[0, 6, 6, 5, 6, 6, 2, 2]]
    check_quantised(qx, sx, *quantise64(token, None, rho))


@pytest.mark.parametrize("offsets", [[0, 40, 20, 60], [-5, 10, 1 << 30, 7], [64, 0, 0, 64], [70, 80, 90, 100], [-9, -8, -7, -6], [(1 << 31) - 1, -(1 << 31), 5, 9]])
def test_offsets_that_break_the_rules_stay_within_the_arrays(offsets):
    M, N, K = 64, 72, 144
    o = torch.tensor(offsets, dtype=I32).cuda()
    x, il, qw, sw = rand(1, M, K).to(BF16), 0.5 + rand(2, 3, K).abs(), codes(3, 3, N, K), rand(4, 3, N).abs()
    qg, sg, y = Guarded(M, K, I8), Guarded(M, 1, F32), Guarded(M, N, BF16)
    svdq.quantize_act_int8_grouped(x, o, il, out=(qg.t, sg.t[:, 0]))
    svdq.linear_w8a8_grouped(codes(5, M, K), rand(6, M), o, qw, sw, out=y.t)
    torch.cuda.synchronize()
    assert qg.intact() and sg.intact() and y.intact()


def moe(layer_up, layer_down, x, ids, weights):
    """A router's choice through two grouped layers, as a program would: order by expert, two products with a GELU between, weighted sum."""
    T, k = ids.shape
    flat = ids.reshape(-1)
    order = torch.sort(flat, stable=True).indices
    offsets = torch.zeros(layer_up.qw.shape[0] + 1, dtype=I32, device="cuda")
    offsets[1:] = torch.bincount(flat, minlength=layer_up.qw.shape[0]).cumsum(0)
    rows = (order // k).to(I32)
    y = layer_down.forward(layer_up.forward(x, offsets, 0.9, rows=rows), offsets, gelu=True)
    return torch.zeros((T, y.shape[1]), device="cuda").index_add_(0, rows.long(), y.float() * weights.reshape(-1)[order][:, None])


@pytest.mark.parametrize("T,k,E", [(1, 2, 8), (40, 2, 8), (600, 4, 16)])
def test_router_and_two_grouped_layers(T, k, E):
    D, H = 272, 528
    up = svdq.W8A8Experts(0.5 + rand(1, E, D).abs(), codes(2, E, H, D), 0.0005 + 0.0005 * rand(3, E, H).abs(), rand(4, E, H, scale=0.1))
    down = svdq.W8A8Experts(None, codes(5, E, D, H), 0.0005 + 0.0005 * rand(6, E, D).abs(), None)
    x = rand(7, T, D).to(BF16)
    g = torch.Generator().manual_seed(T)
    ids = torch.rand((T, E), generator=g).topk(k, dim=1).indices.cuda()
    weights = torch.rand((T, k), generator=g).cuda()
    got = moe(up, down, x, ids, weights)
    want, size = torch.zeros((T, D), dtype=F64, device="cuda"), torch.zeros((T, D), dtype=F64, device="cuda")
    for j in range(k):
        for t in range(T):
            e = int(ids[t, j])
            q, s = quantise64(x[t:t + 1], up.inv_lambda[e], 0.9)
            u = svdq.linear_w8a8(q.to(I8), s.to(F32), up.qw[e], up.sw[e], up.bias[e])                 # bf16, as between the layers
            check_product(u, q, s, up.qw[e], up.sw[e], up.bias[e])
            q, s = quantise64(svdq.debug_gelu(u), None, 1.0)
            y = ((q @ down.qw[e].to(F64).t()) * s[:, None] * down.sw[e].to(F64))[0]
            want[t] += y * weights[t, j].to(F64)
            size[t] += y.abs() * weights[t, j].to(F64)
    # y is rounded to bf16 (half a step: 2^-8), then k products and sums in binary32
    assert bool(((got.to(F64) - want).abs() <= size * (1.01 * 2.0 ** -8 + (k + 8) * 2.0 ** -24)).all())


@pytest.mark.parametrize("M", [1, 30, 300])
def test_layer_is_its_two_halves(M):
    """W8A8Linear against the two functions bit for bit, with strided x, a given output, and x as its own output."""
    K = N = 1040
    lin = svdq.W8A8Linear(0.5 + rand(1, K).abs(), codes(2, N, K), 0.001 * rand(3, N).abs(), rand(4, N))
    x = rand(5, M, K + 16).to(BF16)[:, :K]
    want = svdq.linear_w8a8(*svdq.quantize_act_int8(x, lin.inv_lambda, 0.8), lin.qw, lin.sw, lin.bias)
    y = Guarded(M, N, BF16, ld=N + 8)
    assert torch.equal(lin.forward(x, 0.8), want) and torch.equal(lin.forward(x, 0.8, out=y.t), want) and y.intact()
    own = x.clone(memory_format=torch.contiguous_format)        # contiguous() of one row is that row
    assert torch.equal(lin.forward(own, 0.8, out=own), want)
    assert lin.forward(x[:0], 0.8).shape == (0, N)
    none = svdq.W8A8Experts(lin.inv_lambda[None], lin.qw[None], lin.sw[None], lin.bias[None])
    assert torch.equal(none.forward(x, offsets_of([M]), 0.8), want)


@pytest.mark.parametrize("M,N,K,E", [(1, 1, 16, 0), (1, 5120, 4096, 0), (5, 77, 144, 0), (16, 512, 512, 0), (17, 100, 528, 0), (256, 512, 512, 0), (40, 1000, 1408, 0), (33, 640, 1424, 0),
                                     (100, 333, 2064, 0), (4, 4096, 4096, 0), (3, 200, 2992, 0), (1, 64, 64, 3), (20, 96, 272, 5), (50, 200, 1040, 40), (9, 300, 4096, 1000), (100, 128, 512, 2)])
@pytest.mark.parametrize("gelu", [False, True])
def test_small_layers(M, N, K, E, gelu):
    """Layers that are one launch against the two functions, bit for bit: outputs, and the codes and scales that the C function leaves."""
    lead = (E,) if E else ()
    qw, sw, bias, il = codes(1, *lead, N, K), 0.001 * rand(2, *lead, N).abs(), rand(3, *lead, N), 0.5 + rand(4, *lead, K).abs()
    tokens = max(1, M // 3) if E else M
    x = rand(5, tokens, K + 16).to(BF16)[:, :K]
    x[tokens // 2, K // 3] = float("nan") if M % 2 else 0.0
    if not E:
        want_q, want_s = svdq.quantize_act_int8(x, il, 0.8, gelu=gelu)
        want, written = svdq.linear_w8a8(want_q, want_s, qw, sw, bias), slice(None)
        offsets = rows = rho = None
    else:
        first, rho = min(2, M - 1), 0.3 + 0.7 * torch.rand(M, device="cuda")
        offsets = offsets_of(loads_of(M, M - first, E), first)
        rows = torch.from_numpy(np.random.default_rng(6).integers(-1, tokens + 1, M)).to(I32).cuda()
        want_q, want_s = svdq.quantize_act_int8_grouped(x, offsets, il, rho, rows=rows, gelu=gelu)
        want, written = svdq.linear_w8a8_grouped(want_q, want_s, offsets, qw, sw, bias), experts_of(offsets, M) >= 0
    y, qx, sx = Guarded(M, N, BF16, ld=N + 3), Guarded(M, K, I8), Guarded(M, 1, F32)
    layer = binding._LayerInt8(E, N, K, il.data_ptr(), qw.data_ptr(), sw.data_ptr(), bias.data_ptr())
    at = lambda t: None if t is None else t.data_ptr()
    rc = svdq.load_library().svdq_layer_int8_forward(ctypes.addressof(layer), x.data_ptr(), K + 16, tokens, at(rows), at(offsets), 0.8, at(rho), int(gelu), M,
                                                     qx.t.data_ptr(), sx.t.data_ptr(), y.t.data_ptr(), N + 3, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    same = lambda a, b, t: torch.equal(a[written].contiguous().view(t), b[written].contiguous().view(t))
    assert same(y.t, want, torch.int16) and same(qx.t, want_q, I8) and same(sx.t[:, 0], want_s, I32)
    assert y.intact(written) and qx.intact(written) and sx.intact(written)
    module = svdq.W8A8Experts(il, qw, sw, bias) if E else svdq.W8A8Linear(il, qw, sw, bias)
    got = module.forward(x, offsets, rho, rows=rows, gelu=gelu) if E else module.forward(x, 0.8, gelu=gelu)
    assert same(got, want, torch.int16)


def test_captured_calls_and_other_streams():
    """A dense and a grouped layer in a graph, replayed with eager calls of the same layers between; offsets change between replays."""
    K, N, M, E = 1040, 520, 96, 6
    lin = svdq.W8A8Linear(None, codes(1, N, K), 0.001 * rand(2, N).abs(), None)
    ex = svdq.W8A8Experts(0.5 + rand(3, E, K).abs(), codes(4, E, N, K), 0.001 * rand(5, E, N).abs(), rand(6, E, N))
    x, offsets = rand(7, M, K).to(BF16), offsets_of([16] * E)
    rows = torch.arange(M, dtype=I32).flip(0).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            lin.forward(x), ex.forward(x, offsets, 0.9, rows=rows)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = lin.forward(x), ex.forward(x, offsets, 0.9, rows=rows)
    for i in range(4):
        x.copy_(rand(10 + i, M, K))
        offsets.copy_(offsets_of(loads_of(i, M, E)))
        want_a, want_b = lin.forward(x).clone(), ex.forward(x, offsets, 0.9, rows=rows).clone()
        torch.cuda.synchronize()
        graph.replay()
        lin.forward(x[:5])
        torch.cuda.synchronize()
        assert torch.equal(a, want_a) and torch.equal(b, want_b)
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = []
    for st in streams:
        with torch.cuda.stream(st):
            got.append((lin.forward(x), ex.forward(x, offsets, 0.9, rows=rows)))
    torch.cuda.synchronize()
    assert all(torch.equal(p, want_a) and torch.equal(r, want_b) for p, r in got)


def test_addresses_beyond_32_bits():
    """Codes, weights of an expert and outputs that lie more than 2^32 bytes behind their tensors' starts."""
    M, K, N = 270_000, 16384, 24
    q = torch.zeros((M, K), dtype=I8, device="cuda")
    some = torch.tensor([0, 1, 262_143, 262_144, 262_145, M - 130, M - 1], device="cuda")
    q[some] = codes(1, len(some), K)
    s, qw, sw = torch.rand(M, device="cuda"), codes(2, N, K), rand(3, N).abs()
    y = svdq.linear_w8a8(q, s, qw, sw, out_dtype=F32)
    check_product(y[some], q[some], s[some], qw, sw, None)
    assert int((y != 0).any(dim=1).sum()) <= len(some)
    y = Guarded(3, 5000, BF16, ld=3_000_000_000 // 2)
    w, b = codes(4, 5000, 64), rand(5, 5000).abs()
    svdq.linear_w8a8(q[:3, :64].contiguous(), s[:3], w, b, out=y.t)
    check_product(y.t, q[:3, :64], s[:3], w, b, None)
    del y, q
    E, N, K, M = 70, 8192, 8192, 140
    qw = torch.empty((E, N, K), dtype=I8, device="cuda")
    qw.view(-1, K).copy_(codes(6, 8192, K).repeat(E, 1))
    for e in range(E):
        qw[e, :, :16] = e
    q, s, sw, o = codes(7, M, K), rand(8, M).abs(), 0.1 + torch.rand((E, N), device="cuda"), offsets_of([2] * E)
    check_grouped(svdq.linear_w8a8_grouped(q, s, o, qw, sw), q, s, o, qw, sw, None)
    x = rand(9, 5, 16384).to(BF16)
    big = torch.zeros((270_000, 16384), dtype=BF16, device="cuda")
    big[-5:] = x
    rows = torch.arange(270_000 - 5, 270_000, dtype=I32).cuda()
    check_quantised(*svdq.quantize_act_int8_grouped(big, offsets_of([5]), rows=rows), *quantise64(x, None, 1.0))


@pytest.mark.parametrize("M,N,K", [(40, 70, 16), (64, 33, 112), (300, 130, 144), (64, 64, 400), (500, 1000, 528), (1024, 2560, 1008), (130, 5120, 1552), (200, 5120, 2064), (40, 48, 640)])
@pytest.mark.parametrize("at_q,at_w", [(16, 0), (0, 48), (112, 112), (64, 96)])
def test_operands_that_begin_anywhere_in_a_line(M, N, K, at_q, at_w):
    """Rows of codes and weights at every sixteenth byte of a memory line."""
    q, qw = (codes(s, n * K + 256)[at:at + n * K].view(n, K) for s, n, at in ((1, M, at_q), (2, N, at_w)))
    s, sw, bias = 0.01 + rand(3, M).abs(), 0.01 + rand(4, N).abs(), rand(5, N)
    for dtype in (BF16, F32):
        check_product(svdq.linear_w8a8(q, s, qw, sw, bias, out_dtype=dtype), q, s, qw, sw, bias)
    E = 3
    qw = codes(6, E * N * K + 256)[at_w:at_w + E * N * K].view(E, N, K)
    sw, offsets = 0.01 + rand(7, E, N).abs(), offsets_of([M // 3, 0, M - M // 3])
    check_grouped(svdq.linear_w8a8_grouped(q, s, offsets, qw, sw), q, s, offsets, qw, sw, None)


@pytest.mark.parametrize("N,K,E", [(512, 512, 0), (2048, 1408, 0), (640, 4096, 0), (512, 528, 8), (256, 64, 300)])
def test_last_rows_whose_codes_stay_on_the_chip(N, K, E):
    """The most rows that are one launch without memory for codes, and one more."""
    lead = (E,) if E else ()
    qw, sw, bias, il = codes(1, *lead, N, K), 0.001 * rand(2, *lead, N).abs(), rand(3, *lead, N), 0.5 + rand(4, *lead, K).abs()
    module = svdq.W8A8Experts(il, qw, sw, bias) if E else svdq.W8A8Linear(il, qw, sw, bias)
    most = module._descriptor().rows_on_chip
    for M in (most, most + 1):
        x = rand(5, M, K).to(BF16)
        if E:
            offsets = offsets_of([1] * min(E, M) + [0] * (E - min(E, M)))
            offsets[-1] = M                                            # the last expert has the rest: as many tiles as there can be
            qx, sx = svdq.quantize_act_int8_grouped(x, offsets, il, 0.9)
            want, got = svdq.linear_w8a8_grouped(qx, sx, offsets, qw, sw, bias), module.forward(x, offsets, 0.9)
        else:
            want, got = svdq.linear_w8a8(*svdq.quantize_act_int8(x, il, 0.9), qw, sw, bias), module.forward(x, 0.9)
        assert torch.equal(got, want)


@pytest.mark.parametrize("M,N,K", [(3, 40, 272), (700, 600, 1552)])
def test_rows_of_an_x_without_rows(M, N, K):
    """Zeros all of them, in one launch and in two: codes and scales 0, outputs the biases."""
    E = 2
    x, rows, offsets = torch.empty((0, K), dtype=BF16, device="cuda"), torch.arange(-1, M - 1, dtype=I32).cuda(), offsets_of([M // 3, M - M // 3])
    il, qw, sw, bias = 0.5 + rand(1, E, K).abs(), codes(2, E, N, K), rand(3, E, N).abs(), rand(4, E, N)
    qx, sx = svdq.quantize_act_int8_grouped(x, offsets, il, 0.9, rows=rows)
    assert not qx.any() and not sx.any()
    assert torch.equal(svdq.W8A8Experts(il, qw, sw, bias).forward(x, offsets, 0.9, rows=rows), bias[experts_of(offsets, M)].to(BF16))


@pytest.mark.parametrize("K,N", [(272, 40), (2064, 600)])
def test_scales_that_would_be_infinite(K, N):
    """From a row's own ratio: 0, as every scale that is no normal number, with codes 0 and the biases as outputs; the largest finite scale is an ordinary one."""
    M = 6
    x = torch.zeros((M, K), dtype=BF16, device="cuda")
    x[:, 1], x[:, 2] = 2.0, -1.0
    rho = torch.tensor([1.0, float("inf"), 3e38, 1.5e38, 1.7e38, -float("inf")]).cuda()   # 2 rho past 3.4e38: rows 1, 2; and -inf, not positive
    offsets, qw, sw, bias = offsets_of([2, 4]), codes(1, 2, N, K), rand(2, 2, N).abs() * 1e-38, rand(3, 2, N)
    none = torch.tensor([False, True, True, False, False, True], device="cuda")
    qx, sx = svdq.quantize_act_int8_grouped(x, offsets, rho=rho)
    assert bool((sx[none] == 0).all()) and not qx[none].any()
    check_quantised(qx[~none], sx[~none], *quantise64(x[~none], None, rho[~none]))
    y = svdq.W8A8Experts(None, qw, sw, bias).forward(x, offsets, rho)
    assert torch.equal(y[none], bias[experts_of(offsets, M)].to(BF16)[none]) and bool(torch.isfinite(y[0]).all())
    assert torch.equal(y.view(torch.int16), svdq.linear_w8a8_grouped(qx, sx, offsets, qw, sw, bias).view(torch.int16))
