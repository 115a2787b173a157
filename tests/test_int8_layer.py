"""The 8-bit layer's host side (no GPU): what the C ABI and the Python functions refuse."""
import copy
import ctypes

import pytest
import torch

import paper_2605_27003_amd as svdq
from paper_2605_27003_amd import binding

INV, SHAPE = -1, -2
A, Z, F32, BF16 = 256, None, torch.float32, torch.bfloat16


def test_quantise_refusals():
    q = binding.load_library().svdq_quantize_act_int8
    ok = dict(x=A, ldx=512, il=A, rho=0.9, gelu=0, M=4, K=512, qx=A, sx=A)
    call = lambda **kw: q(*{**ok, **kw}.values(), Z)
    for kw in (dict(x=Z), dict(qx=Z), dict(sx=Z), dict(M=-1), dict(rho=0.0), dict(rho=1.5), dict(rho=float("nan"))):
        assert call(**kw) == INV, kw
    for kw in (dict(K=0), dict(K=-16), dict(K=520), dict(K=32768 + 16, ldx=40000), dict(ldx=496), dict(ldx=516), dict(x=A + 8), dict(il=A + 4), dict(qx=A + 8),
               dict(sx=A + 2), dict(M=(1 << 26) + 1)):
        assert call(**kw) == SHAPE, kw
    assert call(M=0) == 0 and call(M=0, il=Z) == 0


def test_product_refusals():
    g = binding.load_library().svdq_linear_w8a8
    ok = dict(qx=A, sx=A, qw=A, sw=A, bias=Z, M=4, N=100, K=512, y=A, ldy=100, dtype=0)
    call = lambda **kw: g(*{**ok, **kw}.values(), Z)
    for kw in (dict(qx=Z), dict(sx=Z), dict(qw=Z), dict(sw=Z), dict(y=Z), dict(M=-1), dict(dtype=2)):
        assert call(**kw) == INV, kw
    for kw in (dict(N=0), dict(K=0), dict(K=40), dict(K=32784), dict(ldy=99), dict(qx=A + 8), dict(qw=A + 4), dict(sx=A + 2), dict(sw=A + 1), dict(bias=A + 2),
               dict(y=A + 1), dict(y=A + 2, dtype=1), dict(M=(1 << 26) + 1), dict(M=1 << 26, N=1 << 30, ldy=1 << 30)):
        assert call(**kw) == SHAPE, kw
    assert call(M=0) == 0


def test_grouped_refusals():
    lib = binding.load_library()
    ok = dict(x=A, ldx=512, x_rows=9, rows=A, offsets=A, E=3, il=A, rho=0.9, row_rho=Z, gelu=0, M=4, K=512, qx=A, sx=A)
    call = lambda **kw: lib.svdq_quantize_act_int8_grouped(*{**ok, **kw}.values(), Z)
    for kw in (dict(offsets=Z), dict(E=0), dict(E=-1), dict(x_rows=-1), dict(rho=2.0), dict(x=Z)):
        assert call(**kw) == INV, kw
    for kw in (dict(E=1025), dict(offsets=A + 2), dict(rows=A + 2), dict(row_rho=A + 1), dict(K=24)):
        assert call(**kw) == SHAPE, kw
    assert call(M=0) == 0 and call(M=0, rows=Z, x_rows=-1) == 0 and call(M=0, rho=0.0, row_rho=A) == 0
    ok2 = dict(qx=A, sx=A, qw=A, sw=A, bias=A, offsets=A, E=3, M=4, N=100, K=512, y=A, ldy=100, dtype=1)
    call2 = lambda **kw: lib.svdq_linear_w8a8_grouped(*{**ok2, **kw}.values(), Z)
    assert call2(offsets=Z) == INV and call2(E=0) == INV and call2(E=1025) == SHAPE and call2(ldy=8) == SHAPE and call2(M=0) == 0
    layer = binding._LayerInt8(0, 100, 512, A, A, A, A)
    ok3 = dict(layer=ctypes.addressof(layer), x=A, ldx=512, x_rows=4, rows=Z, offsets=Z, rho=0.9, row_rho=Z, gelu=0, M=4, qx=A, sx=A, y=A, ldy=104)
    call3 = lambda **kw: lib.svdq_layer_int8_forward(*{**ok3, **kw}.values(), Z)
    assert call3(layer=Z) == INV and call3(offsets=A) == INV and call3(rows=A) == INV and call3(row_rho=A) == INV      # not a grouped layer
    assert call3(ldy=96) == SHAPE and call3(sx=Z) == INV and call3(M=0) == 0
    layer.E = 2
    assert call3() == INV and call3(offsets=A, M=0) == 0 and call3(offsets=A, rho=-1.0) == INV
    layer.E = -1
    assert call3(offsets=A) == INV


def test_python_refuses_what_the_kernels_would_misread():
    """Tensors off the GPU, of other types, shapes or orders never reach a kernel."""
    x, qx = torch.zeros((4, 64), dtype=BF16), torch.zeros((4, 64), dtype=torch.int8)
    qw, s = torch.zeros((8, 64), dtype=torch.int8), torch.ones(8)
    for call in (lambda: svdq.quantize_act_int8(x), lambda: svdq.linear_w8a8(qx, torch.ones(4), qw, s),
                 lambda: svdq.quantize_act_int8_grouped(x, torch.zeros(3, dtype=torch.int32)),
                 lambda: svdq.linear_w8a8_grouped(qx, torch.ones(4), torch.zeros(2, dtype=torch.int32), qw[None], s[None]),
                 lambda: svdq.W8A8Linear(None, qw, s).forward(x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for bad in (x.float(), x[0], x[:, ::2]):
        with pytest.raises(ValueError):
            svdq.quantize_act_int8(bad)
    for args in ((None, qw.float(), s), (None, qw, s.double()), (None, qw, s[:4]), (None, qw[:, ::2], s), (torch.ones(32), qw, s), (None, qw, s, torch.ones(1)),
                 (None, qw[None], s[None])):
        with pytest.raises(ValueError):
            svdq.W8A8Linear(*args)
    for args in ((None, qw, s), (None, qw[None], s), (torch.ones(64), qw[None], s[None])):
        with pytest.raises(ValueError):
            svdq.W8A8Experts(*args)


def test_the_layers_descriptor_follows_its_tensors():
    qw, s = torch.zeros((8, 64), dtype=torch.int8), torch.ones(8)
    lin = svdq.W8A8Linear(None, qw, s)
    first = lin._descriptor()
    assert lin._descriptor() is first and (first.E, first.N, first.K, first.bias) == (0, 8, 64, None)
    lin.bias = torch.ones(8)
    assert lin._descriptor().bias == lin.bias.data_ptr()
    other = copy.deepcopy(lin)
    assert other._descriptor().qw == other.qw.data_ptr() != qw.data_ptr()
    lin.sw = torch.ones(9)
    with pytest.raises(ValueError):
        lin._descriptor()


def test_descriptor_follows_memory_given_to_the_same_tensor():
    qw, sw, bias, il = torch.zeros((32, 48), dtype=torch.int8), torch.ones(32), torch.ones(32), torch.ones(48)
    layer = svdq.W8A8Linear(il, qw, sw, bias)
    first = layer._descriptor()
    assert layer._descriptor() is first and first.qw == qw.data_ptr()
    for name in ("inv_lambda", "qw", "sw", "bias"):
        held = getattr(layer, name)
        held.data = held.clone()
        assert getattr(layer._descriptor(), name) == held.data_ptr()
    layer.qw.data = torch.zeros((32, 64), dtype=torch.int8)
    with pytest.raises(ValueError, match="inv_lambda"):
        layer._descriptor()


def test_rows_whose_codes_stay_on_the_chip():
    """Without memory for codes and scales: up to svdq_layer_int8_rows_on_chip rows, and where y is not x."""
    lib = binding.load_library()

    def rows(E, N, K):
        layer = binding._LayerInt8(E, N, K, A, A, A, A)
        return lib.svdq_layer_int8_rows_on_chip(ctypes.addressof(layer))
    # 512 tiles of 16 x 32 up to K = 1408; four rows of a longer K; nothing beyond 4096
    assert [rows(*a) for a in ((0, 512, 512), (0, 512, 1408), (0, 512, 1424), (0, 32, 4096), (0, 32, 4112), (0, 16384, 64), (0, 16416, 64))] == [512, 512, 4, 4, 0, 16, 0]
    # an expert with rows can add a tile that is not full
    assert rows(8, 512, 512) == 16 * (32 - 8) + 15 and rows(1024, 512, 512) == 31 and rows(1, 32, 64) == 16 * 511 + 15
    assert [rows(*a) for a in ((0, 0, 64), (0, 32, 72), (-1, 32, 64), (1025, 32, 64), (0, 32, 0))] == [0] * 5 and lib.svdq_layer_int8_rows_on_chip(None) == 0
    far = 1 << 30
    layer = binding._LayerInt8(0, 512, 512, A, A, A, A)
    ok = dict(L=ctypes.addressof(layer), x=A, ldx=512, x_rows=0, rows=Z, offsets=Z, rho=0.9, row_rho=Z, gelu=0, M=4, qx=Z, sx=Z, y=far, ldy=512)
    call = lambda **kw: lib.svdq_layer_int8_forward(*{**ok, **kw}.values(), Z)
    assert call(M=0) == 0
    for kw in (dict(M=513), dict(y=A), dict(qx=A), dict(sx=A)):
        assert call(**kw) == INV, kw


@pytest.mark.parametrize("grouped", [False, True])
def test_descriptor_follows_views_given_to_the_same_tensor(grouped):
    """A smaller view, another type or another order of the memory that a held tensor has already: taken up, or refused."""
    E, N, K = 2, 48, 48
    lead = (E,) if grouped else ()

    def made():
        return (svdq.W8A8Experts if grouped else svdq.W8A8Linear)(torch.ones(lead + (K,)), torch.zeros(lead + (N, K), dtype=torch.int8), torch.ones(lead + (N,)),
                                                                  torch.ones(lead + (N,)))
    layer = made()
    first = layer._descriptor()
    for name in ("qw", "sw", "bias"):                                 # fewer channels, from where the held ones begin
        held = getattr(layer, name)
        held.data = held.data.flatten()[:held.numel() // 3].view(*lead, N // 3, *held.shape[1 + grouped:])
    now = layer._descriptor()
    assert (now.N, now.K, now.qw, now.sw, now.bias) == (N // 3, K, first.qw, first.sw, first.bias) and now.shape[1] == N // 3
    # one tensor alone no longer fits the others, is of another type, or has its values in another order
    for name in ("inv_lambda", "qw", "sw", "bias"):
        half = lambda t: t.flatten()[:t.numel() // 2].view(*t.shape[:-1], t.shape[-1] // 2)
        for change in (half, lambda t: t.view(torch.uint8 if t.dtype is torch.int8 else torch.int32), lambda t: t[..., None],
                       lambda t: t.as_strided(t.shape, (0,) * t.dim()), lambda t: t.mT if t.shape == lead + (N, K) and t.dtype is torch.int8 else t[..., :1]):
            layer = made()
            held = getattr(layer, name)
            layer._descriptor()
            held.data = change(held.data)
            with pytest.raises(ValueError):
                layer._descriptor()
            with pytest.raises(ValueError):                           # not on the second call either
                layer._descriptor()
    layer = made()
    layer._descriptor()
    layer.qw.transpose_(-1, -2)
    with pytest.raises(ValueError, match="qw"):
        layer._descriptor()


def test_rows_of_an_x_without_rows_are_not_refused():
    """An empty tensor has no address: x is needed only where a row number can lie within it.  (K = 520 and ldy = 96 are refused behind that check.)"""
    lib = binding.load_library()
    ok = dict(x=Z, ldx=520, x_rows=0, rows=A, offsets=A, E=3, il=A, rho=0.9, row_rho=Z, gelu=0, M=4, K=520, qx=A, sx=A)
    call = lambda **kw: lib.svdq_quantize_act_int8_grouped(*{**ok, **kw}.values(), Z)
    assert call() == SHAPE and call(x_rows=1) == INV and call(rows=Z) == INV and call(qx=Z) == INV
    layer = binding._LayerInt8(2, 100, 512, A, A, A, A)
    ok = dict(layer=ctypes.addressof(layer), x=Z, ldx=512, x_rows=0, rows=A, offsets=A, rho=0.9, row_rho=Z, gelu=0, M=4, qx=A, sx=A, y=A, ldy=96)
    call = lambda **kw: lib.svdq_layer_int8_forward(*{**ok, **kw}.values(), Z)
    assert call() == SHAPE and call(x_rows=1) == INV and call(rows=Z) == INV
