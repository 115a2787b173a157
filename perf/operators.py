"""Performance cases of the 8-bit layer and of its products grouped by expert.

Operators, by `kind`:

  product   y = (qx qw^T) sx sw + bias from 8-bit codes: one scale a token (sx), one a channel (sw), 32-bit integer sums
  layer     the same from bf16 activations: smoothing, one clipped scale a token, 8-bit codes, then the product.  `gelu`: of
            the activated input, as in front of a feed-forward block's down-projection
  grouped   the product where rows are ordered by expert and expert e multiplies rows offsets[e] .. offsets[e + 1]
  experts   the grouped layer: rows gathered from tokens in the experts' order (`tokens`: so many, each taken as often as there
            are rows for it), smoothed by their expert's vector, clipped by their own ratio, quantised and multiplied

A token's scale is s = (rho max|x^|) / 127 with x^ = x inv_lambda and its codes are the whole numbers nearest to x^ (1 / s), at
most 127, each step one binary32 operation; outputs are bf16, or binary32 where `f32` is set.

Inputs are synthetic: Gaussian activations with a few outlier channels, N(0, 0.02^2) weights rounded to 8 bits by channel.
Expert loads fall off as a power of their rank (`skew`), the ranks dealt to experts by the seed.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
HIDDEN, FFN = 5120, 13824                       # widths of the DiT block that bench.py times
LARGEST = 75600 * FFN * HIDDEN                  # products of the largest listed case


def listed():
    return [
        # one row through the widest projection of a DiT block's conditioning (the step's embedding to six modulation vectors):
        # nothing but the weights to read, and the launch
        dict(name="product_1", kind="product", M=1, K=HIDDEN, N=6 * HIDDEN, f32=True),
        # a handful of tokens, a decoding batch or a short conditioning sequence, on the hidden width
        dict(name="product_24", kind="product", M=24, K=HIDDEN, N=HIDDEN, f32=False),
        # a ragged token count and an odd number of channels, K no multiple of a tile's depth
        dict(name="product_ragged", kind="product", M=2305, K=4112, N=4999, f32=True),
        # a feed-forward down-projection of a 480p clip from codes that another pass made
        dict(name="product_480p", kind="product", M=32760, K=FFN, N=HIDDEN, f32=False),
        # a single small layer: launches and the host's path
        dict(name="layer_tiny", kind="layer", M=256, K=512, N=512, gelu=False),
        # key / value projection of a 512-token conditioning sequence
        dict(name="layer_cond512", kind="layer", M=512, K=HIDDEN, N=HIDDEN, gelu=False),
        # attention output projection of a 480p clip, the module that a 4-bit model keeps at more bits
        dict(name="layer_attn480p", kind="layer", M=32760, K=HIDDEN, N=HIDDEN, gelu=False),
        # feed-forward down-projection of a 720p clip behind its GELU, the other module that is kept at more bits
        dict(name="layer_ffn720p", kind="layer", M=75600, K=FFN, N=HIDDEN, gelu=True),
        # decoding with many experts: a few rows, most experts with none
        dict(name="grouped_decode", kind="grouped", M=32, E=64, K=2048, N=2816, skew=0.5),
        # a prompt over few wide experts, uneven loads
        dict(name="grouped_wide", kind="grouped", M=16384, E=8, K=4096, N=14336, skew=0.7),
        # a prompt over many narrow experts from its tokens on: 2048 tokens, each taken by eight experts, ragged and some empty
        dict(name="experts_prompt", kind="experts", M=16384, tokens=2048, E=128, K=2048, N=1536, skew=1.0),
        # clips at different denoising steps in one batch, rows of the early steps for one expert and of the late steps for the other
        dict(name="experts_two", kind="experts", M=32760, tokens=32760, E=2, K=HIDDEN, N=HIDDEN, skew=1.0),
    ]


def _log(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // multiple * multiple, max(multiple, int(round(v / multiple)) * multiple))


def draw(rng):
    kind = rng.choice(["product", "layer", "grouped", "experts"])
    K = _log(rng, 64, FFN, 16)
    if kind in ("product", "layer"):
        N = _log(rng, 8, 6 * HIDDEN)
        M = _log(rng, 1, min(75600, LARGEST // (N * K), 75600 * FFN // N))
        if kind == "product":
            return dict(kind=kind, M=M, K=K, N=N, f32=rng.random() < 0.3)
        return dict(kind=kind, M=M, K=K, N=N, gelu=rng.random() < 0.3)
    N = _log(rng, 64, 14336, rng.choice([1, 8, 128]))
    E = _log(rng, 2, min(256, max(2, 1500000000 // (N * K))))
    M = _log(rng, 1, min(32760, LARGEST // (N * K)))
    skew = rng.choice([0.0, 0.5, 1.0, 1.5])
    if kind == "grouped":
        return dict(kind=kind, M=M, E=E, K=K, N=N, skew=skew)
    return dict(kind=kind, M=M, tokens=max(1, M // rng.choice([1, 2, 4, 8])), E=E, K=K, N=N, skew=skew)


def _loads(case):
    """Rows of each expert, by rank: shares of M that fall off as a power of the rank, rounded so that they sum to M."""
    E, M = case["E"], case["M"]
    share = [(r + 1.0) ** -case["skew"] for r in range(E)]
    ends = [0.0]
    for s in share:
        ends.append(ends[-1] + s)
    cut = [round(M * v / ends[-1]) for v in ends]
    return [b - a for a, b in zip(cut, cut[1:])]


# ---- inputs ------------------------------------------------------------------------------------
def _activations(g, M, K, gelu=False):
    """[M, K] bf16: N(0, 1) with 0.5 % outlier channels x 20, or the spread of a tensor in front of a GELU."""
    x = torch.randn((M, K), generator=g, device=DEVICE, dtype=torch.bfloat16)
    if gelu:
        return x.mul_(1.5)
    x[:, torch.randperm(K, generator=g, device=DEVICE)[:max(1, K // 200)]] *= 20.0
    return x


def _weights(g, shape):
    """8-bit codes of N(0, 0.02^2) weights, nearest on each channel's grid, and the channels' scales."""
    qw = torch.empty(shape, dtype=torch.int8, device=DEVICE)
    sw = torch.empty(shape[:-1], dtype=torch.float32, device=DEVICE)
    for q, s in zip(qw.view(-1, *shape[-2:]), sw.view(-1, shape[-2])):
        w = torch.randn(q.shape, generator=g, device=DEVICE).mul_(0.02)
        s.copy_(w.abs().amax(dim=1) / 127.0)
        q.copy_(w.div_(s[:, None]).round_())
    return qw, sw


def _codes(g, M, K):
    """8-bit codes of Gaussian tokens, the largest of each at 127, and scales around those that such tokens get."""
    z = torch.randn((M, K), generator=g, device=DEVICE)
    z *= 127.0 / z.abs().amax(dim=1, keepdim=True)
    return z.round_().to(torch.int8), 0.02 + 0.02 * torch.rand(M, generator=g, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    kind, M, K, N, E = case["kind"], case["M"], case["K"], case["N"], case.get("E")
    s = dict(kind=kind, gelu=case.get("gelu", False), dtype=torch.float32 if case.get("f32") else torch.bfloat16)
    s["qw"], s["sw"] = _weights(g, (E, N, K) if E else (N, K))
    s["bias"] = torch.randn((E, N) if E else (N,), generator=g, device=DEVICE) * 0.01
    if E:
        loads = _loads(case)
        random.Random(seed).shuffle(loads)
        s["loads"] = loads                       # known where rows were put in the experts' order
        s["offsets"] = torch.tensor([0] + loads).cumsum(0).to(torch.int32).to(DEVICE)
    if kind in ("product", "grouped"):
        s["qx"], s["sx"] = _codes(g, M, K)
        return s
    s["inv_lambda"] = 0.5 + torch.rand((E, K) if E else (K,), generator=g, device=DEVICE)
    if kind == "layer":
        s["x"], s["rho"] = _activations(g, M, K, s["gelu"]), random.Random(seed).choice([0.8, 0.9, 1.0])
    else:
        s["x"] = _activations(g, case["tokens"], K)
        s["rows"] = (torch.randperm(M, generator=g, device=DEVICE) % case["tokens"]).to(torch.int32)
        s["rho"] = torch.tensor([0.8, 0.9, 1.0], device=DEVICE)[torch.randint(3, (M,), generator=g, device=DEVICE)]
    if own:                                      # handles: they keep references, and buffers from their first call on
        import paper_2605_27003_amd as svdq
        made = svdq.W8A8Experts if E else svdq.W8A8Linear
        s["module"] = made(s["inv_lambda"], s["qw"], s["sw"], s["bias"])
    return s


# ---- one pass ----------------------------------------------------------------------------------
def _quantise(x, inv_lambda, rho, gelu):
    """Codes, as numbers, and scales of x [M, K]; inv_lambda [K] or [M, K], rho a number or [M]."""
    x = x.float()
    if gelu:
        x = (x / (1.0 + torch.exp(-1.5957691216057308 * (x + 0.044715 * x * x * x)))).to(torch.bfloat16).float()
    x = x * inv_lambda
    s = rho * x.abs().amax(dim=1) / torch.full((), 127.0, device=x.device)
    fine = s >= torch.finfo(torch.float32).tiny
    s = torch.where(fine, s, torch.zeros_like(s))
    inv = torch.where(fine, 1.0 / s, torch.zeros_like(s))
    return (x * inv[:, None]).round().clamp(-127.0, 127.0), s


def _product(q, s, qw, sw, bias):
    return (q.float() @ qw.float().t()) * s[:, None] * sw + bias


def _grouped(q, s, st):
    parts = zip(q.split(st["loads"]), s.split(st["loads"]), st["qw"], st["sw"], st["bias"])
    return torch.cat([_product(*p) for p in parts if len(p[0])])


def run(s):
    kind = s["kind"]
    if own:
        if kind == "layer":
            return s["module"].forward(s["x"], s["rho"], gelu=s["gelu"])
        if kind == "experts":
            return s["module"].forward(s["x"], s["offsets"], s["rho"], rows=s["rows"])
        import paper_2605_27003_amd as svdq
        if kind == "product":
            return svdq.linear_w8a8(s["qx"], s["sx"], s["qw"], s["sw"], s["bias"], out_dtype=s["dtype"])
        return svdq.linear_w8a8_grouped(s["qx"], s["sx"], s["offsets"], s["qw"], s["sw"], s["bias"], out_dtype=s["dtype"])
    if kind == "product":
        y = _product(s["qx"], s["sx"], s["qw"], s["sw"], s["bias"])
    elif kind == "layer":
        y = _product(*_quantise(s["x"], s["inv_lambda"], s["rho"], s["gelu"]), s["qw"], s["sw"], s["bias"])
    elif kind == "grouped":
        y = _grouped(s["qx"], s["sx"], s)
    else:
        rows = torch.arange(s["rows"].numel(), device=DEVICE)
        expert = torch.bucketize(rows, s["offsets"][1:-1], right=True)
        y = _grouped(*_quantise(s["x"][s["rows"]], s["inv_lambda"][expert], s["rho"], False), s)
    return y.to(s["dtype"])


# ---- what a pass cannot do without -------------------------------------------------------------
def work(case):
    kind, M, K, N = case["kind"], case["M"], case["K"], case["N"]
    experts = sum(n > 0 for n in _loads(case)) if "E" in case else 1
    b = experts * (K * N + 8 * N) + M * N * (4 if case.get("f32") else 2)
    if kind in ("product", "grouped"):
        b += M * K + 4 * M
    else:
        b += min(M, case.get("tokens", M)) * K * 2 + experts * 4 * K
    if kind == "experts":
        b += 8 * M                               # each row's token and clipping ratio
    if "E" in case:
        b += 4 * (case["E"] + 1)
    return {"bytes": float(b), "flops": 2.0 * M * N * K}


# ---- the definition in 64 bits -----------------------------------------------------------------
def _f32(t):
    """Rounded to binary32, held in 64 bits: one binary32 operation of a definition (products of a binary32 and a bf16 or
    binary32 number are exact in 64 bits or far from a tie, quotients never so near one that the second rounding matters)."""
    return t.to(torch.float32).to(torch.float64)


def _exact_codes(x, inv_lambda, rho, gelu):
    x = x.to(torch.float64)
    if gelu:
        x = (x * 0.5 * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))).to(torch.bfloat16).to(torch.float64)
    x = _f32(x * inv_lambda.to(torch.float64))
    if not torch.is_tensor(rho):
        rho = torch.tensor(rho, dtype=torch.float32, device=x.device)
    s = _f32(_f32(x.abs().amax(dim=1) * rho.to(torch.float64)) / 127.0)
    s[s < 2.0 ** -126] = 0.0
    inv = torch.zeros_like(s)
    inv[s > 0] = _f32(1.0 / s[s > 0])
    q = torch.round(_f32(x * inv[:, None]))
    return q.clamp_(-127.0, 127.0), s


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("product", "grouped"):
        q, sx = s["qx"].to(torch.float64), s["sx"].to(torch.float64)
    elif case["kind"] == "layer":
        q, sx = _exact_codes(s["x"], s["inv_lambda"], s["rho"], s["gelu"])
    else:
        expert = torch.repeat_interleave(torch.tensor(s["loads"])).to(DEVICE)
        q, sx = _exact_codes(s["x"][s["rows"].long()], s["inv_lambda"][expert], s["rho"], False)
    N = case["N"]
    y = torch.empty((case["M"], N), dtype=torch.float64, device=DEVICE)
    qw, sw, bias = s["qw"].view(-1, N, case["K"]), s["sw"].view(-1, N), s["bias"].view(-1, N)
    begin = 0
    for e, n in enumerate(s.get("loads", [case["M"]])):
        if n:
            t = torch.mm(q[begin:begin + n], qw[e].to(torch.float64).t())
            y[begin:begin + n] = t * sx[begin:begin + n, None] * sw[e].to(torch.float64) + bias[e].to(torch.float64)
        begin += n
    return y
