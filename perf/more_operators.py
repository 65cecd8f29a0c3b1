"""What the performance of the 4-bit operators and of gradient clipping is measured on: microscaled 4-bit floating point (blocks of 32 values
that share a power of two), its products, and the global norm of many gradients with the clipping by it.

A program that uses them holds a scoring head W [V][F] over V items (or codewords), or the layers below one, in 4 bits: it quantises W and its
features X [R][F] in blocks of 32, forms the logits X W^T as a 4-bit product, goes back through the same product for the gradients
of X and W, and clips all gradients by their global norm before the update.  A program that only answers keeps W's codes and
takes one query or a few at a time.  Feature lengths are this repository's query dimensions (96, 128, 960) or generic powers of two; numbers of
items are its database sizes (10^4, 10^6), its codebooks' (16 * 256 codewords) or generic.

Kinds of case:
  roundtrip  values [rows][cols] -> codes and scales -> the values that these stand for, by rows, or by rows and columns
  product    X [M][K] as values, or held as codes, W [N][K] held as codes -> X W^T [M][N]
  norm       gradients -> their global norm
  clip       gradients -> norm, and the gradients times a factor that brings the norm to at most 1, in buffers of another type or the same
  step       a layer's forward and backward products from X, W and the gradient of its outputs, the gradient of W clipped in its place
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_SMALLEST_AMAX = 2.0 ** -100
_MOST_EXPONENT = 125        # 6 * 2^125 is finite


def listed():
    return [
        # a service's batch of 100 queries, the longest query dimension here: launch latency
        dict(name="roundtrip_queries", kind="roundtrip", rows=100, cols=960, type="bf16", out="bf16", block=1, fit=False, both=False),
        # the weights after an update in 32 bits, as the forward and the backward product want them
        dict(name="roundtrip_weights", kind="roundtrip", rows=10007, cols=4096, type="f32", out="bf16", block=32, fit=True, both=True),
        # one query scored against a head: reading the weights is all there is
        dict(name="product_single", kind="product", M=1, N=16384, K=4096, type="bf16", out="bf16", held=False, fit=False),
        # a handful of queries against every item of a database of a million
        dict(name="product_items", kind="product", M=8, N=1_000_000, K=960, type="bf16", out="f32", held=False, fit=False),
        # nothing is a round number
        dict(name="product_ragged", kind="product", M=333, N=5003, K=1000, type="f16", out="f32", held=False, fit=True),
        # two matrices that are both held: all codewords against all items
        dict(name="product_held", kind="product", M=4096, N=10_000, K=960, type="f32", out="f16", held=True, fit=False),
        # a training batch against a wide head
        dict(name="product_large", kind="product", M=8192, N=8192, K=8192, type="bf16", out="bf16", held=False, fit=False),
        # a small head over features of three lengths: latency
        dict(name="clip_small", kind="clip", count=6, least=96, most=40_000, type="f32", out="f32", above=True),
        # the gradients of a deep model in 16 bits with a loss scale, into its 32-bit gradients
        dict(name="clip_model", kind="clip", count=290, least=960, most=12_000_000, type="f16", out="f32", above=True),
        # many odd tensors, most of them short, norm below the bound
        dict(name="clip_ragged", kind="clip", count=1000, least=1, most=300_000, type="bf16", out="bf16", above=False),
        # what a rank adds to the norm of all ranks
        dict(name="norm_model", kind="norm", count=64, least=4096, most=16_000_000, type="f32"),
        # a layer from 960 features to 16384 items on a batch
        dict(name="step", kind="step", T=4096, N=16384, K=960, fit=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo + 1, hi))))))


def draw(rng):
    """One more case of the same kinds, sizes spread between a single row or value and the largest listed ones."""
    what = rng.choice(["roundtrip", "roundtrip", "product", "product", "product", "product", "clip", "clip", "norm", "step"])
    half = rng.random() < 0.5
    if what == "roundtrip":
        rows = _log(rng, 1, 16384)
        return dict(kind="roundtrip", rows=rows, cols=_log(rng, 32, min(32768, 4.0e7 / rows)), type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    out=rng.choice(["bf16", "bf16", "f32"]), block=rng.choice([1, 1, 32]), fit=half, both=rng.random() < 0.5)
    if what == "product":
        M = rng.choice([_log(rng, 1, 16), _log(rng, 1, 8192), _log(rng, 1, 8192)])
        K = _log(rng, 96, 16384)
        return dict(kind="product", M=M, N=_log(rng, 256, min(1_000_000, 9.0e8 / K, 6.0e7 / M, 5.0e11 / M / K)), K=K, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    out=rng.choice(["bf16", "bf16", "f32", "f16"]), held=rng.random() < 0.3, fit=half)
    if what in ("norm", "clip"):
        count = _log(rng, 1, 1000)
        least = _log(rng, 1, 10_000)
        c = dict(kind=what, count=count, least=least, most=least + _log(rng, 1, min(2.0e7, 1.0e8 / count)), type=rng.choice(["bf16", "f16", "f32"]))
        if what == "clip":
            c.update(out=rng.choice([c["type"], "f32"]), above=half)
        return c
    T, K = _log(rng, 16, 4096), rng.choice([96, 128, 960, _log(rng, 64, 4096)])
    return dict(kind="step", T=T, N=_log(rng, 256, min(32768, 6.0e10 / T / K)), K=K, fit=half)


def _numbers(c):
    """The tensors' numbers of values: from `least` to `most` in equal ratios, long and short ones mixed."""
    n = c["count"]
    sizes = [int(round(c["least"] * (c["most"] / c["least"]) ** (k / max(1, n - 1)))) for k in range(n)]
    return [sizes[k * 7 % n] if n % 7 else sizes[k * 11 % n] if n % 11 else sizes[k] for k in range(n)]


# ---- inputs

def _gaussian(rows, cols, dtype, g, scale=1.0):
    """Activations have a few channels that are much larger than the rest."""
    x = torch.randn((rows, cols), device="cuda", generator=g).mul_(scale)
    x[:, torch.rand((cols,), device="cuda", generator=g) < 0.01] *= 20.0
    return x.to(dtype)


def _codes_like(rows, cols):
    """A buffer for codes: two to a byte, each row starting on 16 bytes."""
    return torch.zeros((rows, -(-cols // 32) * 16), dtype=torch.uint8, device="cuda")[:, :-(-cols // 2)]


def _scales_like(rows, cols):
    """A buffer for scales: a byte per 32 values, each row starting on 4 bytes."""
    return torch.zeros((rows, -(-cols // 128) * 4), dtype=torch.uint8, device="cuda")[:, :-(-cols // 32)]


def _held(x, block, fit):
    """A matrix as a program holds it: codes and scales."""
    codes, scales = _codes_like(*x.shape), _scales_like(*x.shape)
    c, e = _plain_quantise(x, block, fit)
    codes.copy_(_plain_pack(c))
    scales.copy_(e)
    return codes, scales


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = c["kind"]
    s = dict(c=c)
    if kind == "roundtrip":
        rows, cols = c["rows"], c["cols"]
        s["x"] = _gaussian(rows, cols, _TYPES[c["type"]], g, 0.02 if c["block"] == 32 else 1.0)
        s["codes"], s["scales"] = _codes_like(rows, cols), _scales_like(rows, cols)
        s["out"] = torch.empty((rows, cols), dtype=_TYPES[c["out"]], device="cuda")
        if c["both"]:
            s["codes_t"], s["scales_t"] = _codes_like(cols, rows), _scales_like(cols, rows)
            s["out_t"] = torch.empty((cols, rows), dtype=_TYPES[c["out"]], device="cuda")
    elif kind == "product":
        M, N, K = c["M"], c["N"], c["K"]
        x = _gaussian(M, K, _TYPES[c["type"]], g)
        if c["held"]:
            s["a"], s["a_scales"] = _held(x, 1, c["fit"])
        else:
            s["a"], s["a_scales"] = x, None
        s["w"], s["w_scales"] = _held(torch.randn((N, K), device="cuda", generator=g).mul_(0.02), 32 if N * K < 1 << 28 else 1, c["fit"])
        s["out"] = torch.empty((M, N), dtype=_TYPES[c["out"]], device="cuda")
        s["workspace"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    elif kind in ("norm", "clip"):
        sizes = _numbers(c)
        flat = torch.randn((sum(sizes),), device="cuda", generator=g)
        spread = torch.exp2(4.0 * torch.rand((len(sizes),), device="cuda", generator=g))         # layers differ
        flat *= spread.repeat_interleave(torch.tensor(sizes, device="cuda"))
        norm = flat.square().sum(dtype=torch.float64).sqrt().float()
        s["scale"] = 2.0 ** -12 if c["type"] == "f16" else 1.0                                  # the loss scale's reciprocal
        flat *= (4.0 if c.get("above") else 0.4) / s["scale"] / norm
        flat = flat.to(_TYPES[c["type"]])
        s["grads"] = list(flat.split(sizes))
        s["norm"] = torch.empty((1,), device="cuda")
        s["out"] = torch.empty((sum(sizes),), dtype=_TYPES[c["out"]], device="cuda") if kind == "clip" else None
        s["outs"] = list(s["out"].split(sizes)) if kind == "clip" else None
        s["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        if own:         # the handle over its gradients' addresses that a program makes once; the plain form has none
            from paper_1912_08756_amd import binding as icq
            s["list"] = icq.icq_grad_list_create(s["grads"], s["outs"])
    else:
        T, N, K = c["T"], c["N"], c["K"]
        s["x"] = _gaussian(T, K, torch.bfloat16, g)
        s["w"] = torch.randn((N, K), device="cuda", generator=g).mul_(0.06)
        s["g"] = (torch.randn((T, N), device="cuda", generator=g) * torch.rand((T, 1), device="cuda", generator=g)).to(torch.bfloat16)
        for name, rows, cols in (("x", T, K), ("w", N, K), ("g", T, N)):
            s[name + "_codes"], s[name + "_scales"] = _codes_like(rows, cols), _scales_like(rows, cols)
            s[name + "_codes_t"], s[name + "_scales_t"] = _codes_like(cols, rows), _scales_like(cols, rows)
        s["y"], s["dx"] = torch.empty((T, N), dtype=torch.bfloat16, device="cuda"), torch.empty((T, K), dtype=torch.bfloat16, device="cuda")
        s["dw"], s["norm"] = torch.empty((N, K), device="cuda"), torch.empty((1,), device="cuda")
        s["workspace"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
        if own:
            from paper_1912_08756_amd import binding as icq
            s["list"] = icq.icq_grad_list_create([s["dw"]])
    return s


# ---- the plain forms

def _plain_quantise(x, block, fit):
    """(codes [rows][cols], biased exponents of the scales [rows][blocks of 32]) of a matrix; with block = 32 the squares of 32 x 32 share a scale."""
    rows, cols = x.shape
    x = x.float()
    pad = torch.nn.functional.pad(x.abs(), (0, -cols % 32, 0, -rows % block))
    amax = pad.view(pad.shape[0] // block, block, pad.shape[1] // 32, 32).amax((1, 3))          # (a NaN is the largest)
    del pad
    bad = ~torch.isfinite(amax)
    mantissa, exponent = torch.frexp(torch.where(bad, 1.0, amax).clamp(min=_SMALLEST_AMAX))    # amax = mantissa * 2^exponent, mantissa in [0.5, 1); 6 = 0.75 * 2^3
    exponent = exponent - 3
    if fit:
        exponent = (exponent + (mantissa > 0.75).int()).clamp(max=_MOST_EXPONENT)
    bad, exponent = bad.repeat_interleave(block, 0)[:rows], exponent.repeat_interleave(block, 0)[:rows]
    a = torch.ldexp(x, -exponent.repeat_interleave(32, 1)[:, :cols])
    sign = a < 0
    a = a.abs_()
    # steps of 1/2 up to 2, of 1 up to 4, of 2 up to 6, ties to the even code
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, 2 + torch.round(a), 4 + torch.round(a / 2).clamp(max=3)))
    code = torch.where(bad.repeat_interleave(32, 1)[:, :cols], 0.0, code).to(torch.uint8)
    return code | (sign & (code > 0)).to(torch.uint8) << 3, torch.where(bad, 255, exponent + 127).to(torch.uint8)


def _plain_pack(codes):
    codes = torch.nn.functional.pad(codes, (0, codes.shape[1] % 2))
    return codes[:, ::2] | codes[:, 1::2] << 4


def _plain_values(codes, exponents):
    """What codes, one to a byte, and scales stand for."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    scales = torch.where(exponents == 255, math.nan, torch.ldexp(torch.ones((), device=codes.device), exponents.int() - 127))
    return table[codes.int()] * scales.repeat_interleave(32, 1)[:, :codes.shape[1]]


def _plain_unpack(codes, cols):
    return torch.stack([codes & 15, codes >> 4], 2).flatten(1)[:, :cols]


def _plain_clip(grads, outs, scale, most):
    total = torch.stack([x.float().square().sum(dtype=torch.float64) for x in grads]).sum()
    norm = (total.sqrt() * scale).float()
    if outs is not None:
        factor = torch.where(norm <= most, 1.0, most / norm) * scale
        for x, out in zip(grads, outs):
            out.copy_(x.float() * factor)
    return norm.reshape(1)


def _run_plain(s):
    c, kind = s["c"], s["c"]["kind"]
    if kind == "roundtrip":
        dtype = _TYPES[c["out"]]
        values = _plain_values(*_plain_quantise(s["x"], c["block"], c["fit"])).to(dtype)
        if not c["both"]:
            return values
        return values, _plain_values(*_plain_quantise(s["x"].t(), c["block"], c["fit"])).to(dtype)
    if kind == "product":
        K = c["K"]
        x = _plain_values(_plain_unpack(s["a"], K), s["a_scales"]) if c["held"] else _plain_values(*_plain_quantise(s["a"], 1, c["fit"]))
        return (x @ _plain_values(_plain_unpack(s["w"], K), s["w_scales"]).t()).to(_TYPES[c["out"]])
    if kind in ("norm", "clip"):
        norm = _plain_clip(s["grads"], s["outs"], s["scale"], 1.0)
        return norm if kind == "norm" else (norm, s["out"])
    values = lambda x, block: _plain_values(*_plain_quantise(x, block, c["fit"]))  # noqa: E731
    w = values(s["w"], 32)
    y = values(s["x"], 1) @ w.t()
    dx = values(s["g"], 1) @ w
    dw = values(s["g"].t(), 1) @ values(s["x"].t(), 1).t()
    norm = _plain_clip([dw], [dw], 1.0, 1.0)
    return y.bfloat16(), dx.bfloat16(), dw, norm


# ---- the framework's calls

def _run_own(s):
    from paper_1912_08756_amd import binding as icq
    c, kind = s["c"], s["c"]["kind"]
    if kind == "roundtrip":
        if not c["both"]:
            icq.icq_mx_quantize(s["x"], s["codes"], s["scales"], block_rows=c["block"], fit=c["fit"])
            return icq.icq_mx_dequantize(s["codes"], s["scales"], s["out"])
        icq.icq_mx_quantize(s["x"], s["codes"], s["scales"], s["codes_t"], s["scales_t"], block_rows=c["block"], fit=c["fit"])
        return icq.icq_mx_dequantize(s["codes"], s["scales"], s["out"]), icq.icq_mx_dequantize(s["codes_t"], s["scales_t"], s["out_t"])
    if kind == "product":
        return icq.icq_mx_matmul(s["a"], s["a_scales"], s["w"], s["w_scales"], s["out"], s["workspace"], K=c["K"], fit=c["fit"])
    if kind == "norm":
        return icq.icq_grad_norm(s["list"], s["norm"], s["workspace"], scale=s["scale"])
    if kind == "clip":
        icq.icq_grad_norm_clip(s["list"], s["norm"], 1.0, s["workspace"], scale=s["scale"])
        return s["norm"], s["out"]
    fit, N, K, T, ws = c["fit"], c["N"], c["K"], c["T"], s["workspace"]
    for name in ("x", "w", "g"):
        icq.icq_mx_quantize(s[name], s[name + "_codes"], s[name + "_scales"], s[name + "_codes_t"], s[name + "_scales_t"],
                            block_rows=32 if name == "w" else 1, fit=fit)
    icq.icq_mx_matmul(s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["y"], ws, K=K)
    icq.icq_mx_matmul(s["g_codes"], s["g_scales"], s["w_codes_t"], s["w_scales_t"], s["dx"], ws, K=N)
    icq.icq_mx_matmul(s["g_codes_t"], s["g_scales_t"], s["x_codes_t"], s["x_scales_t"], s["dw"], ws, K=T)
    icq.icq_grad_norm_clip(s["list"], s["norm"], 1.0, ws)
    return s["y"], s["dx"], s["dw"], s["norm"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the least that a pass reads, writes and computes

_PER = 0.5 + 1 / 32         # bytes a value held in 4 bits


def work(case):
    c = case
    kind = c["kind"]
    if kind == "roundtrip":
        n, ways = c["rows"] * c["cols"], 2 if c["both"] else 1
        return dict(bytes=n * (_SIZE[c["type"]] + ways * (_PER + _SIZE[c["out"]])), flops=4.0 * n * ways)
    if kind == "product":
        M, N, K = c["M"], c["N"], c["K"]
        return dict(bytes=M * K * (_PER if c["held"] else _SIZE[c["type"]]) + N * K * _PER + M * N * _SIZE[c["out"]], flops=2.0 * M * N * K)
    if kind in ("norm", "clip"):
        n = sum(_numbers(c))
        return dict(bytes=n * (_SIZE[c["type"]] + (_SIZE[c["out"]] if kind == "clip" else 0)) + 4, flops=(3.0 if kind == "clip" else 2.0) * n)
    T, N, K = c["T"], c["N"], c["K"]
    return dict(bytes=T * K * 4 + N * K * 8 + T * N * 4, flops=6.0 * T * N * K)


# ---- the definitions in 64 bits

def _exact_values(x, block, fit):
    """What the blocks of a matrix become: exponents by counting powers of two, values by the places between which they lie."""
    rows, cols = x.shape
    full = torch.zeros((-(-rows // block) * block, -(-cols // 32) * 32), dtype=torch.float64, device=x.device)
    full[:rows, :cols] = x.double()
    tiles = full.reshape(-1, block, full.shape[1] // 32, 32)
    amax = tiles.abs().amax(3).amax(1)
    used = torch.nan_to_num(amax, nan=1.0, posinf=1.0).clamp(min=_SMALLEST_AMAX)
    e = torch.floor(torch.log2(used))
    e = e - (torch.exp2(e) > used).double() + (torch.exp2(e + 1) <= used).double() - 2
    if fit:
        e = (e + (used > 6 * torch.exp2(e)).double()).clamp(max=_MOST_EXPONENT)
    scale = torch.exp2(e)[:, None, :, None]
    size = tiles.abs() / scale
    grid = (0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
    value, last = torch.zeros_like(size), 0.0
    for k, v in enumerate(grid):        # a tie goes to the code of even number: down to the first, third, ... neighbour, up to the second, ...
        middle = (v + last) / 2
        value = torch.where(size >= middle if k % 2 else size > middle, v, value)
        last = v
    value = torch.where(torch.isfinite(amax)[:, None, :, None], torch.copysign(value, tiles) * scale, math.nan)
    return value.reshape(full.shape)[:rows, :cols]


def _exact_held(codes, scales, cols):
    """What a held matrix stands for: sign, exponent and mantissa of each half byte."""
    out = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    for h in (0, 1):
        n = (codes.long() >> 4 * h) % 16
        e, m = n % 8 // 2, (n % 2).double()
        out[:, h::2] = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e.double() - 1)) * torch.where(n >= 8, -1.0, 1.0)
    for k in range(scales.shape[1]):
        out[:, 32 * k:32 * k + 32] *= torch.where(scales[:, k:k + 1] == 255, math.nan, torch.exp2(scales[:, k:k + 1].double() - 127))
    return out[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = s["c"], case["kind"]
    if kind == "roundtrip":
        values = _exact_values(s["x"], c["block"], c["fit"])
        return (values, _exact_values(s["x"].t(), c["block"], c["fit"])) if c["both"] else values
    if kind == "product":
        x = _exact_held(s["a"], s["a_scales"], c["K"]) if c["held"] else _exact_values(s["a"], 1, c["fit"])
        parts = [x @ _exact_held(s["w"][at:at + 65536], s["w_scales"][at:at + 65536], c["K"]).t().contiguous() for at in range(0, c["N"], 65536)]
        return torch.cat(parts, 1)
    if kind in ("norm", "clip"):
        whole = torch.cat([x.double() for x in s["grads"]]) * s["scale"]
        norm = torch.linalg.vector_norm(whole)
        return norm.reshape(1) if kind == "norm" else (norm.reshape(1), whole / torch.clamp(norm, min=1.0))
    x, w, g = _exact_values(s["x"], 1, c["fit"]), _exact_values(s["w"], 32, c["fit"]), _exact_values(s["g"], 1, c["fit"])
    gt, xt = _exact_values(s["g"].t(), 1, c["fit"]), _exact_values(s["x"].t(), 1, c["fit"])
    dw = gt @ xt.t()
    norm = torch.linalg.vector_norm(dw)
    return x @ w.t(), g @ w, dw / torch.clamp(norm, min=1.0), norm.reshape(1)
