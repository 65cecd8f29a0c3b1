"""What the performance of the training-side operators is measured on: 8-bit products with a scale per block
of 128, and the distillation of a scoring head from the lists that a search returns.

A program that uses them has a scoring head W [V][F] over V items (or codewords) and features X [R][F]:
it quantises X and W in blocks, forms the logits X W^T as an 8-bit product, takes the loss of those logits
against the neighbour lists of its index (ids and distances, short lists padded), and goes back through
the same product for the gradients of X and W.  Feature lengths are this repository's query dimensions (96,
128, 960) or generic powers of two; vocabularies are its database sizes (10^4, 10^6 items), its codebooks'
(16 * 256 codewords) or generic; list lengths are its result lists'.

Kinds of case:
  quantise   values [rows][cols] -> codes and scales, blocks of 1 x 128 or 128 x 128, as rows or as rows and columns
  product    X [M][K] quantised in the call, W [N][K] held quantised with 128 x 128 blocks -> X W^T [M][N]
  gradient   G [T][M] and X [T][N] quantised by columns in the call -> G^T X [M][N], blocks of 1 x 128 on both sides
  distill    logits [R][V] and lists [R][topk] -> loss and gradient
  step       all of it: logits, loss, gradients of features and weights
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
_SMALLEST_AMAX = 2.0 ** -100
_PAD = 0xFFFFFFFF


def listed():
    return [
        # a service's batch of 100 queries, the longest query dimension here: launch latency
        dict(name="quantise_queries", kind="quantise", rows=100, cols=960, type="bf16", format="e4m3", block=1, pow2=False, both=False),
        # the logits' gradient of a batch, needed by rows for the features' gradient and by columns for the weights'
        dict(name="quantise_gradient", kind="quantise", rows=8192, cols=16000, type="bf16", format="e5m2", block=1, pow2=True, both=True),
        # the weights after an update in 32 bits, both orientations
        dict(name="quantise_weights", kind="quantise", rows=10007, cols=4096, type="f32", format="e4m3", block=128, pow2=False, both=True),
        # one query scored against all items: reading the weights is all there is
        dict(name="product_single", kind="product", M=1, N=16384, K=4096, type="bf16", out="bf16", pow2=False),
        # nothing is a round number
        dict(name="product_ragged", kind="product", M=333, N=5003, K=1000, type="f16", out="f32", pow2=False),
        # a training batch against a wide head
        dict(name="product_large", kind="product", M=8192, N=8192, K=8192, type="bf16", out="bf16", pow2=True),
        # the weights' gradient, summed over 4096 rows of a batch
        dict(name="gradient_weights", kind="gradient", T=4096, M=10000, N=960, type="bf16", out="f32", pow2=False),
        # the tiny workload: 100 queries, 10^4 items, lists of 10
        dict(name="distill_tiny", kind="distill", R=100, V=10_000, topk=10, type="f32", rest=False, apart=False, pad=0),
        # a training batch over a large vocabulary of items
        dict(name="distill_batch", kind="distill", R=4096, V=131_072, topk=100, type="bf16", rest=False, apart=False, pad=0),
        # a handful of queries against every item of a database of a million, with the mass off the list
        dict(name="distill_items", kind="distill", R=8, V=1_000_000, topk=100, type="f32", rest=True, apart=False, pad=0),
        # odd sizes, rows in a wider buffer, loss and gradient as two calls
        dict(name="distill_ragged", kind="distill", R=777, V=50_021, topk=47, type="f16", rest=True, apart=True, pad=7),
        # a whole step of a head over 16384 items from features of 960 dimensions
        dict(name="step", kind="step", R=2048, V=16384, F=960, topk=20, pow2=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo + 1, hi))))))


def draw(rng):
    """One more case of the same kinds, sizes spread between a single row and the largest listed ones."""
    what = rng.choice(["quantise", "quantise", "product", "product", "product", "gradient", "distill", "distill", "distill", "step"])
    half = rng.random() < 0.5
    if what == "quantise":
        rows = _log(rng, 1, 16384)
        return dict(kind="quantise", rows=rows, cols=_log(rng, 32, min(32768, 1.3e8 / rows)), type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    format=rng.choice(["e4m3", "e4m3", "e5m2"]), block=rng.choice([1, 1, 128]), pow2=half, both=rng.random() < 0.5)
    if what == "product":
        M, K = _log(rng, 1, 8192), _log(rng, 96, 8192)
        return dict(kind="product", M=M, N=_log(rng, 256, min(32768, 5.0e11 / M / K)), K=K, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    out=rng.choice(["bf16", "bf16", "f32", "f16"]), pow2=half)
    if what == "gradient":
        T, N = _log(rng, 32, 8192), _log(rng, 96, 4096)
        return dict(kind="gradient", T=T, M=_log(rng, 256, min(16384, 2.0e11 / T / N)), N=N, type=rng.choice(["bf16", "f16"]),
                    out=rng.choice(["f32", "f32", "bf16"]), pow2=half)
    if what == "distill":
        V = _log(rng, 1000, 1_000_000)
        return dict(kind="distill", R=_log(rng, 1, min(8192, 3.0e8 / V)), V=V, topk=rng.choice([1, 10, 20, 50, 100, rng.randint(1, 500)]),
                    type=rng.choice(["bf16", "bf16", "f16", "f32"]), rest=half, apart=rng.random() < 0.3, pad=rng.choice([0, 0, 0, rng.randint(1, 40)]))
    R, F = _log(rng, 16, 4096), rng.choice([96, 128, 960, _log(rng, 64, 4096)])
    return dict(kind="step", R=R, V=_log(rng, 1000, min(32768, 1.0e11 / R / F)), F=F, topk=rng.choice([10, 20, 100]), pow2=half)


# ---- inputs

def _blocks(n):
    return (n + 127) // 128


def _up16(n):
    return (n + 15) // 16 * 16


def _codes_like(rows, cols, dtype):
    """A code buffer: rows of `cols` codes, each row starting on 16 bytes."""
    return torch.zeros((rows, _up16(cols)), dtype=torch.uint8, device="cuda").view(dtype)[:, :cols]


def _outliers(x, g):
    """Activations have a few channels that are much larger than the rest."""
    big = torch.rand((x.shape[1],), device="cuda", generator=g) < 0.01
    x[:, big] *= 20.0
    return x


def _gaussian(rows, cols, dtype, g, scale=1.0):
    return _outliers(torch.randn((rows, cols), device="cuda", generator=g).mul_(scale), g).to(dtype)


def _lists(R, V, topk, g):
    """Lists of distinct ids with ascending distances, as a search returns them: about one in eight is short, the last row's is empty
    where there are several rows."""
    topk = min(topk, V)
    step = V // topk
    ids = torch.arange(topk, device="cuda") * step + torch.randint(0, step, (R, topk), device="cuda", generator=g)
    ids = ids.gather(1, torch.rand((R, topk), device="cuda", generator=g).argsort(1))
    dist = 4.0 + 6.0 * torch.rand((R, topk), device="cuda", generator=g).sort(1).values
    length = torch.where(torch.rand((R,), device="cuda", generator=g) < 0.125,
                         torch.randint(1, topk + 1, (R,), device="cuda", generator=g), topk)
    if R > 1:
        length[-1] = 0
    short = torch.arange(topk, device="cuda")[None, :] >= length[:, None]
    dist = dist.masked_fill(short, math.inf)
    return ids.masked_fill(short, _PAD), dist


def _as_u32(ids):
    return torch.where(ids > 0x7FFFFFFF, ids - (1 << 32), ids).to(torch.int32)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = c["kind"]
    s = dict(c=c)
    if kind == "quantise":
        rows, cols, f = c["rows"], c["cols"], _FORMATS[c["format"]]
        s["x"] = _gaussian(rows, cols, _TYPES[c["type"]], g, 0.02 if c["block"] == 128 else 1.0)
        R, C = (_blocks(rows), _blocks(cols)) if c["block"] == 128 else (rows, cols)
        s["codes"], s["scales"] = _codes_like(rows, cols, f), torch.empty((R, _blocks(cols)), device="cuda")
        if c["both"]:
            s["codes_t"], s["scales_t"] = _codes_like(cols, rows, f), torch.empty((C, _blocks(rows)), device="cuda")
    elif kind == "product":
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = _gaussian(M, K, _TYPES[c["type"]], g)
        codes, s["w_scales"] = _plain_quantise(torch.randn((N, K), device="cuda", generator=g).mul_(0.02), "e4m3", 128, c["pow2"])
        s["w"] = _codes_like(N, K, torch.float8_e4m3fn)
        s["w"].copy_(codes)
        s["x_codes"], s["x_scales"] = _codes_like(M, K, torch.float8_e4m3fn), torch.empty((M, _blocks(K)), device="cuda")
        s["out"] = torch.empty((M, N), dtype=_TYPES[c["out"]], device="cuda")
    elif kind == "gradient":
        T, M, N = c["T"], c["M"], c["N"]
        s["g"] = (torch.randn((T, M), device="cuda", generator=g) * torch.rand((T, 1), device="cuda", generator=g).mul_(1e-3)).to(_TYPES[c["type"]])
        s["x"] = _gaussian(T, N, _TYPES[c["type"]], g)
        s["g_codes"], s["g_scales"] = _codes_like(M, T, torch.float8_e5m2), torch.empty((M, _blocks(T)), device="cuda")
        s["x_codes"], s["x_scales"] = _codes_like(N, T, torch.float8_e4m3fn), torch.empty((N, _blocks(T)), device="cuda")
        s["out"] = torch.empty((M, N), dtype=_TYPES[c["out"]], device="cuda")
    elif kind == "distill":
        R, V = c["R"], c["V"]
        ids, s["dist"] = _lists(R, V, c["topk"], g)
        s["ids"] = _as_u32(ids)
        wide = torch.randn((R, V + c["pad"]), device="cuda", generator=g).mul_(2.0)
        # a student on its way: the listed items stand out, the nearer the more
        lift = torch.where(ids == _PAD, 0.0, 12.0 - s["dist"]) + torch.randn(ids.shape, device="cuda", generator=g)
        wide.scatter_add_(1, ids.clamp(max=V - 1), torch.where(ids == _PAD, 0.0, lift))
        s["logits"] = wide.to(_TYPES[c["type"]])[:, :V]
        s["grad"] = torch.empty((R, V + c["pad"]), dtype=_TYPES[c["type"]], device="cuda")[:, :V]
        s["scale"], s["teacher_scale"] = 0.5, -1.25
        s["lse"] = None
        if c["rest"]:       # the teacher holds 70 to 98 % of its mass in the list
            z = torch.where(ids == _PAD, -math.inf, s["dist"] * s["teacher_scale"])
            s["lse"] = torch.nan_to_num(torch.logsumexp(z, 1), neginf=0.0) - torch.log(0.7 + 0.28 * torch.rand((R,), device="cuda", generator=g))
        # gradients held in 16 bits with five of exponent come with a loss scale
        s["grad_loss"] = torch.rand((R,), device="cuda", generator=g).mul_(10.0 if c["type"] == "f16" else 0.01)
        s["loss"], s["stats"] = torch.empty((R,), device="cuda"), torch.empty((R, 4), device="cuda")
    else:
        R, V, F, pow2 = c["R"], c["V"], c["F"], c["pow2"]
        s["x"] = _gaussian(R, F, torch.bfloat16, g)
        codes, s["w_scales"] = _plain_quantise(torch.randn((V, F), device="cuda", generator=g).mul_(0.06), "e4m3", 128, pow2)
        s["w"], s["w_t"] = _codes_like(V, F, torch.float8_e4m3fn), _codes_like(F, V, torch.float8_e4m3fn)
        s["w"].copy_(codes)
        s["w_t"].copy_(codes.float().t().to(torch.float8_e4m3fn))
        s["w_scales_t"] = s["w_scales"].t().contiguous()
        ids, s["dist"] = _lists(R, V, c["topk"], g)
        s["ids"] = _as_u32(ids)
        s["teacher_scale"] = -1.25
        s["grad_loss"] = torch.full((R,), 1.0, device="cuda")
        e4, e5 = torch.float8_e4m3fn, torch.float8_e5m2
        s["x_codes"], s["x_scales"] = _codes_like(R, F, e4), torch.empty((R, _blocks(F)), device="cuda")
        s["xt_codes"], s["xt_scales"] = _codes_like(F, R, e4), torch.empty((F, _blocks(R)), device="cuda")
        s["g_codes"], s["g_scales"] = _codes_like(R, V, e5), torch.empty((R, _blocks(V)), device="cuda")
        s["gt_codes"], s["gt_scales"] = _codes_like(V, R, e5), torch.empty((V, _blocks(R)), device="cuda")
        s["logits"], s["grad"] = torch.empty((R, V), device="cuda"), torch.empty((R, V), device="cuda")
        s["loss"] = torch.empty((R,), device="cuda")
        s["dx"], s["dw"] = torch.empty((R, F), dtype=torch.bfloat16, device="cuda"), torch.empty((V, F), dtype=torch.bfloat16, device="cuda")
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms

def _plain_scale(amax, form, pow2):
    amax = amax.clamp(min=_SMALLEST_AMAX)
    if not pow2:
        return amax / torch.full_like(amax, _LARGEST[form])     # (a plain number as divisor becomes a product with its rounded reciprocal)
    mantissa, exponent = torch.frexp(amax)      # amax = mantissa * 2^exponent, mantissa in [0.5, 1); the formats' largest: 0.875 * 2^9, 0.875 * 2^16
    return torch.ldexp(torch.ones_like(amax), exponent - (9 if form == "e4m3" else 16) + (mantissa > 0.875).int())


def _spread(scales, rows, cols, block):
    """Scales of 1 x 128 or 128 x 128 blocks, one per value."""
    x = scales.repeat_interleave(128, 1)[:, :cols]
    return x.repeat_interleave(128, 0)[:rows] if block == 128 else x


def _plain_quantise(x, form, block, pow2):
    """(codes, scales) of the blocks of a matrix."""
    rows, cols = x.shape
    x = x.float()
    size = torch.nn.functional.pad(torch.where(torch.isfinite(x), x.abs(), 0.0), (0, -cols % 128, 0, -rows % block))
    amax = size.view(size.shape[0] // block, block, size.shape[1] // 128, 128).amax((1, 3))
    scales = _plain_scale(amax, form, pow2)
    return (x * _spread(1.0 / scales, rows, cols, block)).to(_FORMATS[form]), scales


def _plain_product(a, a_scales, b, b_scales, b_block):
    x = a.float() * _spread(a_scales, *a.shape, 1)
    y = b.float() * _spread(b_scales, *b.shape, b_block)
    return x @ y.t()


def _plain_distill(logits, ids, dist, scale, teacher_scale, lse, grad_loss):
    R, V = logits.shape
    s = logits.float() * scale
    top = s.amax(1, keepdim=True)
    e = torch.exp(s - top)
    total = e.sum(1, keepdim=True)
    on = (ids >= 0) & (ids < V)
    at = torch.where(on, ids, 0).long()
    z = torch.where(on, dist * teacher_scale, -math.inf)
    if lse is None:
        z_top = z.amax(1, keepdim=True)
        z_top = torch.where(torch.isfinite(z_top), z_top, 0.0)
        teacher = z_top + torch.log(torch.exp(z - z_top).sum(1, keepdim=True))
    else:
        teacher = lse[:, None]
    log_p = torch.where(on, z - teacher, 0.0)
    p = torch.where(on, torch.exp(log_p), 0.0)
    log_q = s.gather(1, at) - top - torch.log(total)
    loss = (p * (log_p - log_q)).sum(1)
    c = torch.ones_like(total)
    if lse is not None:
        listed_at = torch.zeros((R, V + 1), dtype=torch.bool, device=s.device).scatter_(1, torch.where(on, at, V), True)[:, :V]
        q_rest = torch.where(listed_at, 0.0, e).sum(1, keepdim=True) / total
        p_rest = (1.0 - p.sum(1, keepdim=True)).clamp(min=0.0)
        some = p_rest > 0
        loss = loss + torch.where(some, p_rest * (torch.log(torch.where(some, p_rest, 1.0)) - torch.log(q_rest)), 0.0)[:, 0]
        c = 1.0 - p_rest / q_rest
    has = on.any(1)
    q = e / total
    grad = q * c
    listed_grad = q.gather(1, at) - p
    grad = torch.cat([grad, grad[:, :1]], 1).scatter_(1, torch.where(on, at, V), listed_grad)[:, :V]
    grad = grad * (scale * grad_loss * has)[:, None]
    return torch.where(has, loss, 0.0), grad


def _run_plain(s):
    c, kind = s["c"], s["c"]["kind"]
    if kind == "quantise":
        codes, scales = _plain_quantise(s["x"], c["format"], c["block"], c["pow2"])
        if not c["both"]:
            return codes, scales
        codes_t, scales_t = _plain_quantise(s["x"].t(), c["format"], c["block"], c["pow2"])
        return codes, scales, codes_t, scales_t
    if kind == "product":
        return _plain_product(*_plain_quantise(s["x"], "e4m3", 1, c["pow2"]), s["w"], s["w_scales"], 128).to(_TYPES[c["out"]])
    if kind == "gradient":
        a, b = _plain_quantise(s["g"].t(), "e5m2", 1, c["pow2"]), _plain_quantise(s["x"].t(), "e4m3", 1, c["pow2"])
        return _plain_product(*a, *b, 1).to(_TYPES[c["out"]])
    if kind == "distill":
        loss, grad = _plain_distill(s["logits"], s["ids"], s["dist"], s["scale"], s["teacher_scale"], s["lse"], s["grad_loss"])
        return loss, grad.to(s["logits"].dtype)
    logits = _plain_product(*_plain_quantise(s["x"], "e4m3", 1, c["pow2"]), s["w"], s["w_scales"], 128)
    loss, grad = _plain_distill(logits, s["ids"], s["dist"], 1.0, s["teacher_scale"], None, s["grad_loss"])
    dx = _plain_product(*_plain_quantise(grad, "e5m2", 1, c["pow2"]), s["w_t"], s["w_scales_t"], 128)
    dw = _plain_product(*_plain_quantise(grad.t(), "e5m2", 1, c["pow2"]), *_plain_quantise(s["x"].t(), "e4m3", 1, c["pow2"]), 1)
    return logits, loss, dx.bfloat16(), dw.bfloat16()


# ---- the framework's calls

def _run_own(s):
    from paper_1912_08756_amd import binding as icq
    c, kind = s["c"], s["c"]["kind"]
    if kind == "quantise":
        if not c["both"]:
            icq.icq_block_quantize(s["x"], s["codes"], s["scales"], block_rows=c["block"], pow2=c["pow2"])
            return s["codes"], s["scales"]
        icq.icq_block_quantize(s["x"], s["codes"], s["scales"], s["codes_t"], s["scales_t"], block_rows=c["block"], pow2=c["pow2"])
        return s["codes"], s["scales"], s["codes_t"], s["scales_t"]
    if kind == "product":
        icq.icq_block_quantize(s["x"], s["x_codes"], s["x_scales"], pow2=c["pow2"])
        icq.icq_block_matmul(s["x_codes"], s["x_scales"], s["w"], s["w_scales"], s["out"], s["workspace"], pow2=c["pow2"])
        return s["out"]
    if kind == "gradient":
        icq.icq_block_quantize(s["g"], None, None, s["g_codes"], s["g_scales"], pow2=c["pow2"])
        icq.icq_block_quantize(s["x"], None, None, s["x_codes"], s["x_scales"], pow2=c["pow2"])
        icq.icq_block_matmul(s["g_codes"], s["g_scales"], s["x_codes"], s["x_scales"], s["out"], s["workspace"], pow2=c["pow2"])
        return s["out"]
    if kind == "distill":
        lists = (s["ids"], s["dist"], s["scale"], s["teacher_scale"], s["lse"])
        if c["apart"]:
            icq.icq_distill(s["logits"], *lists, s["loss"], s["stats"], workspace=s["workspace"])
            icq.icq_distill_backward(s["logits"], *lists, s["stats"], s["grad_loss"], s["grad"])
        else:
            icq.icq_distill(s["logits"], *lists, s["loss"], grad_loss=s["grad_loss"], grad=s["grad"], workspace=s["workspace"])
        return s["loss"], s["grad"]
    pow2 = c["pow2"]
    icq.icq_block_quantize(s["x"], s["x_codes"], s["x_scales"], s["xt_codes"], s["xt_scales"], pow2=pow2)
    icq.icq_block_matmul(s["x_codes"], s["x_scales"], s["w"], s["w_scales"], s["logits"], s["workspace"], pow2=pow2)
    icq.icq_distill(s["logits"], s["ids"], s["dist"], 1.0, s["teacher_scale"], None, s["loss"], grad_loss=s["grad_loss"], grad=s["grad"],
                    workspace=s["workspace"])
    icq.icq_block_quantize(s["grad"], s["g_codes"], s["g_scales"], s["gt_codes"], s["gt_scales"], pow2=pow2)
    icq.icq_block_matmul(s["g_codes"], s["g_scales"], s["w_t"], s["w_scales_t"], s["dx"], s["workspace"], pow2=pow2)
    icq.icq_block_matmul(s["gt_codes"], s["gt_scales"], s["xt_codes"], s["xt_scales"], s["dw"], s["workspace"], pow2=pow2)
    return s["logits"], s["loss"], s["dx"], s["dw"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the least that a pass reads, writes and computes

def work(case):
    c, size = case, {"f32": 4, "f16": 2, "bf16": 2}
    kind = c["kind"]
    if kind == "quantise":
        n, b = c["rows"] * c["cols"], 128 * c["block"]
        return dict(bytes=n * (size[c["type"]] + (2 if c["both"] else 1)) + (8 if c["both"] else 4) * n / b, flops=4 * n)
    if kind == "product":
        M, N, K = c["M"], c["N"], c["K"]
        return dict(bytes=M * K * size[c["type"]] + N * K * (1 + 4 / 16384) + M * N * size[c["out"]], flops=2.0 * M * N * K)
    if kind == "gradient":
        T, M, N = c["T"], c["M"], c["N"]
        return dict(bytes=T * (M + N) * size[c["type"]] + M * N * size[c["out"]], flops=2.0 * M * N * T)
    if kind == "distill":
        n = c["R"] * c["V"]
        return dict(bytes=2 * n * size[c["type"]] + c["R"] * (8 * c["topk"] + 12), flops=10.0 * n)
    R, V, F = c["R"], c["V"], c["F"]
    return dict(bytes=4 * R * F + 4 * V * F + 4 * R * V + 8 * R * c["topk"], flops=6.0 * R * V * F)


# ---- the definitions in 64 bits

def _exact_codes(x, form, block, pow2):
    """Values that the codes of x stand for, without and with their scales, and the scales.  The definition fixes the roundings to 32 bits: of
    amax / largest, of the scale's reciprocal and of the value times that."""
    rows, cols = x.shape
    across, down = -(-cols // 128), -(-rows // block)
    full = torch.zeros((down * block, across * 128), dtype=torch.float64, device=x.device)
    full[:rows, :cols] = x.double()
    tiles = full.reshape(down, block, across, 128)
    amax = torch.nan_to_num(tiles, nan=0.0, posinf=0.0, neginf=0.0).abs().amax(3).amax(1).clamp(min=_SMALLEST_AMAX)
    if pow2:
        scales = torch.exp2(torch.ceil(torch.log2(amax / _LARGEST[form])))
        scales = torch.where(amax / scales > _LARGEST[form], scales * 2, scales)
        scales = torch.where(amax / scales * 2 <= _LARGEST[form], scales / 2, scales)
    else:
        scales = (amax / _LARGEST[form]).float().double()
    inverse = (1.0 / scales).float().double()
    units = (tiles * inverse[:, None, :, None]).float()
    values = units.to(_FORMATS[form]).double()
    whole = lambda t: t.reshape(down * block, across * 128)[:rows, :cols]  # noqa: E731
    return whole(values), whole(values * scales[:, None, :, None]), scales


def _exact_head(codes, scales):
    """What weights held in 128 x 128 blocks stand for."""
    w = codes.double()
    for k in range(scales.shape[1]):
        w[:, 128 * k:128 * k + 128] *= scales[:, k].double().repeat_interleave(128)[:w.shape[0], None]
    return w


def _exact_distill(logits, ids, dist, scale, teacher_scale, lse, grad_loss):
    R, V = logits.shape
    log_q = torch.log_softmax(logits.double() * scale, 1)
    on = (ids >= 0) & (ids < V)
    z = torch.where(on, dist.double() * teacher_scale, -math.inf)
    p = torch.exp(z - (lse.double()[:, None] if lse is not None else torch.logsumexp(z, 1, keepdim=True)))
    p = torch.where(on, p, 0.0)
    at = torch.where(on, ids, 0).long()
    loss = (torch.xlogy(p, p) - torch.where(p > 0, p * log_q.gather(1, at), 0.0)).sum(1)
    off = log_q.exp()
    target = torch.zeros_like(off).scatter_add_(1, at, p)
    if lse is not None:
        off.scatter_(1, torch.where(on, at, 0), torch.where(on, 0.0, off.gather(1, at)))       # the first place is only marked where it is listed
        first = (on & (ids == 0)).any(1)
        off[:, 0] = torch.where(first, 0.0, log_q[:, 0].exp())
        p_rest = (1 - p.sum(1)).clamp(min=0)
        q_rest = off.sum(1)
        loss = loss + torch.xlogy(p_rest, p_rest) - torch.xlogy(p_rest, q_rest)
        target += off * (p_rest / q_rest)[:, None]
    has = on.any(1)
    grad = (log_q.exp() - target) * (grad_loss.double() * scale * has)[:, None]
    return torch.where(has, loss, 0.0), grad


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = s["c"], case["kind"]
    if kind == "quantise":
        codes, _, scales = _exact_codes(s["x"], c["format"], c["block"], c["pow2"])
        if not c["both"]:
            return codes, scales
        codes_t, _, scales_t = _exact_codes(s["x"].t(), c["format"], c["block"], c["pow2"])
        return codes, scales, codes_t, scales_t
    if kind == "product":
        return _exact_codes(s["x"], "e4m3", 1, c["pow2"])[1] @ _exact_head(s["w"], s["w_scales"]).t()
    if kind == "gradient":
        return _exact_codes(s["g"].t(), "e5m2", 1, c["pow2"])[1] @ _exact_codes(s["x"].t(), "e4m3", 1, c["pow2"])[1].t()
    if kind == "distill":
        return _exact_distill(s["logits"], s["ids"], s["dist"], s["scale"], s["teacher_scale"], s["lse"], s["grad_loss"])
    w = _exact_head(s["w"], s["w_scales"])
    logits = _exact_codes(s["x"], "e4m3", 1, c["pow2"])[1] @ w.t()
    loss, grad = _exact_distill(logits, s["ids"], s["dist"], 1.0, s["teacher_scale"], None, s["grad_loss"])
    dx = _exact_codes(grad, "e5m2", 1, c["pow2"])[1] @ w
    dw = _exact_codes(grad.t(), "e5m2", 1, c["pow2"])[1] @ _exact_codes(s["x"].t(), "e4m3", 1, c["pow2"])[1].t()
    return logits, loss, dx, dw
