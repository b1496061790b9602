"""The operators of a layer and its loss whose speed matters to a program that trains with this library: how to make, run
and check them.

  norm        mv_layernorm_forward    a layer norm, with the mean and reciprocal deviation that its backward pass takes
  norm_grad   mv_layernorm_backward   the gradients of its input, weight and bias
  linear8     mv_f8_linear            a layer's product with weights held in 8-bit floating point
  grad8       mv_f8_linear_grad       both gradients of that product
  distill     mv_distill_loss         distillation from a teacher's top logits, with or without a label's cross entropy: the
                                      loss of every row, alone or with the gradient of the logits
  distill_grad  mv_distill_grad       that gradient, from what a call for the loss alone kept

8-bit values: 128 consecutive values share a power of two 2^s, s the smallest whole number for which the largest magnitude
is at most 448 * 2^s, and at least -127, held as the byte s + 127; each value is the nearest of 4 exponent and 3 fraction
bits (1 + f / 8) 2^e, e from -6 to 8, or f / 8 * 2^-6, at most 448, ties to the even f, times 2^s.  Rows are whole blocks.

Distillation: p = softmax(t / T) over a row's list of the teacher's top logits, q = softmax(z / T) and s = softmax(z) over all of
the student's; loss = soft T^2 sum p (log p - log q) + hard (-log s[label]).  An entry whose index is not a coordinate is
not in the list, a label that is not one takes its term away.  A row's statistics: its largest logit m, sum exp((z - m) / T)
and sum exp(z - m), a sum that no term needs as 0.

Sizes are those of this repository's layers and examples, and generic ones.
"""
import math

import torch

own = False                    # True: the library's operators; False: the same in plain torch

NORM_MOST = 134_000_000        # values of a drawn layer norm
PRODUCT_MOST = 270_000_000_000 # m n k of a drawn product: below the largest listed one
LOGITS_MOST = 530_000_000      # of a drawn distillation


def listed():
    return [
        # A batch of the example's inputs before its first layer: a launch is the whole cost.
        {"name": "norm_small", "op": "norm", "rows": 96, "n": 200, "src": "f32", "dst": "f32", "weights": "f32"},
        # A long batch of wide activations.
        {"name": "norm_large", "op": "norm", "rows": 16_384, "n": 8192, "src": "bf16", "dst": "bf16", "weights": "f32"},
        # Backward over a short batch of an odd width: the weight's gradient is a reduction of its own.
        {"name": "norm_grad_odd", "op": "norm_grad", "rows": 1000, "n": 2047, "src": "f32", "dst": "f32", "weights": "f32"},
        # Backward over a long batch.
        {"name": "norm_grad_large", "op": "norm_grad", "rows": 16_384, "n": 4096, "src": "bf16", "dst": "bf16", "weights": "bf16"},
        # One image or token through ResNet-50's classifier.
        {"name": "linear8_one", "op": "linear8", "m": 1, "n": 1000, "k": 2048, "src": "f32", "dst": "f32"},
        # A few at once through a large layer: reading its weights is the cost.
        {"name": "linear8_few", "op": "linear8", "m": 5, "n": 16_384, "k": 8192, "src": "bf16", "dst": "bf16"},
        # A long batch through a large layer.
        {"name": "linear8_large", "op": "linear8", "m": 4096, "n": 8192, "k": 8192, "src": "bf16", "dst": "bf16"},
        # The backward pass of a 3x3 layer of ResNet-50 (512 to 512 channels at 7 x 7) as a product over a batch of 100.
        {"name": "grad8_r50_3x3", "op": "grad8", "m": 4900, "n": 512, "k": 4608, "src": "bf16", "dst": "f32"},
        # The example's own loss: ten classes, a teacher's best four.
        {"name": "distill_small", "op": "distill", "rows": 96, "n": 10, "top": 4, "src": "f32", "dst": "f32", "temperature": 2.0,
         "soft": 0.5, "hard": 0.5, "grad": True},
        # A validation pass: the loss alone, over an odd number of classes, without labels.
        {"name": "distill_loss", "op": "distill", "rows": 2000, "n": 50_001, "top": 50, "src": "f32", "dst": "f32", "temperature": 1.0,
         "soft": 1.0, "hard": 0.0, "grad": False},
        # A training step over a large vocabulary: loss and gradient at once.
        {"name": "distill_large", "op": "distill", "rows": 4096, "n": 131_072, "top": 64, "src": "bf16", "dst": "bf16",
         "temperature": 2.0, "soft": 0.7, "hard": 0.3, "grad": True},
        # The backward pass by itself, as a program has it that learns the gradient of the loss only afterwards.
        {"name": "distill_grad", "op": "distill_grad", "rows": 3000, "n": 32_768, "top": 20, "src": "bf16", "dst": "bf16",
         "temperature": 3.0, "soft": 1.0, "hard": 0.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "linear8", "linear8", "grad8", "distill", "distill", "distill_grad"])
    types = ("f32", "bf16")
    if op in ("norm", "norm_grad"):
        n = _log_int(rng, 1, 40_000)
        return {"op": op, "rows": min(_log_int(rng, 1, 32_768), NORM_MOST // n), "n": n, "src": rng.choice(types),
                "dst": rng.choice(types), "weights": rng.choice(types)}
    if op in ("linear8", "grad8"):
        m, n, k = _log_int(rng, 1, 8192), _log_int(rng, 10, 16_384), _log_int(rng, 27, 8192)
        if op == "linear8" and rng.random() < 0.4:
            m = rng.randint(1, 16)
        m = max(1, min(m, PRODUCT_MOST // ((1 if op == "linear8" else 2) * n * k)))
        return {"op": op, "m": m, "n": n, "k": k, "src": rng.choice(types), "dst": rng.choice(types)}
    n = _log_int(rng, 2, 200_000)
    case = {"op": op, "rows": min(_log_int(rng, 1, 8192), LOGITS_MOST // n), "n": n, "top": min(_log_int(rng, 1, 256), n),
            "src": rng.choice(types), "dst": rng.choice(types), "temperature": rng.choice((1.0, 2.0, round(rng.uniform(0.5, 5.0), 3)))}
    case["soft"], case["hard"] = rng.choice(((1.0, 0.0), (0.5, 0.5), (0.9, 0.1)))
    if op == "distill":
        case["grad"] = rng.random() < 0.7
    return case


# ---- inputs -------------------------------------------------------------------------------------------------------

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _up(x, m):
    return (x + m - 1) // m * m


class State:
    """A program's buffers."""


def _normal(shape, gen, dtype, spread):
    """Normal values with another scale for each column, over decades where `spread` is large."""
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * torch.exp(spread * torch.randn((1, shape[1]), generator=gen, device="cuda"))).to(dtype)


def _prepare_norm(s, case, gen):
    rows, n, src, dst = case["rows"], case["n"], TYPES[case["src"]], TYPES[case["dst"]]
    # a residual stream: a few columns far larger than the others, rows off centre
    s.x = (_normal((rows, n), gen, torch.float32, 0.7) + 0.5 * torch.randn((rows, 1), generator=gen, device="cuda")).to(src)
    s.gamma = (1.0 + 0.2 * torch.randn(n, generator=gen, device="cuda")).to(TYPES[case["weights"]])
    s.beta = (0.1 * torch.randn(n, generator=gen, device="cuda")).to(TYPES[case["weights"]])
    s.mean, s.rstd = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    if case["op"] == "norm":
        s.y = torch.zeros((rows, n), dtype=dst, device="cuda")
        return
    x = s.x.float()
    s.mean.copy_(x.mean(1))
    s.rstd.copy_(((x - s.mean[:, None]).square().mean(1) + EPS).rsqrt())
    s.dy = (0.01 * torch.randn((rows, n), generator=gen, device="cuda")).to(src)
    s.dx = torch.zeros((rows, n), dtype=dst, device="cuda")
    s.dgamma, s.dbeta = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    s.scratch = None


def _prepare_product(s, case, gen):
    m, n, k = case["m"], case["n"], case["k"]
    s.x = _normal((m, k), gen, TYPES[case["src"]], 0.5)
    w = _normal((n, k), gen, torch.float32, 0.2) / math.sqrt(k)
    if case["op"] == "linear8":
        s.codes, s.scales = _hold(w)
        s.y = torch.zeros((m, n), dtype=TYPES[case["dst"]], device="cuda")
    else:
        s.dy = _normal((m, n), gen, TYPES[case["src"]], 0.5) * 0.01
        s.codes, s.scales = _hold(w.t().contiguous())     # along n, the contraction of dx
        s.dx = torch.zeros((m, k), dtype=TYPES[case["dst"]], device="cuda")
        s.dw = torch.zeros((n, k), device="cuda")
    s.scratch = None


def _prepare_distill(s, case, gen):
    rows, n, top = case["rows"], case["n"], case["top"]
    z = torch.randn((rows, n), generator=gen, device="cuda").mul_(1.5)
    # a teacher's best coordinates of each row, all of them different, best first; about one row in five has a shorter list
    start = torch.randint(0, n, (rows, 1), generator=gen, device="cuda")
    at = torch.arange(top, device="cuda")
    idx = (start + at * max(1, n // top)) % n
    t = 9.0 - 5.0 * torch.log1p(at.float()) / math.log1p(top) + torch.randn((rows, top), generator=gen, device="cuda")
    t = t.sort(1, descending=True)[0]
    # what a student knows of it by now
    z.scatter_add_(1, idx, 0.7 * t + torch.randn((rows, top), generator=gen, device="cuda"))
    length = torch.randint(1, top + 1, (rows, 1), generator=gen, device="cuda")
    whole = torch.rand((rows, 1), generator=gen, device="cuda") < 0.8
    s.idx = torch.where(whole | (at < length), idx, -1).to(torch.int32)
    s.top = t.to(TYPES[case["src"]])
    s.label = idx[:, 0].to(torch.int32)
    s.label[torch.rand(rows, generator=gen, device="cuda") < 0.05] = -1        # padding
    s.z = z.to(TYPES[case["src"]])
    s.grad = torch.full((rows,), 1.0 / rows, device="cuda")
    s.loss, s.stats = torch.zeros(rows, device="cuda"), torch.zeros((rows, 3), device="cuda")
    wanted = case["op"] == "distill_grad" or case["grad"]
    s.dz = torch.zeros((rows, n), dtype=TYPES[case["dst"]], device="cuda") if wanted else None
    s.scratch = None
    if case["op"] == "distill_grad":
        z = s.z.float()
        s.stats[:, 0] = z.amax(1)
        z -= s.stats[:, :1]
        s.stats[:, 1] = torch.exp(z / case["temperature"]).sum(1)
        s.stats[:, 2] = torch.exp(z).sum(1)


def prepare(case, seed):
    s = State()
    s.case = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] in ("norm", "norm_grad"):
        _prepare_norm(s, case, gen)
    elif case["op"] in ("linear8", "grad8"):
        _prepare_product(s, case, gen)
    else:
        _prepare_distill(s, case, gen)
    return s


# ---- plain torch --------------------------------------------------------------------------------------------------

def _power(e):
    """2 ** e in fp32, e from -127 to 127."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _split(x):
    """Per block of 128 of x's rows: the values over the block's power of two on the 8-bit grid, and the exponent."""
    rows, n = x.shape
    v = torch.nn.functional.pad(x.float(), (0, _up(n, 128) - n)).view(rows, -1, 128)
    f, e = torch.frexp(v.abs().amax(2, keepdim=True))
    e = torch.where(f > 0, e - 9 + (f > 0.875), -127).clamp(min=-127)
    t = v * _power(-e)
    a = t.abs()
    step = _power((torch.frexp(a)[1] - 1).clamp(min=-6) - 3)
    return torch.copysign(torch.round(a / step) * step, t), e


def _held(x):
    """x as 8 bits hold it, in fp32."""
    q, e = _split(x)
    return (q * _power(e)).view(x.shape[0], -1)[:, : x.shape[1]]


def _hold(x):
    """Codes and scales of x: what a program keeps of its weights."""
    q, e = _split(x)
    rows, blocks = e.shape[:2]
    scales = torch.zeros((rows, _up(blocks, 4)), dtype=torch.uint8, device="cuda")
    scales[:, :blocks] = (e[:, :, 0] + 127).to(torch.uint8)
    return q.to(torch.float8_e4m3fn).view(torch.uint8).view(rows, 128 * blocks), scales


def _values(codes, scales, n, dtype=torch.float32):
    """What codes and scales stand for, rows of n values."""
    q = codes.view(torch.float8_e4m3fn).to(dtype).view(codes.shape[0], -1, 128)
    e = scales[:, : q.shape[1], None].to(torch.int32) - 127
    return (q * _power(e)).view(codes.shape[0], -1)[:, :n]


def _scratch(s, need):
    """The program's scratch, kept with its weights."""
    if s.scratch is None or s.scratch.numel() < need:
        s.scratch = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s.scratch


def _plain_norm(s, case):
    x, gamma = s.x.float(), s.gamma.float()
    if case["op"] == "norm":
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = 1.0 / torch.sqrt(c.square().mean(1) + EPS)
        y = c * rstd[:, None] * gamma + s.beta.float()
        return {"y": y.to(TYPES[case["dst"]]), "mean": mean, "rstd": rstd}
    h = (x - s.mean[:, None]) * s.rstd[:, None]
    dy = s.dy.float()
    d = dy * gamma
    dx = s.rstd[:, None] * (d - d.mean(1, keepdim=True) - h * (d * h).mean(1, keepdim=True))
    return {"dx": dx.to(TYPES[case["dst"]]), "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}


def _plain_distill(s, case):
    temperature, soft, hard = case["temperature"], case["soft"], case["hard"]
    n = case["n"]
    z = s.z.float()
    rows = torch.arange(z.shape[0], device="cuda")
    live = (s.idx >= 0) & (s.idx < n)
    at = torch.where(live, s.idx, 0).long()
    t = torch.where(live, s.top.float() / temperature, -math.inf)
    t = t - t.amax(1, keepdim=True)
    log_p = t - torch.log(torch.exp(t).sum(1, keepdim=True))
    p = torch.exp(log_p)
    labelled = (s.label >= 0) & (s.label < n)
    label = torch.where(labelled, s.label, 0).long()
    if case["op"] == "distill":
        largest = z.amax(1)
        z = z - largest[:, None]
        sums = torch.exp(z / temperature).sum(1, keepdim=True)
        hard_sums = torch.exp(z).sum(1, keepdim=True) if hard else None
    else:
        z = z - s.stats[:, :1]
        sums, hard_sums = s.stats[:, 1:2], s.stats[:, 2:3]
    out = {}
    if case["op"] == "distill":
        log_q = z.gather(1, at) / temperature - torch.log(sums)
        loss = soft * temperature ** 2 * torch.where(live, p * (log_p - log_q), 0.0).sum(1)
        if hard:
            loss = loss + hard * torch.where(labelled, torch.log(hard_sums[:, 0]) - z[rows, label], 0.0)
        out["loss"] = loss
        out["stats"] = torch.stack([largest, sums[:, 0], hard_sums[:, 0] if hard else torch.zeros_like(largest)], 1)
    if s.dz is not None:
        dz = torch.exp(z / temperature) * (soft * temperature / sums)
        if hard:
            share = torch.where(labelled, hard, 0.0)[:, None]
            dz += torch.exp(z) * (share / hard_sums)
            dz.scatter_add_(1, label[:, None], -share)
        dz.scatter_add_(1, at, -soft * temperature * p)
        out["dz"] = (dz * s.grad[:, None]).to(TYPES[case["dst"]])
    return out


def _run_plain(s):
    case = s.case
    op = case["op"]
    if op in ("norm", "norm_grad"):
        return _plain_norm(s, case)
    if op == "linear8":
        return {"y": (_held(s.x) @ _values(s.codes, s.scales, case["k"]).t()).to(TYPES[case["dst"]])}
    if op == "grad8":
        dx = _held(s.dy) @ _values(s.codes, s.scales, case["n"]).t()
        return {"dx": dx.to(TYPES[case["dst"]]), "dw": _held(s.dy.t()) @ _held(s.x.t()).t()}
    return _plain_distill(s, case)


def run(s):
    if not own:
        return _run_plain(s)
    from paper_2011_06495_amd import binding as B
    case = s.case
    op = case["op"]
    if op == "norm":
        B.mv_layernorm_forward(s.x, s.gamma, s.beta, EPS, s.y, s.mean, s.rstd)
        return {"y": s.y, "mean": s.mean, "rstd": s.rstd}
    if op == "norm_grad":
        scratch = _scratch(s, B.mv_layernorm_scratch_bytes(case["rows"], case["n"]))
        B.mv_layernorm_backward(s.x, s.dy, s.gamma, s.mean, s.rstd, s.dx, s.dgamma, s.dbeta, scratch)
        return {"dx": s.dx, "dgamma": s.dgamma, "dbeta": s.dbeta}
    if op == "linear8":
        scratch = _scratch(s, B.mv_f8_linear_scratch_bytes(case["m"], case["n"], case["k"]))
        B.mv_f8_linear(s.x, s.codes, s.scales, s.y, scratch)
        return {"y": s.y}
    if op == "grad8":
        scratch = _scratch(s, B.mv_f8_linear_grad_scratch_bytes(case["m"], case["n"], case["k"]))
        B.mv_f8_linear_grad(s.x, s.dy, s.codes, s.scales, s.dx, s.dw, scratch)
        return {"dx": s.dx, "dw": s.dw}
    label = s.label if case["hard"] else None
    if op == "distill_grad":
        B.mv_distill_grad(s.z, s.idx, s.top, label, case["temperature"], case["soft"], case["hard"], s.stats, s.dz, grad=s.grad)
        return {"dz": s.dz}
    scratch = _scratch(s, B.mv_distill_scratch_bytes(case["rows"], case["n"]))
    B.mv_distill_loss(s.z, s.idx, s.top, label, case["temperature"], case["soft"], case["hard"], s.loss, scratch, stats=s.stats,
                      dz=s.dz, grad=s.grad if case["grad"] else None)
    return {"loss": s.loss, "stats": s.stats, **({"dz": s.dz} if case["grad"] else {})}


def work(case):
    """Bytes of the inputs, read once, and of the outputs, written once; additions, multiplications and exponentials for
    the operations."""
    op, size = case["op"], {"f32": 4, "bf16": 2}
    src, dst = size[case["src"]], size[case["dst"]]
    if op in ("norm", "norm_grad"):
        values, n = case["rows"] * case["n"], case["n"]
        if op == "norm":
            return {"bytes": values * (src + dst) + 2 * n * size[case["weights"]] + 8 * case["rows"], "flops": 8 * values}
        return {"bytes": values * (2 * src + dst) + n * (size[case["weights"]] + 8) + 8 * case["rows"], "flops": 14 * values}
    if op in ("linear8", "grad8"):
        m, n, k = case["m"], case["n"], case["k"]
        if op == "linear8":
            return {"bytes": m * k * src + n * k * 129 / 128 + m * n * dst, "flops": 2 * m * n * k}
        return {"bytes": m * (k + n) * src + n * k * 129 / 128 + m * k * dst + n * k * 4, "flops": 4 * m * n * k}
    values, grad = case["rows"] * case["n"], op == "distill_grad" or case["grad"]
    terms = 2 if case["hard"] and case["temperature"] != 1.0 else 1
    passes = (op == "distill") + grad
    return {"bytes": values * (src + (dst if grad else 0)) + case["rows"] * (case["top"] * (4 + src) + 12),
            "flops": values * terms * 3 * passes}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _near(x):
    """x, rows, in 64 bits as 8 bits hold it: the nearer of the grid's two neighbours, the even one in the middle."""
    rows, n = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -n % 128)).reshape(rows, -1, 128)
    top = x.abs().max(2, keepdim=True).values
    power = torch.exp2(torch.clamp(torch.ceil(torch.log2(top.clamp(min=2.0 ** -149) / 448.0)), min=-127.0))
    power = torch.where(top > 448.0 * power, 2.0 * power, torch.where((2.0 * top <= 448.0 * power) & (power > 2.0 ** -127), 0.5 * power,
                                                                    power))
    a = x.abs() / power
    unit = torch.exp2(torch.clamp(torch.floor(torch.log2(a.clamp(min=2.0 ** -40))), min=-6.0) - 3.0)
    low = torch.floor(a / unit)
    rest = a / unit - low
    low += (rest > 0.5) | ((rest == 0.5) & (low % 2.0 == 1.0))
    return (torch.sign(x) * low * unit * power).reshape(rows, -1)[:, :n]


def _exact_norm(s, case):
    x, gamma = s.x.double(), s.gamma.double()
    if case["op"] == "norm":
        mean = x.sum(1) / case["n"]
        var = ((x - mean[:, None]) ** 2).sum(1) / case["n"]
        rstd = (var + EPS) ** -0.5
        return {"y": (x - mean[:, None]) * rstd[:, None] * gamma + s.beta.double(), "mean": mean, "rstd": rstd}
    dx = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    dgamma, dbeta = (torch.zeros(case["n"], dtype=torch.float64, device="cuda") for _ in range(2))
    step = max(1, (1 << 24) // case["n"])
    for r in range(0, case["rows"], step):
        rstd = s.rstd[r:r + step].double()
        h = (x[r:r + step] - s.mean[r:r + step].double()[:, None]) * rstd[:, None]
        dy = s.dy[r:r + step].double()
        dgamma += (dy * h).sum(0)
        dbeta += dy.sum(0)
        d = dy * gamma
        along = (d * h).sum(1) / case["n"]
        dx[r:r + step] = (d - (d.sum(1) / case["n"])[:, None] - h * along[:, None]) * rstd[:, None]
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _exact_distill(s, case):
    rows, n, temperature, soft, hard = case["rows"], case["n"], case["temperature"], case["soft"], case["hard"]
    loss, stats = (torch.zeros(shape, dtype=torch.float64, device="cuda") for shape in (rows, (rows, 3)))
    dz = torch.empty((rows, n), dtype=torch.float64, device="cuda") if s.dz is not None else None
    step = max(1, (1 << 25) // n)
    for r in range(0, rows, step):
        z = s.z[r:r + step].double()
        idx, t = s.idx[r:r + step].long(), s.top[r:r + step].double()
        there = (idx > -1) & (idx < n)
        weight = torch.exp((t - t.max(1, keepdim=True).values) / temperature) * there
        p = weight / weight.sum(1, keepdim=True)
        teacher = torch.zeros(z.shape, dtype=torch.float64, device="cuda")
        for j in range(idx.shape[1]):
            teacher.scatter_add_(1, idx[:, j:j + 1].clamp(min=0), p[:, j:j + 1])
        label = s.label[r:r + step].long()
        truth = torch.zeros(z.shape, dtype=torch.float64, device="cuda")
        truth.scatter_(1, label.clamp(min=0)[:, None], (label > -1).double()[:, None])
        known = (label > -1).double()[:, None]
        if case["op"] == "distill":
            q, s1 = torch.log_softmax(z / temperature, 1), torch.log_softmax(z, 1)
            # every coordinate of a list is another one
            loss[r:r + step] = soft * temperature ** 2 * (torch.where(p > 0, p * torch.log(p.clamp(min=1e-300)), 0.0).sum(1) -
                                                          (teacher * q).sum(1)) - hard * (truth * s1).sum(1)
            q, s1 = torch.exp(q), torch.exp(s1)
            most = z.max(1).values
            stats[r:r + step, 0] = most
            stats[r:r + step, 1] = torch.exp(torch.logsumexp(z / temperature, 1) - most / temperature)
            if hard:
                stats[r:r + step, 2] = torch.exp(torch.logsumexp(z, 1) - most)
        else:
            st = s.stats[r:r + step].double()
            q, s1 = torch.exp((z - st[:, :1]) / temperature) / st[:, 1:2], torch.exp(z - st[:, :1]) / st[:, 2:3]
        if dz is not None:
            dz[r:r + step] = (soft * temperature * (q - teacher) + hard * (known * s1 - truth)) * s.grad[r:r + step].double()[:, None]
    return {**({"loss": loss, "stats": stats} if case["op"] == "distill" else {}), **({"dz": dz} if dz is not None else {})}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "norm_grad"):
        return _exact_norm(s, case)
    if op == "linear8":
        return {"y": _near(s.x) @ _values(s.codes, s.scales, case["k"], torch.float64).t()}
    if op == "grad8":
        return {"dx": _near(s.dy) @ _values(s.codes, s.scales, case["n"], torch.float64).t(),
                "dw": _near(s.dy.t()) @ _near(s.x.t()).t()}
    return _exact_distill(s, case)
