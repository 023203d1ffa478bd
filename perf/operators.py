"""The operators that let a training step keep less: the loss of a wide last layer whose logits are
never stored, with its gradients (linear_xent), activations kept in 8 bits (checkpoint_pack,
checkpoint_unpack) and the weight gradient that reads them (checkpoint_wgrad).

listed() names the cases, draw() gives further ones of the same ranges, prepare() makes what a
program holds before the call, run() is one pass: the plain form in elementary operations, or the
library's entry points where `own` is set.  work() says what a pass cannot do without, exact() what
it returns, from the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------------------------
#
# xent:  n rows of k features, c classes, the share `labelled` of the rows has a label; "train" returns
#        the loss and both gradients, "score" the loss of every row.
# pack:  n x k activations to 8 bits and back.
# wgrad: weight gradient k x m of n rows from 8-bit activations; with `masked`, of the gradient times
#        the ReLU derivative given as bits.

def listed():
    return [
        # one new node scored against a thousand classes: a call that is all latency
        {"name": "score_1_1000_f32", "op": "xent", "form": "score", "n": 1, "k": 128, "c": 1000,
         "labelled": 1.0, "dtype": "f32"},
        # a validation pass of odd size, losses row by row
        {"name": "score_10007_5003_bf16", "op": "xent", "form": "score", "n": 10007, "k": 256, "c": 5003,
         "labelled": 1.0, "dtype": "bf16"},
        # a small batch of nodes against a large vocabulary: weights and their gradient are most of
        # the traffic
        {"name": "train_96_32000_bf16", "op": "xent", "form": "train", "n": 96, "k": 256, "c": 32000,
         "labelled": 1.0, "dtype": "bf16"},
        # a full graph of which one node in ten has a label, classes of a citation graph (172)
        {"name": "train_262144_172_f32", "op": "xent", "form": "train", "n": 262144, "k": 128, "c": 172,
         "labelled": 0.1, "dtype": "f32"},
        # a middle-sized graph, every node with a label, fp32
        {"name": "train_4096_32768_f32", "op": "xent", "form": "train", "n": 4096, "k": 256, "c": 32768,
         "labelled": 1.0, "dtype": "f32"},
        # the largest: wide features, a large vocabulary, bf16 storage, a few rows without a label
        {"name": "train_16384_50001_bf16", "op": "xent", "form": "train", "n": 16384, "k": 512, "c": 50001,
         "labelled": 0.95, "dtype": "bf16"},
        # activations of the 4096-node configuration
        {"name": "pack_4096_64_f32", "op": "pack", "n": 4096, "k": 64, "dtype": "f32"},
        # activations of the R-MAT scale 20 configuration's hidden layers
        {"name": "pack_1m_256_f32", "op": "pack", "n": 1 << 20, "k": 256, "dtype": "f32"},
        # inputs of the 2.45M-node configuration, bf16, 100 columns: the last group is a part of one
        {"name": "pack_2m_100_bf16", "op": "pack", "n": 2450000, "k": 100, "dtype": "bf16"},
        # first layer of the 4096-node configuration
        {"name": "wgrad_4096_64_32_f32", "op": "wgrad", "n": 4096, "k": 64, "m": 32, "masked": True, "dtype": "f32"},
        # hidden layer of the R-MAT scale 20 configuration
        {"name": "wgrad_1m_256_256_f32", "op": "wgrad", "n": 1 << 20, "k": 256, "m": 256, "masked": True, "dtype": "f32"},
        # hidden layer of the 2.45M-node configuration, bf16 storage
        {"name": "wgrad_2m_256_256_bf16", "op": "wgrad", "n": 2450000, "k": 256, "m": 256, "masked": False, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: half of them round (a multiple of 32), half of them any number."""
    w = _log_int(rng, lo, hi)
    return max(32, (w + 16) // 32 * 32) if rng.random() < 0.5 else w


def draw(rng):
    op = rng.choice(["xent", "xent", "xent", "xent", "pack", "wgrad", "wgrad"])
    dtype = rng.choice(["f32", "bf16"])
    while True:
        if op == "xent":
            form = rng.choice(["train", "train", "train", "score"])
            case = {"op": op, "form": form, "n": _log_int(rng, 1, 300000), "k": _width(rng, 24, 512),
                    "c": _log_int(rng, 40, 60000), "labelled": rng.choice([1.0, 1.0, 0.9, 0.3, 0.05]), "dtype": dtype}
            rows = max(1.0, case["n"] * case["labelled"])
            if rows * case["c"] <= 7.5e8 and rows * case["k"] * case["c"] <= 4.0e11 and case["n"] * case["k"] <= 4e7:
                return case
        elif op == "pack":
            case = {"op": op, "n": _log_int(rng, 1, 2450000), "k": _width(rng, 20, 602), "dtype": dtype}
            if case["n"] * case["k"] <= 2.6e8:
                return case
        else:
            case = {"op": op, "n": _log_int(rng, 200, 2450000), "k": _width(rng, 24, 602), "m": _width(rng, 24, 512),
                    "masked": rng.random() < 0.5, "dtype": dtype}
            if case["n"] * case["k"] * case["m"] <= 1.2e11 and case["n"] * (case["k"] + case["m"]) <= 1.2e9:
                return case


# ---- inputs -------------------------------------------------------------------------------------

def _matrix(rows, cols, dtype):
    """rows x cols on a pitch of whole 16-byte groups."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.empty(rows, (cols + per - 1) // per * per, device="cuda", dtype=dtype)[:, :cols]


def _normal(gen, rows, cols, dtype):
    """Normal values with a scale of its own for every row, as aggregated features of nodes of few
    and of many neighbors have."""
    x = _matrix(rows, cols, dtype)
    scale = torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=gen))
    x.copy_(torch.randn(rows, cols, device="cuda", generator=gen).mul_(scale))
    return x


class State:
    pass


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = State()
    s.case = case
    n, k, dtype = case["n"], case["k"], DTYPES[case["dtype"]]
    if case["op"] == "xent":
        c = case["c"]
        s.h = _normal(gen, n, k, dtype)
        # logits of a model that has learnt something: a spread of a few units
        s.w = _matrix(k, c, torch.float32)
        s.w.normal_(0.0, 2.0 / math.sqrt(k), generator=gen)
        # some classes are frequent, most are rare
        y = (torch.rand(n, device="cuda", generator=gen).square() * c).int().clamp_(max=c - 1)
        if case["labelled"] < 1.0:
            off = torch.rand(n, device="cuda", generator=gen) >= case["labelled"]
            off[0] = False
            y[off] = -1
        s.labels = y
        s.row_loss = torch.empty(n, device="cuda")
        s.loss = torch.zeros(1, device="cuda", dtype=torch.float64)
        if case["form"] == "train":
            s.dh, s.dw = _matrix(n, k, dtype), _matrix(k, c, torch.float32)
    elif case["op"] == "pack":
        s.x = _normal(gen, n, k, dtype)
        s.back = _matrix(n, k, dtype)
        s.codes = torch.empty(n, (k + 15) // 16 * 16, device="cuda", dtype=torch.int8)[:, :k]
        s.exponents = torch.empty(n, (k + 31) // 32, device="cuda", dtype=torch.uint8)
    else:
        m = case["m"]
        # what packing normal values leaves: a largest code between 64 and 127 in every group of 32 columns,
        # steps around 2^-5
        x = _normal(gen, n, k, dtype)
        groups = (k + 31) // 32
        s.codes = torch.empty(n, (k + 15) // 16 * 16, device="cuda", dtype=torch.int8)[:, :k]
        s.exponents = torch.empty(n, groups, device="cuda", dtype=torch.uint8)
        for g in range(groups):
            part = x[:, 32 * g:32 * g + 32].float()
            step = torch.ceil(torch.log2(part.abs().amax(1).clamp_(min=1e-30) / 127.0))
            s.codes[:, 32 * g:32 * g + 32] = torch.round(part * torch.exp2(-step)[:, None]).clamp_(-127, 127)
            s.exponents[:, g] = step + 133
        s.g = _normal(gen, n, m, dtype)
        s.mask = None
        if case["masked"]:
            # the derivative of a ReLU: about half of the elements
            s.mask = torch.randint(-2 ** 31, 2 ** 31, (n, (m + 31) // 32), device="cuda", generator=gen).int()
        s.dw = _matrix(k, m, torch.float32)
    return s


# ---- one pass -----------------------------------------------------------------------------------

def _powers(e):
    """2^e of whole numbers e, exactly, from -126 to 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _steps(exponents, cols):
    """The powers of two of the groups of 32 columns, for every column."""
    return _powers(exponents.int() - 133).repeat_interleave(32, dim=1)[:, :cols]


def _plain_xent(s):
    c, train = s.w.shape[1], s.case["form"] == "train"
    rows = ((s.labels >= 0) & (s.labels < c)).nonzero()[:, 0]
    y = s.labels[rows].long()[:, None]
    h = s.h[rows].float()
    logits = h @ s.w
    top = logits.amax(1, keepdim=True)
    at_label = logits.gather(1, y)
    p = torch.exp(logits.sub_(top))
    total = p.sum(1, keepdim=True)
    losses = (torch.log(total) + top - at_label)[:, 0]
    if not train:
        return torch.zeros_like(s.row_loss).index_copy_(0, rows, losses)
    p.div_(total)
    p.scatter_add_(1, y, torch.full_like(at_label, -1.0))
    p.div_(rows.numel())
    dh = torch.zeros(s.h.shape, device="cuda", dtype=s.h.dtype)
    dh[rows] = (p @ s.w.t()).to(s.h.dtype)
    return {"loss": losses.double().mean().float(), "dh": dh, "dw": h.t() @ p}


def _plain_pack(s):
    n, k = s.x.shape
    x = torch.nn.functional.pad(s.x.float(), (0, -k % 32)).view(n, -1, 32)
    top = x.abs().amax(2, keepdim=True)
    step = torch.frexp(top)[1] - 7
    step += top * _powers(-step) >= 127.5
    step.clamp_(min=-133)
    codes = torch.round(x * _powers(-step))
    return (codes * _powers(step)).view(n, -1)[:, :k].to(s.x.dtype)


def _plain_wgrad(s):
    z = s.codes.float() * _steps(s.exponents, s.codes.shape[1])
    g = s.g.float()
    if s.mask is not None:
        bit = torch.arange(g.shape[1], device="cuda")
        g = g * ((s.mask[:, bit // 32] >> (bit % 32).int()) & 1)
    return z.t() @ g


def run(s):
    op = s.case["op"]
    if not own:
        return {"xent": _plain_xent, "pack": _plain_pack, "wgrad": _plain_wgrad}[op](s)
    import paper_2501_01951_amd as mg
    if op == "xent":
        if s.case["form"] == "score":
            mg.linear_xent(s.h, s.w, s.labels, row_loss=s.row_loss)
            return s.row_loss
        mg.linear_xent(s.h, s.w, s.labels, loss=s.loss, dH=s.dh, dW=s.dw)
        return {"loss": s.loss[0].float(), "dh": s.dh, "dw": s.dw}
    if op == "pack":
        kept = mg.Checkpoint(s.codes, s.exponents)
        mg.checkpoint_pack(s.x, kept)
        mg.checkpoint_unpack(kept, s.back)
        return s.back
    mg.checkpoint_wgrad(mg.Checkpoint(s.codes, s.exponents), s.g, s.dw, mask=s.mask)
    return s.dw


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    n, k = float(case["n"]), float(case["k"])
    e = 2.0 if case["dtype"] == "bf16" else 4.0
    if case["op"] == "xent":
        c, rows = float(case["c"]), max(1.0, case["n"] * case["labelled"])
        # labelled rows and weights read; with gradients, both of those written, rows without a label as zeros
        bytes_, flops = 4.0 * n + e * rows * k + 4.0 * k * c, 2.0 * rows * k * c
        if case["form"] == "train":
            return {"bytes": bytes_ + e * n * k + 4.0 * k * c, "flops": 3.0 * flops}
        return {"bytes": bytes_ + 4.0 * n, "flops": flops}
    kept = n * k + n * math.ceil(k / 32.0)
    if case["op"] == "pack":
        return {"bytes": 2.0 * (e * n * k + kept), "flops": 4.0 * n * k}
    m = float(case["m"])
    return {"bytes": kept + e * n * m + (n * m / 8.0 if case["masked"] else 0.0) + 4.0 * k * m, "flops": 2.0 * n * k * m}


# ---- the same from the definitions in 64 bits -----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "xent":
        return _exact_xent(s)
    if case["op"] == "pack":
        return _exact_pack(s)
    n, k = s.codes.shape
    powers = _exact_powers()
    dw = torch.zeros(k, s.g.shape[1], device="cuda", dtype=torch.float64)
    block = max(1, (1 << 27) // (k + s.g.shape[1]))
    for r in range(0, n, block):
        z = torch.empty(min(block, n - r), k, device="cuda", dtype=torch.float64)
        for g in range(s.exponents.shape[1]):
            scale = powers[s.exponents[r:r + block, g].long()]
            z[:, 32 * g:32 * g + 32] = s.codes[r:r + block, 32 * g:32 * g + 32].double() * scale[:, None]
        up = s.g[r:r + block].double()
        if s.mask is not None:
            for j in range(up.shape[1]):
                up[:, j] *= torch.bitwise_and(torch.bitwise_right_shift(s.mask[r:r + block, j // 32], j % 32), 1)
        dw += torch.matmul(z.transpose(0, 1).contiguous(), up)
    return dw


def _exact_xent(s):
    n, c = s.h.shape[0], s.w.shape[1]
    w = s.w.double()
    wt = w.transpose(0, 1).contiguous()
    have = torch.nonzero(torch.logical_and(s.labels >= 0, s.labels < c)).flatten()
    count = have.shape[0]
    losses = torch.zeros(n, device="cuda", dtype=torch.float64)
    train = s.case["form"] == "train"
    dh = torch.zeros(s.h.shape, device="cuda", dtype=torch.float64) if train else None
    dw = torch.zeros_like(w) if train else None
    block = max(1, (1 << 28) // c)
    for b in range(0, count, block):
        rows = have[b:b + block]
        h = s.h[rows].double()
        logp = torch.log_softmax(torch.matmul(h, w), 1)
        i = torch.arange(rows.shape[0], device="cuda")
        y = s.labels[rows].long()
        losses[rows] = -logp[i, y]
        if train:
            logp.exp_()
            logp[i, y] -= 1.0
            logp *= 1.0 / count
            dh[rows] = torch.matmul(logp, wt)
            dw += torch.matmul(h.transpose(0, 1).contiguous(), logp)
    if not train:
        return losses
    return {"loss": losses.sum() / count, "dh": dh, "dw": dw}


def _exact_powers():
    """2^-133 .. 2^122 as a table from the host (the device's pow need not be exact)."""
    return torch.tensor([2.0 ** e for e in range(-133, 123)], dtype=torch.float64, device="cuda")


def _exact_pack(s):
    powers = _exact_powers()
    out = torch.empty(s.x.shape, device="cuda", dtype=torch.float64)
    for g in range(0, s.x.shape[1], 32):
        x = s.x[:, g:g + 32].double()
        # the smallest power of two at which the largest value is rounded to 127 at most
        step = torch.floor(torch.log2(x.abs().amax(1).clamp_(min=2.0 ** -126))).long() - 6
        step += torch.round(x.abs().amax(1) / powers[step + 133]) > 127
        unit = powers[step + 133][:, None]
        out[:, g:g + 32] = torch.round(x / unit) * unit
    return out
