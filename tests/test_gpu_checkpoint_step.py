"""The GCN step that keeps its aggregates in 8 bits and no logits: all of its operators together, against dense products
in 64 bits."""
import pytest

from parity import say

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def mg():
    import paper_2501_01951_amd as m

    m.load_library()
    return m


def problem(mg, n, dims, dtype, seed, labelled=0.7):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    src = torch.randint(0, n, (6 * n,), device="cuda", generator=gen, dtype=torch.int32)
    dst = torch.randint(0, n, (6 * n,), device="cuda", generator=gen, dtype=torch.int32)
    g = mg.build_csr(src, dst, n)
    mg.normalize(g)
    arr = g.arrays()
    a = torch.zeros(n, n, device="cuda", dtype=torch.float64)
    row = torch.repeat_interleave(torch.arange(n, device="cuda"), arr["rowptr"].diff())
    a[row, arr["col"].long()] = arr["val"].double()
    x = torch.randn(n, dims[0], device="cuda", generator=gen).to(dtype)
    ws = []
    for f, m in zip(dims, dims[1:]):
        w = torch.zeros(f, (m + 3) // 4 * 4, device="cuda")[:, :m]
        w.normal_(0, (2.0 / f) ** 0.5, generator=gen)
        ws.append(w)
    y = torch.randint(0, dims[-1], (n,), device="cuda", generator=gen, dtype=torch.int32)
    y[torch.rand(n, device="cuda", generator=gen) >= labelled] = -1
    return g, a, x, ws, y


def values(kept):
    unit = torch.tensor([2.0 ** e for e in range(-133, 123)], device="cuda", dtype=torch.float64)[kept.exponents.long()]
    unit = unit.repeat_interleave(32, 1)[:, :kept.codes.shape[1]]
    return kept.codes.double() * unit, unit


def bits(mask, m):
    j = torch.arange(m, device="cuda")
    return ((mask[:, j // 32] >> (j % 32).int()) & 1).bool()


def reference(step, a, x, ws, y):
    """Loss and gradients of the step's own ReLU decisions (one of a pre-activation within rounding of zero may fall either way),
    in 64 bits; the hidden layers' weight gradients of the aggregates in 64 bits, and the gradients they are of."""
    L, n = len(ws), x.shape[0]
    h, zs, pre = x.double(), [], []
    for l, w in enumerate(ws):
        zs.append(a @ h)
        p = zs[-1] @ w.double()
        if l < L - 1:
            pre.append(p)
            h = torch.where(bits(step.positive[l], p.shape[1]), p, 0.0)
    rows = ((y >= 0) & (y < p.shape[1])).nonzero()[:, 0]
    logp = torch.log_softmax(p[rows], 1)
    at = torch.arange(rows.numel(), device="cuda")
    losses = torch.zeros(n, device="cuda", dtype=torch.float64)
    losses[rows] = -logp[at, y[rows].long()]
    d = logp.exp()
    d[at, y[rows].long()] -= 1
    g = torch.zeros_like(p)
    g[rows] = d / rows.numel()
    dws, gs = [None] * L, [None] * L
    for l in range(L - 1, -1, -1):
        dws[l], gs[l] = zs[l].t().contiguous() @ g, g
        if l > 0:
            g = a.t().contiguous() @ (g @ ws[l].double().t().contiguous())
            g = torch.where(bits(step.positive[l - 1], g.shape[1]), g, 0.0)
    return losses, losses.sum() / rows.numel(), zs, pre, dws, gs


def near(got, want, rel, what):
    off = ((got.double() - want).norm() / want.norm()).item()
    assert off <= rel, (what, off)


@pytest.mark.parametrize("dims", [(40, 64, 48, 333), (100, 32, 32, 32, 700), (24, 50)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step(mg, dims, dtype):
    """fp32: chains of up to a dozen products with fp32 sums, each off by a few 2^-24 of its terms: 1e-5 in 2-norm.  bf16: every
    stored tensor is rounded by 2^-8 at most, 2^-9.8 in the mean, and a dozen of them follow each other: 2e-2."""
    say(f"checkpoint step {dims} {dtype}")
    rel = 1e-5 if dtype == "f32" else 2e-2
    g, a, x, ws, y = problem(mg, 700, dims, DTYPES[dtype], 3)
    step = mg.GCNCheckpointStep(g, x, ws, y)
    for w in step.dw:
        w.fill_(float("nan"))
    step.step()
    torch.cuda.synchronize()
    losses, loss, zs, pre, dws, gs = reference(step, a, x, ws, y)
    near(step.loss[0], loss, rel, "loss")
    near(step.dw[-1], dws[-1], rel, "dW of the last layer")
    for l in range(len(ws) - 1):
        # ReLU decisions differ only next to zero
        flipped = bits(step.positive[l], pre[l].shape[1]) != (pre[l] > 0)
        assert (pre[l][flipped].abs() <= 4 * rel * pre[l].abs().mean()).all(), l
        z, unit = values(step.kept[l])
        # an 8-bit aggregate is off by half a step, and by the rounding of what was packed
        assert ((z - zs[l]).abs() <= unit / 2 + rel * zs[l].abs() + rel * zs[l].abs().mean()).all(), l
        near(step.dw[l], z.t().contiguous() @ gs[l], 2 * rel, f"dW of layer {l} of what was kept")
        off = (unit / 2).t().contiguous() @ gs[l].abs()
        assert ((step.dw[l].double() - dws[l]).abs() <= off + 4 * rel * (zs[l].abs().t().contiguous() @ gs[l].abs())).all(), l
    near(step.score(), losses, rel, "score")
    other = torch.randint(0, dims[-1], (700,), device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()
    scored = step.score(other)
    torch.cuda.synchronize()
    assert (scored > 0).all()


def test_full_precision_step_agrees(mg):
    """The loss and the last layer's weight gradient are those of the step that keeps everything."""
    say("checkpoint step beside the full one")
    g, _, x, ws, y = problem(mg, 3000, (64, 96, 200), torch.float32, 5, labelled=1.0)
    step, full = mg.GCNCheckpointStep(g, x, ws, y), mg.GCNStep(g, x, ws, y, reorder=False)
    step.step()
    full.step()
    torch.cuda.synchronize()
    near(step.loss, full.loss, 1e-6, "loss")
    near(step.dw[1], full.dw[1].double(), 1e-5, "dW")
    # an element of Z is off by half a step in 64 to 127 steps, evenly: 2^-7.5 / sqrt(12) of its group's largest, less than
    # a hundredth of the features' size; their sum over the nodes averages it out
    near(step.dw[0], full.dw[0].double(), 0.02, "dW of the 8-bit aggregates")


def test_less_memory(mg):
    n, dims = 20000, (128, 128, 128, 128, 1000)
    gen = torch.Generator(device="cuda").manual_seed(1)
    src, dst = (torch.randint(0, n, (4 * n,), device="cuda", generator=gen, dtype=torch.int32) for _ in range(2))
    g = mg.build_csr(src, dst, n)
    mg.normalize(g)
    x = torch.randn(n, dims[0], device="cuda")
    ws = [torch.randn(a, b, device="cuda") * 0.1 for a, b in zip(dims, dims[1:])]
    y = torch.randint(0, dims[-1], (n,), device="cuda", dtype=torch.int32)
    step = mg.GCNCheckpointStep(g, x, ws, y)
    per_node = sum(k.codes.stride(0) + k.exponents.stride(0) for k in step.kept) + sum(4 * p.stride(0) for p in step.positive)
    assert per_node == 3 * (128 + 4 + 16)
    assert len(step.z) == len(step.h) == 1


def test_captured_step(mg):
    """Recorded and replayed with other weights in between, against the eager step."""
    say("checkpoint step captured")
    g, _, x, ws, y = problem(mg, 900, (40, 64, 300), torch.float32, 8)
    step, eager = mg.GCNCheckpointStep(g, x, ws, y), mg.GCNCheckpointStep(g, x, ws, y)
    eager.step()
    mg.graph_reserve_streams(g, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.step()
    for trip in range(3):
        for w in ws:
            w.mul_(1.1)
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert torch.equal(step.loss, eager.loss)
        assert all(torch.equal(p, q) for p, q in zip(step.dw, eager.dw))


def test_backward_without_its_forward(mg):
    """The gradient that backward starts from is gone after a backward or a score."""
    say("checkpoint step out of order")
    g, _, x, ws, y = problem(mg, 500, (24, 32, 90), torch.float32, 9)
    step = mg.GCNCheckpointStep(g, x, ws, y)
    with pytest.raises(RuntimeError, match="forward"):
        step.backward()
    step.step()
    with pytest.raises(RuntimeError, match="forward"):
        step.backward()
    step.forward()
    step.score()
    with pytest.raises(RuntimeError, match="forward"):
        step.backward()
    want = [w.clone() for w in step.dw]
    step.step()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(step.dw, want))
