"""How near the loss without logits and its gradients come to 64 bits where rounding shows: gradients whose terms cancel,
losses next to zero, features and rows of very different magnitudes."""
import pytest

from parity import say

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

NAN = float("nan")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def mg():
    import paper_2501_01951_amd as m

    m.load_library()
    return m


def matrix(rows, cols, dtype, fill=NAN):
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.full((rows, (cols + per - 1) // per * per), fill, device="cuda", dtype=dtype)[:, :cols]


def inputs(n, k, c, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed + 7 * n + 3 * k + c)
    h, w = matrix(n, k, dtype), matrix(k, c, torch.float32)
    h[:] = torch.randn(n, k, device="cuda", generator=gen)
    w[:] = torch.randn(k, c, device="cuda", generator=gen) * (2.0 / k ** 0.5)
    y = torch.randint(0, c, (n,), device="cuda", generator=gen, dtype=torch.int32)
    return h, w, y


def results(mg, h, w, y):
    """loss, row_loss, dH, dW"""
    out = (torch.full((1,), NAN, device="cuda", dtype=torch.float64), torch.full((h.shape[0],), NAN, device="cuda"),
           matrix(*h.shape, h.dtype), matrix(*w.shape, torch.float32))
    mg.linear_xent(h, w, y, loss=out[0], row_loss=out[1], dH=out[2], dW=out[3])
    torch.cuda.synchronize()
    return out


def reference(h, w, y):
    """losses and (softmax - onehot) / n of rows that all have a label"""
    logp = torch.log_softmax(h.double() @ w.double(), 1)
    at = torch.arange(h.shape[0], device="cuda")
    g = logp.exp()
    g[at, y.long()] -= 1
    return -logp[at, y.long()], g / h.shape[0]


def within(what, got, ref, off):
    bad = ~((got.double() - ref).abs() <= off)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist(), off[bad][:4].tolist())


def steps(terms):
    """What a sum of products of two f16 terms each is off by, of the sum of |a| |b|: 2^-22 of either operand and the product
    of both rests; fp32 sums of 16 terms in three products to a step, cut to 2^-23, and up to 64 pieces joined."""
    return (3 + 3 * (terms // 16 + 1) + 64) * 2.0 ** -22


@pytest.mark.parametrize("common", [16.0, 64.0])
@pytest.mark.parametrize("n,k,c", [(600, 64, 700), (300, 130, 200), (2100, 256, 1500), (500, 40, 60)])
def test_gradient_of_bf16_features_whose_weights_have_a_common_part(mg, n, k, c, common):
    """The classes' weights of a feature are a common number, which cancels in sum G W, and a spread of 1/4 around it.  G and W
    are fp32 numbers: what is left is off by the rounding to bf16 (2^-8) and by what 22 bits of them leave, 2^-22 of
    their products (half a thousandth here; 11 bits would leave 2^-11).  The features are so small that the logits, and
    with them G, are exact to 2^-21 of G."""
    say(f"linear_xent n={n} k={k} c={c} common part {common}")
    h, w, y = inputs(n, k, c, torch.bfloat16, 31)
    h.mul_(2.0 ** -14)
    gen = torch.Generator(device="cuda").manual_seed(5)
    w.copy_(torch.randn(k, c, device="cuda", generator=gen) / 4 + common * (1 + torch.rand(k, 1, device="cuda", generator=gen)))
    dh = results(mg, h, w, y)[2]
    _, g = reference(h, w, y)
    wd = w.double().t().contiguous()
    # off in G: its logits' errors, sum |h| |w| steps, and the resolution 2^-39
    e = (h.double().abs() @ w.double().abs()).amax(1, keepdim=True) * steps(k) + 2.0 ** -21
    g_off = (g.abs() * 2 * e) + 2.0 ** -39 / n
    want = g @ wd
    within("dH", dh, want, want.abs() * 2.0 ** -8 + g_off @ wd.abs() + (g.abs() @ wd.abs()) * steps(c))


@pytest.mark.parametrize("size", [1.0, 30.0, 300.0, 1500.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [50, 190, 700, 5000])
def test_losses_of_confident_rows(mg, c, dtype, size):
    """Logits of `size` and more, and the label the largest of them.  No loss is below zero; and one whose row has no other logit
    within 20 of the largest is off by what the other logits' differences from it are, relative to itself, and by a rounding to
    2^-23 of 1 + sum exp, the least of a sum of fp32 numbers, and of its logarithm."""
    say(f"linear_xent confident rows c={c} {dtype} size {size}")
    h, w, y = inputs(800, 64, c, DTYPES[dtype], 32)
    w.mul_(size)
    s = h.double() @ w.double()
    y.copy_(s.argmax(1))
    row_loss = results(mg, h, w, y)[1]
    assert (row_loss >= 0).all(), row_loss.min()
    far = s.sort(1, descending=True)[0]
    sure = far[:, 0] - far[:, 1] > 20
    assert size == 1.0 or sure.sum() > 20
    want = reference(h, w, y)[0]
    e = (h.double().abs() @ w.double().abs()).amax(1) * steps(64)
    within("row_loss", row_loss[sure], want[sure], (want * torch.expm1(2 * e))[sure] + 2.0 ** -22)
    # any label: a sum of exponentials that has its largest term is at least that
    y.copy_(torch.randint(0, c, (800,), device="cuda", dtype=torch.int32))
    assert (results(mg, h, w, y)[1] >= 0).all()


@pytest.mark.parametrize("side", ["H", "W", "both"])
@pytest.mark.parametrize("power", [-20, -45, -60, -80, -100, 0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [150, 400])
def test_gradients_of_features_that_hardly_count(mg, c, dtype, power, side):
    """Columns of H, or rows of W, next to zero (0: zero): the gradient with respect to the other operand is as large as any
    feature's, and is off by 2^-22 of its feature's largest element (of the other operand, times the sum of |G|) beside what other
    features' are."""
    say(f"linear_xent c={c} {dtype} small {side} 2^{power}")
    h, w, y = inputs(500, 40, c, DTYPES[dtype], 33)
    factor = 2.0 ** power if power else 0.0
    if side != "W":
        h[:, 7] *= factor
        h[:, 30] *= factor
    if side != "H":
        w[11] *= factor
        w[30] *= factor
    loss, row_loss, dh, dw = results(mg, h, w, y)
    want, g = reference(h, w, y)
    n, hd, wd = 500, h.double(), w.double()
    e = (hd.abs() @ wd.abs()).amax(1, keepdim=True) * steps(40) + 2.0 ** -21
    within("row_loss", row_loss, want, 2 * e[:, 0])
    # a probability is off by twice its logits' errors, relative to itself, and by 2^-39
    g_off, a, ht = g.abs().clamp(max=1.0 / n) * 2 * e + 2.0 ** -39 / n, g.abs(), hd.t().contiguous()
    wt = wd.t().contiguous()
    off = g_off @ wt.abs() + (a @ wt.abs()) * steps(c) + a.sum(1, keepdim=True) * wd.abs().amax(1) * 2.0 ** -22
    ref = g @ wt
    within("dH", dh, ref, off + ref.abs() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24))
    off = ht.abs() @ g_off + (ht.abs() @ a) * steps(n) + hd.abs().amax(0)[:, None] * a.sum(0) * 2.0 ** -22
    ref = ht @ g
    within("dW", dw, ref, off + ref.abs() * 2.0 ** -24)


# ---- rows and classes of very different magnitudes -------------------------------------------------

def sum_off(terms):
    """As steps(), or sums of fp32 products, two terms to a step, each cut to 2^-23."""
    return max(steps(terms), (terms // 2 + 70) * 2.0 ** -23)


def check(mg, h, w, y, dtype):
    """Every result against 64 bits, with no allowance for what other rows or classes hold: an element of G is off by its own
    logits' errors, the rounding of a probability, and the resolution of G; one that is 0 or 1 to the last bit by nothing."""
    n, k = h.shape
    c = w.shape[1]
    loss, row_loss, dh, dw = results(mg, h, w, y)
    want, g = reference(h, w, y)
    hd, wd = h.double(), w.double()
    s_off = (hd.abs() @ wd.abs()) * sum_off(k)
    e = s_off.amax(1, keepdim=True) + 2.0 ** -22 * (1 + want[:, None])
    within("row_loss", row_loss, want, 2 * e[:, 0])
    within("loss", loss, want.mean().view(1), 2 * e.mean().view(1) + 1e-15)
    p = g.clone()
    p[torch.arange(n, device="cuda"), y.long()] += 1.0 / n
    g_off = torch.where(g.abs() > 1e-30, (g.abs().clamp(max=1.0 / n) * torch.expm1((2 * e).clamp(max=1.0)) + p * 2.0 ** -22 + 2.0 ** -39 / n), 0.0)
    a, ht, wt = g.abs(), hd.t().contiguous(), wd.t().contiguous()
    ref = g @ wt
    within("dH", dh, ref, g_off @ wt.abs() + (a @ wt.abs()) * sum_off(c) + ref.abs() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24))
    ref = ht @ g
    within("dW", dw, ref, ht.abs() @ g_off + (ht.abs() @ a) * sum_off(n) + ref.abs() * 2.0 ** -24)


@pytest.mark.parametrize("label", ["largest", "any"])
@pytest.mark.parametrize("power", [20, 24, 30, 36, 100])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [150, 700])
def test_one_row_far_larger_than_the_others(mg, c, dtype, power, label):
    """The others' losses and gradients are as good as without it; also dW, to which it adds nothing where its label is its
    largest logit."""
    say(f"linear_xent c={c} {dtype} one row 2^{power} {label}")
    h, w, y = inputs(300, 48, c, DTYPES[dtype], 34)
    h[17] *= 2.0 ** power
    if label == "largest":
        y[17] = (h[17].double() @ w.double()).argmax()
    check(mg, h, w, y, dtype)


@pytest.mark.parametrize("power", [20, 30, 100])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [150, 700])
def test_one_class_far_larger_than_the_others(mg, c, dtype, power):
    """Its logit is by far the largest of half of the rows, and by far the least of the other half, whose losses are the
    others' alone."""
    say(f"linear_xent c={c} {dtype} one class 2^{power}")
    h, w, y = inputs(300, 48, c, DTYPES[dtype], 35)
    w[:, 33] *= 2.0 ** power
    check(mg, h, w, y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,c", [(1, 1, 1), (1, 4, 2), (3, 128, 1000), (129, 100, 300), (64, 602, 65), (513, 257, 700), (40, 8, 9001), (2049, 32, 47),
                                   (3000, 130, 172), (400, 20, 250), (2500, 256, 600), (16700, 8, 8300), (140001, 8, 5), (96, 192, 1000)])
def test_large_products_of_every_size(mg, n, k, c, dtype):
    """Logits of 2^18 and more beside ordinary ones: tiles and pieces of every kind."""
    say(f"linear_xent large products n={n} k={k} c={c} {dtype}")
    h, w, y = inputs(n, k, c, DTYPES[dtype], 36)
    h[n // 2] *= 2.0 ** 20
    if n * c < 1 << 24:
        check(mg, h, w, y, dtype)
        return
    # dW and the mean only: what the rows are is checked at the other sizes
    loss, row_loss, dh, dw = results(mg, h, w, y)
    e = (h.double().abs() @ w.double().abs().amax(1, keepdim=True))[:, 0] * sum_off(k) + 2.0 ** -18
    at, ref = torch.arange(n, device="cuda"), torch.zeros(k, c, device="cuda", dtype=torch.float64)
    for b in range(0, n, 4096):
        want, g = reference(h[b:b + 4096], w, y[b:b + 4096])
        within("row_loss", row_loss[b:b + 4096], want, 2 * e[b:b + 4096])
        g *= g.shape[0] / n
        ref += h[b:b + 4096].double().t().contiguous() @ g
        got, dref = dh[b:b + 4096].double(), g @ w.double().t().contiguous()
        assert (got - dref).norm() <= 4e-3 * dref.norm()
    assert (dw.double() - ref).norm() <= 1e-4 * ref.norm()


def test_large_products_not_finite(mg):
    """Where products are fp32 as where they are not: a row that has an infinity or NaN has a loss and gradient that are NaN, no
    other row has."""
    for value in (float("inf"), -float("inf"), NAN):
        h, w, y = inputs(260, 24, 100, torch.float32, 37)
        h[50] *= 2.0 ** 24
        say(f"linear_xent large products and {value}")
        clean = results(mg, h, w, y)
        h[133, 7] = value
        loss, row_loss, dh, dw = results(mg, h, w, y)
        other = torch.arange(260, device="cuda") != 133
        assert loss.isnan().all() and row_loss[133].isnan() and dh[133].isnan().all() and dw.isnan().all()
        assert torch.equal(row_loss[other], clean[1][other]) and torch.equal(dh[other], clean[2][other])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_graph_whose_products_become_large(mg, dtype):
    """What the products run on is settled by what the operands hold when the graph runs."""
    say(f"linear_xent graph of ordinary and large products {dtype}")
    h, w, y = inputs(900, 64, 500, DTYPES[dtype], 38)
    out = (torch.zeros(1, device="cuda", dtype=torch.float64), torch.zeros(900, device="cuda"), matrix(900, 64, h.dtype), matrix(64, 500, torch.float32))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mg.linear_xent(h, w, y, loss=out[0], row_loss=out[1], dH=out[2], dW=out[3])
    for factor in (1.0, 2.0 ** 22, 2.0 ** -22, 2.0 ** 30):
        h[5] *= factor
        graph.replay()
        eager = results(mg, h, w, y)
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
        assert torch.isfinite(out[1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_products_with_the_gradient_over_the_features(mg, dtype):
    say(f"linear_xent large products, dH over H {dtype}")
    for n, k, c in ((900, 40, 300), (700, 96, 120), (3000, 200, 2000)):
        h, w, y = inputs(n, k, c, DTYPES[dtype], 39)
        h[7] *= 2.0 ** 25
        y[::5] = -1
        dh, dw, again = matrix(n, k, h.dtype), matrix(k, c, torch.float32), matrix(k, c, torch.float32)
        mg.linear_xent(h, w, y, dH=dh, dW=dw)
        mg.linear_xent(h, w, y, dH=h, dW=again)
        torch.cuda.synchronize()
        assert torch.equal(h, dh) and torch.equal(dw, again) and torch.isfinite(dw).all()


@pytest.mark.parametrize("scale", [1.0, 2.0 ** 20])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), NAN])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [1, 50, 64, 190, 700])
def test_a_class_whose_weights_are_not_finite(mg, c, dtype, value, scale):
    """Features that are all of one sign, or short in bits, make a logit of one infinity without a NaN on its way: a row that has one is
    NaN all the same.  Rows of zeros have NaN logits."""
    say(f"linear_xent c={c} {dtype} a class of {value} scale {scale}")
    for at in {0, c // 2, c - 1}:
        h, w, y = inputs(200, 24, c, DTYPES[dtype], 40)
        h.abs_()
        h.mul_(16).ceil_().mul_(scale)
        w[:, at] = value
        y.copy_(torch.where(y == at, (at + 1) % c, y))
        loss, row_loss, dh, dw = results(mg, h, w, y)
        assert loss.isnan().all() and row_loss.isnan().all() and dh.isnan().all() and dw.isnan().all()


@pytest.mark.parametrize("c", [50, 700])
def test_logits_past_the_largest_float(mg, c):
    """fp32 operands that are finite and logits that are not: that row is NaN, others are as they were."""
    say(f"linear_xent c={c} a logit past the largest float")
    h, w, y = inputs(200, 24, c, torch.float32, 41)
    h[9] = -(2.0 ** 100)
    w.abs_()
    clean = results(mg, h, w, y)
    assert torch.isfinite(clean[1]).all()
    h[9] = -(2.0 ** 127)
    row_loss = results(mg, h, w, y)[1]
    other = torch.arange(200, device="cuda") != 9
    assert row_loss[9].isnan() and torch.equal(row_loss[other], clean[1][other])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,c", [(700, 48, 333), (700, 48, 180), (1, 100, 900)])
def test_large_products_output_by_output(mg, n, k, c, dtype):
    """Every output alone has the bits it has beside the others, also where no gradient is asked for."""
    h, w, y = inputs(n, k, c, DTYPES[dtype], 42)
    h[0] *= 2.0 ** 23
    want = results(mg, h, w, y)
    for i, name in enumerate(("loss", "row_loss", "dH", "dW")):
        say(f"linear_xent large products n={n} c={c} {dtype} only {name}")
        got = (torch.full((1,), NAN, device="cuda", dtype=torch.float64), torch.full((n,), NAN, device="cuda"), matrix(n, k, h.dtype),
               matrix(k, c, torch.float32))[i]
        mg.linear_xent(h, w, y, **{name: got})
        torch.cuda.synchronize()
        assert torch.equal(got, want[i])
