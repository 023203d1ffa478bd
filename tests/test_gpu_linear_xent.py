"""The loss of a wide last layer without its logits, and its gradients, against the definition in 64 bits: sizes around
the tiles and pieces, rows without labels, scales of the operands, what is not finite, streams and graphs."""
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


def matrix(rows, cols, dtype, fill=NAN, extra=1):
    """rows x cols on a wider pitch, `fill` in the padding."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.full((rows, (cols + per - 1) // per * per + extra * per), fill, device="cuda", dtype=dtype)


def inputs(n, k, c, dtype, seed=0, spread=2.0, unlabelled=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 7 * n + 3 * k + c)
    h, w = matrix(n, k, dtype), matrix(k, c, torch.float32)
    h[:, :k] = torch.randn(n, k, device="cuda", generator=gen)
    w[:, :c] = torch.randn(k, c, device="cuda", generator=gen) * (spread / k ** 0.5)
    y = torch.randint(0, c, (n,), device="cuda", generator=gen, dtype=torch.int32)
    if unlabelled:
        off = torch.rand(n, device="cuda", generator=gen) < unlabelled
        y[off] = torch.tensor([-1, c, -2 ** 31, 2 ** 31 - 1], device="cuda", dtype=torch.int32)[
            torch.randint(0, 4, (int(off.sum()),), device="cuda", generator=gen)]
        h[off] = NAN  # what a row without a label holds does not matter
    return h[:, :k], w[:, :c], y


class Oracle:
    """The definition in 64 bits, and how far a result may be from it.

    An operand in two f16 terms is off by 2^-22 of itself (2^-11 of 2^-11), in one (bf16 features) by nothing, and the
    product of both rests, 2^-22, is left out: 3 * 2^-22 of |a| |b| per term of a sum.  The sums are fp32, at most
    three products of 16 terms to a step, each rounded or cut to 2^-23 of the running sum, which is at most the sum of
    |a| |b|, and are joined in as many further steps as there are pieces; 2^-39 of the largest values is the resolution
    of the terms.  e: that of the logits.  A row's losses are off by twice its largest e, and by a few roundings
    of numbers as large as its logits; its probabilities by as much relative to themselves, and by 2^-39."""

    def __init__(self, h, w, y, joined=64):
        n, (k, c) = h.shape[0], w.shape
        self.rows = ((y >= 0) & (y < c)).nonzero()[:, 0]
        count = self.count = self.rows.numel()
        self.losses = torch.zeros(n, device="cuda", dtype=torch.float64)
        self.dh, self.dh_off = (torch.zeros(n, k, device="cuda", dtype=torch.float64) for _ in range(2))
        self.dw, self.dw_off = (torch.zeros(k, c, device="cuda", dtype=torch.float64) for _ in range(2))
        self.losses_off = torch.zeros(n, device="cuda", dtype=torch.float64)
        one_term = h.dtype == torch.bfloat16
        wd, wa = w.double(), w.double().abs()
        steps = lambda terms: (3 + (3 * (terms // 16 + 1) + joined)) * 2.0 ** -22
        step = max(1, (1 << 26) // c)
        for b in range(0, count, step):
            r = self.rows[b:b + step]
            hd, yy = h[r].double(), y[r].long()
            at = torch.arange(r.numel(), device="cuda")
            s = hd @ wd
            e = (hd.abs() @ wa).amax(1, keepdim=True) * steps(k) + s.abs().amax(1, keepdim=True) * 2.0 ** -21 + 2.0 ** -21
            logp = torch.log_softmax(s, 1)
            self.losses[r] = -logp[at, yy]
            self.losses_off[r] = 2 * e[:, 0]
            p = logp.exp()
            g_off = p * (2 * e) + 2.0 ** -39
            p[at, yy] -= 1
            g_off += p.abs() * 2.0 ** -22
            p, g_off, a = p / count, g_off / count, p.abs() / count
            self.dh[r] = p @ wd.t().contiguous()
            self.dh_off[r] = g_off @ wa.t().contiguous() + (a @ wa.t().contiguous()) * (steps(c) + (2.0 ** -10 if one_term else 0))
            self.dw += hd.t().contiguous() @ p
            self.dw_off += hd.abs().t().contiguous() @ g_off + (hd.abs().t().contiguous() @ a) * steps(count)
        self.loss = self.losses.sum() / max(count, 1)
        self.loss_off = self.losses_off.sum() / max(count, 1)
        self.dh_off += self.dh.abs() * (2.0 ** -8 if one_term else 2.0 ** -24)

    def check(self, what, got, ref, off):
        bad = ~((got.double() - ref).abs() <= off + 1e-38)
        assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist(),
                               off[bad][:4].tolist())

    def all(self, loss, row_loss, dh, dw):
        self.check("loss", loss, self.loss.view(1), self.loss_off.view(1) + 2.0 ** -24 * self.loss.abs())
        self.check("row_loss", row_loss, self.losses, self.losses_off + 2.0 ** -24 * self.losses.abs())
        self.check("dH", dh, self.dh, self.dh_off)
        self.check("dW", dw, self.dw, self.dw_off + 2.0 ** -24 * self.dw.abs())


def outputs(h, w):
    n, (k, c) = h.shape[0], w.shape
    return (torch.full((1,), NAN, device="cuda", dtype=torch.float64), torch.full((n,), NAN, device="cuda"),
            matrix(n, k, h.dtype, 5.0), matrix(k, c, torch.float32, 5.0))


def poisoned(mg, h, c, gradients=True):
    """A workspace of the asked size that holds NaN, and what follows it."""
    need = mg.linear_xent_workspace(h.dtype, h.shape[0], h.shape[1], c, gradients)
    room = torch.full((need + 4096,), 255, device="cuda", dtype=torch.uint8)
    return room, room[:need]


SIZES = [(1, 1, 1), (1, 4, 2), (1, 128, 1000), (3, 5, 2), (127, 33, 129), (128, 128, 128), (129, 100, 300), (300, 130, 4097),
         (1000, 64, 63), (513, 257, 700), (40, 8, 70001), (64, 602, 65), (2049, 32, 47),
         (16400, 16, 4500),   # pieces of classes, the last one not whole
         (16700, 8, 8300),    # pieces of rows and of classes
         (140001, 8, 5),      # many rows of few classes
         (530001, 4, 3),      # pieces of those
         (70, 2100, 90), (33, 5000, 260),   # more features than a block keeps the scales of
         (96, 192, 1000), (200, 320, 129)]  # features in tiles of 64, and of 128


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,c", SIZES)
def test_loss_and_gradients(mg, n, k, c, dtype):
    say(f"linear_xent n={n} k={k} c={c} {dtype}")
    h, w, y = inputs(n, k, c, DTYPES[dtype])
    loss, row_loss, dh, dw = outputs(h, w)
    room, ws = poisoned(mg, h, c)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :k], dW=dw[:, :c], row_loss=row_loss, workspace=ws)
    torch.cuda.synchronize()
    Oracle(h, w, y).all(loss, row_loss, dh[:, :k], dw[:, :c])
    assert (dh[:, k:] == 5).all() and (dw[:, c:] == 5).all() and (room[ws.numel():] == 255).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,c,share", [(1000, 64, 200, 0.5), (5000, 36, 300, 0.97), (20000, 100, 129, 0.9), (130, 16, 5000, 0.3)])
def test_rows_without_a_label(mg, n, k, c, share, dtype):
    """They cost nothing and spoil nothing, whatever they hold; their gradients and losses are zero."""
    say(f"linear_xent n={n} k={k} c={c} {dtype} without a label {share}")
    h, w, y = inputs(n, k, c, DTYPES[dtype], seed=1, unlabelled=share)
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :k], dW=dw[:, :c], row_loss=row_loss)
    torch.cuda.synchronize()
    o = Oracle(h, w, y)
    assert 0 < o.count < n
    o.all(loss, row_loss, dh[:, :k], dw[:, :c])
    assert (dh[:, k:] == 5).all() and (dw[:, c:] == 5).all()


@pytest.mark.parametrize("n", [0, 1, 300])
def test_no_row_has_a_label(mg, n):
    h, w, y = inputs(n, 20, 50, torch.float32)
    y.fill_(-1)
    loss, row_loss, dh, dw = outputs(h, w)
    say(f"linear_xent without labels n={n}")
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :20], dW=dw[:, :50], row_loss=row_loss)
    torch.cuda.synchronize()
    assert loss.item() == 0 and (row_loss == 0).all() and (dh[:, :20] == 0).all() and (dw[:, :50] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_that_are_not_asked_for(mg, dtype):
    """Every output alone has the bits it has beside the others."""
    h, w, y = inputs(700, 48, 333, DTYPES[dtype], seed=3, unlabelled=0.2)
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :48], dW=dw[:, :333], row_loss=row_loss)
    for only in ("loss", "row_loss", "dH", "dW"):
        say(f"linear_xent {dtype} only {only}")
        l2, r2, h2, w2 = outputs(h, w)
        got = dict(loss=l2, row_loss=r2, dH=h2[:, :48], dW=w2[:, :333])
        mg.linear_xent(h, w, y, **{only: got[only]})
        torch.cuda.synchronize()
        assert torch.equal(got[only], dict(loss=loss, row_loss=row_loss, dH=dh[:, :48], dW=dw[:, :333])[only])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_over_the_features(mg, dtype):
    h, w, y = inputs(900, 40, 300, DTYPES[dtype], seed=4, unlabelled=0.3)
    _, _, dh, _ = outputs(h, w)
    mg.linear_xent(h, w, y, dH=dh[:, :40])
    say(f"linear_xent {dtype} dH over H")
    mg.linear_xent(h, w, y, dH=h)
    torch.cuda.synchronize()
    assert torch.equal(h, dh[:, :40])


def test_gradient_against_differences(mg):
    """Central differences of the loss over the features and weights."""
    h, w, y = inputs(6, 5, 7, torch.float32, seed=5)
    loss, _, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :5], dW=dw[:, :7])
    def value(a, b):
        return torch.nn.functional.cross_entropy(a @ b, y.long()).item()

    # truncation of the difference: step^2 / 6 of a third derivative of a few units; rounding: 2^-52 / step
    a, b, step = h.double().clone(), w.double().clone(), 1e-4
    for t, g in ((a, dh[:, :5]), (b, dw[:, :7])):
        for i in range(t.shape[0]):
            for j in range(t.shape[1]):
                keep = t[i, j].item()
                t[i, j] = keep + step
                up = value(a, b)
                t[i, j] = keep - step
                down = value(a, b)
                t[i, j] = keep
                assert abs((up - down) / (2 * step) - g[i, j].item()) < 1e-6


@pytest.mark.parametrize("spread", [1e-3, 30.0, 3000.0])
def test_flat_and_peaked(mg, spread):
    """Logits all alike, and so far apart that all but one probability is zero."""
    say(f"linear_xent spread {spread}")
    h, w, y = inputs(500, 64, 600, torch.float32, seed=6, spread=spread)
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :64], dW=dw[:, :600], row_loss=row_loss)
    torch.cuda.synchronize()
    Oracle(h, w, y).all(loss, row_loss, dh[:, :64], dw[:, :600])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scales", ["1e-18 1e18", "1e12 1e-13", "by feature", "rows of zeros"])
def test_scales(mg, scales, dtype):
    """Magnitudes far from one, in the features and, the other way round, in the weights; features whose scales differ by
    2^30 both ways; features that are zero everywhere, and weights."""
    say(f"linear_xent scales {scales} {dtype}")
    h, w, y = inputs(400, 32, 150, DTYPES[dtype], seed=8)
    if scales == "by feature":
        e = torch.exp2(torch.linspace(-30, 30, 32, device="cuda").round())
        h.mul_(e.to(h.dtype))
        w.mul_((1 / e)[:, None])
    elif scales == "rows of zeros":
        h[:, 3] = 0
        w[5] = 0
        h[:, 9], w[9] = 0, 0
    else:
        a, b = (float(s) for s in scales.split())
        h.mul_(a)
        w.mul_(b)
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :32], dW=dw[:, :150], row_loss=row_loss)
    torch.cuda.synchronize()
    Oracle(h, w, y).all(loss, row_loss, dh[:, :32], dw[:, :150])


def test_all_features_zero(mg):
    h, w, y = inputs(70, 16, 90, torch.float32)
    h.zero_()
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :16], dW=dw[:, :90], row_loss=row_loss)
    torch.cuda.synchronize()
    Oracle(h, w, y).all(loss, row_loss, dh[:, :16], dw[:, :90])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_another_magnitude(mg, dtype):
    """One row 2^14 times the others, and one weight: the others' elements then have their second terms below the smallest
    normal f16, which keep their bits.  (2^-39 of the largest in a column is below 2^-22 of the others.)"""
    say(f"linear_xent a large row {dtype}")
    h, w, y = inputs(300, 48, 200, DTYPES[dtype], seed=21)
    h[17] *= 2.0 ** 14
    w[5, 7] *= 2.0 ** 10
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :48], dW=dw[:, :200], row_loss=row_loss)
    torch.cuda.synchronize()
    Oracle(h, w, y).all(loss, row_loss, dh[:, :48], dw[:, :200])


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), NAN])
def test_not_finite(mg, value):
    """In a feature of one row: that row's loss and gradient are NaN, no other row's, and the weight gradient is."""
    say(f"linear_xent {value}")
    h, w, y = inputs(260, 24, 100, torch.float32, seed=9)
    h[133, 7] = value
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :24], dW=dw[:, :100], row_loss=row_loss)
    torch.cuda.synchronize()
    other = torch.arange(260, device="cuda") != 133
    assert loss.isnan().all() and row_loss[133].isnan() and dh[133, :24].isnan().all() and dw[:, :100].isnan().all()
    keep = h.clone()
    keep[133] = 0
    o = Oracle(keep, w, y)
    o.check("row_loss", row_loss[other], o.losses[other], o.losses_off[other] + 2.0 ** -24 * o.losses[other].abs())
    o.check("dH", dh[other, :24], o.dh[other], o.dh_off[other])


def test_same_bits_every_time(mg):
    h, w, y = inputs(3000, 96, 2000, torch.float32, seed=10, unlabelled=0.1)
    first = outputs(h, w)
    for got in (first, outputs(h, w), outputs(h, w)):
        mg.linear_xent(h, w, y, loss=got[0], dH=got[2][:, :96], dW=got[3][:, :2000], row_loss=got[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_two_streams_at_once(mg):
    a, b = inputs(2000, 64, 1500, torch.float32, seed=11), inputs(1500, 128, 900, torch.bfloat16, seed=12)
    want, got = [outputs(x[0], x[1]) for x in (a, b)], [outputs(x[0], x[1]) for x in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    call = lambda x, o, s=None: mg.linear_xent(*x, loss=o[0], dH=o[2][:, :x[0].shape[1]], dW=o[3][:, :x[1].shape[1]],
                                               row_loss=o[1], stream=s)
    for x, o in zip((a, b), want):
        call(x, o)
    torch.cuda.synchronize()
    say("linear_xent on two streams")
    for _ in range(3):
        for x, o, s in zip((a, b), got, streams):
            call(x, o, s)
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(o, w))


def test_captured_and_replayed(mg):
    """Two graphs of the same call on other inputs, replayed in turn with eager work between, after the inputs changed."""
    cases = [inputs(1200, 64, 700, torch.float32, seed=s, unlabelled=0.2) for s in (13, 14)]
    outs = [outputs(h, w) for h, w, _ in cases]
    graphs = []
    say("linear_xent captured")
    for (h, w, y), o in zip(cases, outs):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            mg.linear_xent(h, w, y, loss=o[0], dH=o[2][:, :64], dW=o[3][:, :700], row_loss=o[1])
        graphs.append(g)
    for trip in range(3):
        for (h, w, y), o, g in zip(cases, outs, graphs):
            w.mul_(1.0 + 0.25 * trip)
            y.copy_(y.roll(trip))
            h.copy_(torch.where(((y >= 0) & (y < 700))[:, None], h.nan_to_num(0.5), h))
            g.replay()
            eager = outputs(h, w)
            mg.linear_xent(h, w, y, loss=eager[0], dH=eager[2][:, :64], dW=eager[3][:, :700], row_loss=eager[1])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(o, eager))
            assert torch.isfinite(o[0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [40, 200, 700])
def test_products_below_the_smallest_float(mg, c, dtype):
    """All logits vanish, the loss is that of even odds, and the gradients are in the range of the operands."""
    say(f"linear_xent products below the smallest float c={c} {dtype}")
    h, w, y = inputs(300, 36, c, DTYPES[dtype], seed=22)
    h.mul_(2.0 ** -84)
    w.mul_(2.0 ** -66)
    loss, row_loss, dh, dw = outputs(h, w)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :36], dW=dw[:, :c], row_loss=row_loss)
    torch.cuda.synchronize()
    Oracle(h, w, y).all(loss, row_loss, dh[:, :36], dw[:, :c])
    assert (dh[:, :36] != 0).any() and (dw[:, :c] != 0).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,c,share", [(1, 64, 200, 0.0), (128, 40, 256, 0.0), (257, 96, 255, 0.3), (129, 64, 128, 0.0), (3000, 130, 47, 0.2),
                                         (20000, 128, 172, 0.9), (40001, 35, 60, 0.1), (40001, 35, 160, 0.0), (262300, 12, 150, 0.0)])
def test_few_classes(mg, n, k, c, share, dtype):
    """All classes in one tile, of 128 and of 256; gradients written straight to rows that start anywhere; pieces of rows."""
    say(f"linear_xent few classes n={n} k={k} c={c} {dtype}")
    h, w, y = inputs(n, k, c, DTYPES[dtype], seed=23, unlabelled=share)
    loss, row_loss, dh, dw = outputs(h, w)
    room, ws = poisoned(mg, h, c)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :k], dW=dw[:, :c], row_loss=row_loss, workspace=ws)
    again = outputs(h, w)
    mg.linear_xent(h, w, y, loss=again[0], row_loss=again[1])
    mg.linear_xent(h, w, y, dH=h)
    torch.cuda.synchronize()
    assert torch.equal(again[0], loss) and torch.equal(again[1], row_loss) and torch.equal(h, dh[:, :k])
    h, w, y = inputs(n, k, c, DTYPES[dtype], seed=23, unlabelled=share)
    Oracle(h, w, y).all(loss, row_loss, dh[:, :k], dw[:, :c])
    assert (dh[:, k:] == 5).all() and (dw[:, c:] == 5).all() and (room[ws.numel():] == 255).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,c,live", [(12000, 100, 9000, 1), (12000, 100, 9000, 250), (12000, 200, 9000, 3000), (20000, 40, 6000, 700),
                                        (40000, 64, 700, 40), (9000, 130, 500, 129), (17000, 24, 12000, 16500)])
def test_few_rows_of_many_have_a_label(mg, n, k, c, live, dtype):
    """The launches are made for all rows, what they do is dealt out for those with a label."""
    say(f"linear_xent {live} of n={n} k={k} c={c} {dtype}")
    h, w, y = inputs(n, k, c, DTYPES[dtype], seed=24)
    gen = torch.Generator(device="cuda").manual_seed(live)
    off = torch.randperm(n, device="cuda", generator=gen)[live:]
    y[off] = -1
    h[off] = NAN
    loss, row_loss, dh, dw = outputs(h, w)
    room, ws = poisoned(mg, h, c)
    mg.linear_xent(h, w, y, loss=loss, dH=dh[:, :k], dW=dw[:, :c], row_loss=row_loss, workspace=ws)
    torch.cuda.synchronize()
    Oracle(h, w, y).all(loss, row_loss, dh[:, :k], dw[:, :c])
    assert (dh[:, k:] == 5).all() and (dw[:, c:] == 5).all() and (room[ws.numel():] == 255).all()
