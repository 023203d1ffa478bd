"""Labels that are not a class, in the loss of given logits: nothing is read for them."""
import pytest

from parity import say

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    import paper_2501_01951_amd as m

    m.load_library()
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c,pitch", [(3, 8), (8, 8), (47, 64), (50, 57), (64, 65), (100, 128), (172, 176), (173, 177), (700, 704)])
def test_labels_that_are_not_a_class(mg, c, pitch, dtype):
    """The loss is NaN; every other row's gradient is what it was, and such a row's is that of softmax alone."""
    say(f"softmax_xent labels out of range c={c} {dtype}")
    n = 600
    if pitch * torch.empty(0, dtype=dtype).element_size() % 16:
        pitch = (pitch + 7) // 8 * 8
    gen = torch.Generator(device="cuda").manual_seed(c)
    x = torch.randn(n, pitch, device="cuda", generator=gen).to(dtype)[:, :c]
    y = torch.randint(0, c, (n,), device="cuda", generator=gen, dtype=torch.int32)
    clean, got = torch.zeros(n, pitch, device="cuda", dtype=dtype)[:, :c], torch.zeros(n, pitch, device="cuda", dtype=dtype)[:, :c]
    loss = torch.zeros(1, device="cuda", dtype=torch.float64)
    mg.softmax_xent(x, y, clean, loss)
    assert torch.isfinite(loss).all()
    bad = torch.zeros(n, device="cuda", dtype=torch.bool)
    for r, v in ((0, -1), (1, c), (63, -2 ** 31), (64, 2 ** 31 - 1), (n - 1, c + 5), (300, -7)):
        y[r], bad[r] = v, True
    mg.softmax_xent(x, y, got, loss)
    torch.cuda.synchronize()
    assert loss.isnan().all() and torch.equal(got[~bad], clean[~bad])
    want = torch.softmax(x[bad].double(), 1) / n
    # fp32, in units of 2^-24 and relative, as errors of an exponent are: the sum of up to 11 exponentials a lane and 6 exchanges 17, the
    # logarithm, between 4 and 8, rounded 4, the difference from it, below 16, rounded 8, two expf and the products 7
    assert ((got[bad].double() - want).abs() <= want * (2.0 ** -8 if dtype == torch.bfloat16 else 36 * 2.0 ** -24)).all()
