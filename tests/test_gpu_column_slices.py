"""The loss without logits and the weight gradient from 8 bits on the last columns of wider matrices."""
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


def last_columns(x, before):
    """x as the last columns of a matrix with `before` more in front, without columns behind it up to whole 16 bytes."""
    per = 16 // x.element_size()
    rows, cols = x.shape
    wide = torch.full((rows, before + (cols + per - 1) // per * per), 7.0, device="cuda", dtype=x.dtype)
    view = wide[:, before:before + cols]
    view.copy_(x)
    return wide, view


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,c", [(1, 4, 60), (300, 4, 60), (257, 12, 700), (2000, 36, 301), (300, 3, 5)])
def test_loss(mg, n, k, c, dtype):
    say(f"linear_xent of slices n={n} k={k} c={c} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(n + k + c)
    h = torch.randn(n, (k + 7) // 8 * 8, device="cuda", generator=gen).to(DTYPES[dtype])[:, :k]
    w = torch.randn(k, (c + 3) // 4 * 4, device="cuda", generator=gen)[:, :c]
    y = torch.randint(0, c, (n,), device="cuda", generator=gen, dtype=torch.int32)
    want, got = [(torch.zeros(1, device="cuda", dtype=torch.float64), torch.zeros(n, device="cuda")) for _ in range(2)]
    dh, dw = torch.empty_like(last_columns(h, 0)[0])[:, :k], torch.empty_like(last_columns(w, 0)[0])[:, :c]
    mg.linear_xent(h, w, y, loss=want[0], row_loss=want[1], dH=dh, dW=dw)
    for before in (8, 96):
        (_, hs), (_, ws) = last_columns(h, before), last_columns(w, before)
        (dhw, dhs), (dww, dws) = last_columns(torch.zeros_like(dh), before), last_columns(torch.zeros_like(dw), before)
        mg.linear_xent(hs, ws, y, loss=got[0], row_loss=got[1], dH=dhs, dW=dws)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(dhs, dh) and torch.equal(dws, dw)
        for wide, cols in ((dhw, k), (dww, c)):
            assert (wide[:, :before] == 7).all() and (wide[:, before + cols:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,m", [(1, 32, 4), (1000, 64, 4), (700, 100, 12), (3000, 130, 68), (500, 40, 131)])
def test_weight_gradient(mg, n, k, m, dtype):
    say(f"checkpoint_wgrad of slices n={n} k={k} m={m} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(n + k + m)
    kept = mg.checkpoint_pack(torch.randn(n, (k + 3) // 4 * 4, device="cuda", generator=gen)[:, :k])
    g = torch.randn(n, (m + 7) // 8 * 8, device="cuda", generator=gen).to(DTYPES[dtype])[:, :m]
    want = torch.empty(k, (m + 3) // 4 * 4, device="cuda")[:, :m]
    mg.checkpoint_wgrad(kept, g, want)
    for before in (8, 96):
        gs = last_columns(g, before)[1]
        wide, dw = last_columns(torch.zeros_like(want), before)
        mg.checkpoint_wgrad(kept, gs, dw)
        torch.cuda.synchronize()
        assert torch.equal(dw, want) and (wide[:, :before] == 7).all() and (wide[:, before + m:] == 7).all()
