"""Activations next to the largest float in 8 bits: what is read back is finite and as near as anywhere; and slabs of thousands of
rows in the weight gradient."""
import pytest

from parity import say

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

MOST = torch.finfo(torch.bfloat16).max  # 63.75 * 2^122
TOPS = [MOST, torch.finfo(torch.float32).max, 127.4 * 2.0 ** 121, 127.5 * 2.0 ** 121, 127.75 * 2.0 ** 121, 2.0 ** 127, 63.25 * 2.0 ** 122]


@pytest.fixture(scope="module")
def mg():
    import paper_2501_01951_amd as m

    m.load_library()
    return m


def features(dtype):
    """Rows of 70 columns with a largest magnitude next to the largest float in the first or the last group."""
    x = torch.zeros(2 * len(TOPS), 72, device="cuda", dtype=torch.float32)[:, :70]
    for i, t in enumerate(TOPS):
        x[2 * i, 3], x[2 * i + 1, 66] = t, -t
        x[2 * i, 4:32] = torch.arange(28, device="cuda") * (t / 64)
        x[2 * i + 1, 64:66] = torch.tensor([0.5, -0.7], device="cuda") * t
        x[2 * i + 1, :64] = torch.linspace(-3, 3, 64, device="cuda")
    out = torch.zeros(x.shape[0], 72, device="cuda", dtype=dtype)[:, :70]
    out.copy_(x.clamp(-MOST, MOST) if dtype == torch.bfloat16 else x)
    return out


def steps(kept):
    return torch.exp2(kept.exponents.double() - 133).repeat_interleave(32, 1)[:, :kept.codes.shape[1]]


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_read_back(mg, dtype, out):
    say(f"checkpoint next to the largest float {dtype} {out}")
    x = features(dtype)
    assert x.isfinite().all()
    kept = mg.checkpoint_pack(x)
    back = torch.zeros(x.shape[0], 72, device="cuda", dtype=out)[:, :70]
    mg.checkpoint_unpack(kept, back)
    torch.cuda.synchronize()
    assert (kept.exponents == 255).any() and back.isfinite().all()
    assert ((back.double() - x.double()).abs() <= steps(kept) / 2).all()
    # a number past the largest finite bf16 one comes back as that
    want = (kept.codes.double() * steps(kept)).clamp(-MOST, MOST)
    assert torch.equal(back.double(), want)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weight_gradient(mg, dtype, masked):
    """With gradients around 2^-100 the products are ordinary numbers; the sums are fp32, of terms cut to 2^-23."""
    say(f"checkpoint_wgrad next to the largest float {dtype} masked={masked}")
    x = features(torch.float32)
    kept = mg.checkpoint_pack(x)
    n, m = x.shape[0], 40
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = (torch.randn(n, m, device="cuda", generator=gen) * 2.0 ** -100).to(dtype)
    mask, gd = None, g.double()
    if masked:
        mask = torch.randint(-2 ** 31, 2 ** 31, (n, 2), device="cuda", generator=gen).int()
        j = torch.arange(m, device="cuda")
        gd = gd * ((mask[:, j // 32] >> (j % 32).int()) & 1)
    dw = torch.empty(70, m, device="cuda")
    mg.checkpoint_wgrad(kept, g, dw, mask=mask)
    torch.cuda.synchronize()
    z = (kept.codes.double() * steps(kept)).clamp(-MOST, MOST).t().contiguous()
    assert ((dw.double() - z @ gd).abs() <= (z.abs() @ gd.abs()) * 12 * 2.0 ** -23).all()


def test_what_is_not_finite_beside_them(mg):
    """The code of what is not finite in a group of the largest step is still one, and infinite gradients are what they are."""
    say("checkpoint next to the largest float, not finite")
    x = features(torch.float32)
    x[0, 10], x[5, 66] = float("inf"), float("nan")
    kept = mg.checkpoint_pack(x)
    back = torch.zeros(x.shape[0], 72, device="cuda")[:, :70]
    mg.checkpoint_unpack(kept, back)
    g = torch.ones(x.shape[0], 8, device="cuda") * 2.0 ** -100
    g[2, 3] = float("inf")
    dw = torch.empty(70, 8, device="cuda")
    mg.checkpoint_wgrad(kept, g, dw)
    torch.cuda.synchronize()
    assert torch.equal(back.isnan(), ~x.isfinite()) and not back.isinf().any()
    assert dw[10].isnan().all() and dw[66].isnan().all()
    col = back[2].clone()
    want = torch.where(col > 0, float("inf"), torch.where(col < 0, -float("inf"), float("nan")))
    want[10], want[66] = float("nan"), float("nan")
    assert torch.equal(dw[:, 3].nan_to_num(nan=1.0), want.nan_to_num(nan=1.0))


@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,k,m", [(1000003, 40, 24), (300001, 300, 130), (700001, 256, 96)])
def test_slabs_of_many_rows(mg, n, k, m, dtype, masked):
    """Workgroups that walk 590 to 2200 rows, and a last one of less.  A slab's sum of r rows is off by 2^-23 of
    the sum of its |a| |b| per step of 16 rows (three products to a step of fp32 gradients); slabs are joined in 64 bits."""
    say(f"checkpoint_wgrad long slabs n={n} k={k} m={m} {dtype} masked={masked}")
    gen = torch.Generator(device="cuda").manual_seed(n + k)
    codes = torch.randint(-127, 128, (n, (k + 15) // 16 * 16), device="cuda", generator=gen, dtype=torch.int8)[:, :k]
    exps = torch.randint(120, 136, (n, (k + 31) // 32), device="cuda", generator=gen, dtype=torch.uint8)
    g = torch.randn(n, (m + 7) // 8 * 8, device="cuda", generator=gen).to(dtype)[:, :m]
    mask = torch.randint(-2 ** 31, 2 ** 31, (n, (m + 31) // 32), device="cuda", generator=gen).int() if masked else None
    kept = mg.Checkpoint(codes, exps)
    dw = torch.empty(k, (m + 3) // 4 * 4, device="cuda")[:, :m]
    mg.checkpoint_wgrad(kept, g, dw, mask=mask)
    torch.cuda.synchronize()
    ref, mag = (torch.zeros(k, m, device="cuda", dtype=torch.float64) for _ in range(2))
    j = torch.arange(m, device="cuda")
    for r in range(0, n, 65536):
        part = mg.Checkpoint(codes[r:r + 65536], exps[r:r + 65536])
        z = (part.codes.double() * steps(part)).t().contiguous()
        u = g[r:r + 65536].double()
        if masked:
            u = u * ((mask[r:r + 65536][:, j // 32] >> (j % 32).int()) & 1)
        ref += z @ u
        mag += z.abs() @ u.abs()
    # a slab's sum of |a| |b| is its share of them all, within a factor of two
    most = 2400
    off = mag * ((3 if dtype == torch.float32 else 1) * (most // 16 + 2) * 2.0 ** -23) + ref.abs() * 2.0 ** -24
    assert ((dw.double() - ref).abs() <= off).all()
