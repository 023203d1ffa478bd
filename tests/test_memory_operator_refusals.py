"""Arguments that the loss without logits and the 8-bit activations refuse, before they touch a device."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    import paper_2501_01951_amd as mg

    return mg.load_library()


A = ctypes.c_void_p(1 << 20)   # aligned, never read
ODD = ctypes.c_void_p((1 << 20) + 4)
BIG = 1 << 50
NONE = None


def xent(lib, **change):
    a = dict(dtype=0, H=A, ldh=64, W=A, ldw=128, labels=A, n=10, k=64, c=128, loss=A, row_loss=NONE, dH=NONE, ldd=0,
             dW=NONE, ldg=0, ws=A, ws_bytes=BIG, stream=NONE)
    assert set(change) <= set(a)
    a.update(change)
    return lib.mixgcn_linear_xent(*a.values())


@pytest.mark.parametrize("change,word", [
    (dict(dtype=2), b"dtype"), (dict(n=-1), b"sizes"), (dict(k=0), b"sizes"), (dict(c=0), b"sizes"), (dict(c=-5), b"sizes"),
    (dict(loss=NONE), b"nothing"), (dict(H=NONE), b"H: null"), (dict(H=ODD), b"H: not 16"), (dict(ldh=63), b"H: ld <"),
    (dict(ldh=65), b"H: ld *"), (dict(W=NONE), b"W: null"), (dict(ldw=127), b"W: ld <"), (dict(ldw=130), b"W: ld *"),
    (dict(labels=NONE), b"labels"), (dict(dH=ODD, ldd=64), b"dH: not 16"), (dict(dH=ctypes.c_void_p(1 << 21), ldd=60), b"dH: ld <"),
    (dict(dH=A, ldd=128), b"dH over H"), (dict(dW=ctypes.c_void_p(1 << 21), ldg=126), b"dW: ld <"), (dict(dW=A, ldg=128), b"dW must not"),
    (dict(ws=NONE), b"workspace"), (dict(ws=ctypes.c_void_p((1 << 20) + 16)), b"workspace"), (dict(ws_bytes=100), b"workspace smaller"),
    (dict(dtype=1, ldh=68), b"H: ld *"),
])
def test_linear_xent_refuses(lib, change, word):
    assert xent(lib, **change) == -1
    assert word in lib.mixgcn_last_error(), lib.mixgcn_last_error()


@pytest.mark.parametrize("change", [dict(n=(1 << 30) + 1), dict(k=(1 << 16) + 4, ldh=1 << 17), dict(c=(1 << 22) + 4, ldw=1 << 25)])
def test_linear_xent_beyond_its_sizes(lib, change):
    assert xent(lib, **change) == -5


def test_linear_xent_workspace_sizes(lib):
    f = lib.mixgcn_linear_xent_workspace
    for bad in ((2, 1, 1, 1, 0), (0, -1, 1, 1, 0), (0, 1, 0, 1, 0), (0, 1, 1, 0, 0), (0, (1 << 30) + 1, 1, 1, 0),
                (0, 1, (1 << 16) + 1, 1, 0), (0, 1, 1, (1 << 22) + 1, 0)):
        assert f(*bad) == -1
    assert 0 < f(0, 0, 1, 1, 0) <= f(0, 0, 1, 1, 1)
    assert f(0, 1000, 64, 500, 0) < f(0, 1000, 64, 500, 1)
    # far less than the logits and their gradient would take, and bounded however many rows there are
    for dtype, es in ((0, 4), (1, 2)):
        n, k, c = 65536, 256, 100000
        assert f(dtype, n, k, c, 1) < 0.03 * 2 * n * c * es * (2 if es == 2 else 1)
        assert f(dtype, 1 << 30, 64, 1000, 1) - 8 * (1 << 30) < 1 << 31
    # the largest sizes do not overflow
    assert f(0, 1 << 30, 1 << 16, 1 << 22, 1) > 1 << 40


def checkpoint(lib, what, **change):
    a = dict(dtype=0, X=A, ldx=64, n=10, cols=64, codes=A, ldq=64, exponents=A, lde=2)
    a.update(change)
    if what == "pack":
        return lib.mixgcn_checkpoint_pack(a["dtype"], a["X"], a["ldx"], a["n"], a["cols"], a["codes"], a["ldq"],
                                          a["exponents"], a["lde"], None)
    return lib.mixgcn_checkpoint_unpack(a["dtype"], a["codes"], a["ldq"], a["exponents"], a["lde"], a["n"], a["cols"],
                                        a["X"], a["ldx"], None)


@pytest.mark.parametrize("what", ["pack", "unpack"])
@pytest.mark.parametrize("change,word", [
    (dict(dtype=3), b"dtype"), (dict(n=-1), b"sizes"), (dict(cols=0), b"sizes"), (dict(X=NONE), b"X: null"), (dict(X=ODD), b"X: not 16"),
    (dict(ldx=60), b"X: ld <"), (dict(ldx=65), b"X: ld *"), (dict(codes=NONE), b"codes: null"), (dict(codes=ODD), b"codes: not 16"),
    (dict(ldq=48), b"codes: ld <"), (dict(ldq=72), b"codes: ld *"), (dict(exponents=NONE), b"exponents"), (dict(lde=1), b"ld_exponents"),
])
def test_checkpoint_refuses(lib, what, change, word):
    assert checkpoint(lib, what, **change) == -1
    assert word in lib.mixgcn_last_error(), lib.mixgcn_last_error()


def wgrad(lib, **change):
    a = dict(dtype=0, codes=A, ldq=64, exponents=A, lde=2, G=A, ldg=32, dW=A, ldw=32, n=10, k=64, m=32, mask=NONE, ldm=0, beta=0.0,
             ws=A, ws_bytes=BIG, stream=NONE)
    assert set(change) <= set(a)
    a.update(change)
    return lib.mixgcn_checkpoint_wgrad(*a.values())


@pytest.mark.parametrize("change,word", [
    (dict(dtype=2), b"dtype"), (dict(beta=0.5), b"beta"), (dict(beta=float("nan")), b"beta"), (dict(m=0), b"sizes"), (dict(k=0), b"sizes"),
    (dict(n=-1), b"sizes"), (dict(codes=NONE), b"codes: null"), (dict(ldq=63), b"codes: ld"), (dict(exponents=NONE), b"exponents"),
    (dict(lde=1), b"ld_exponents"), (dict(G=ODD), b"G: not 16"), (dict(ldg=31), b"G: ld <"), (dict(dW=NONE), b"dW: null"),
    (dict(ldw=28), b"dW: ld <"), (dict(mask=A, ldm=0), b"ld_mask"), (dict(ws=NONE), b"workspace"), (dict(ws=ODD), b"workspace"),
    (dict(ws_bytes=64), b"workspace smaller"),
])
def test_checkpoint_wgrad_refuses(lib, change, word):
    assert wgrad(lib, **change) == -1
    assert word in lib.mixgcn_last_error(), lib.mixgcn_last_error()


def test_checkpoint_wgrad_workspace_sizes(lib):
    f = lib.mixgcn_checkpoint_wgrad_workspace
    assert f(-1, 1, 1) == -1 and f(1, 0, 1) == -1 and f(1, 1, 0) == -1
    assert f(0, 64, 32) >= 64 * 32 * 4
    assert f(1 << 20, 256, 256) <= 1024 * 128 * 128 * 4


def test_nothing_to_do_touches_nothing(lib):
    """Without rows the pointers of the rows may be null, and a pack or unpack is done."""
    assert checkpoint(lib, "pack", n=0, X=NONE, codes=NONE, exponents=NONE) == 0
    assert checkpoint(lib, "unpack", n=0, X=NONE, codes=NONE, exponents=NONE) == 0


def test_wrappers_refuse_what_does_not_fit():
    import paper_2501_01951_amd as mg

    h, w, y = torch.zeros(4, 8), torch.zeros(8, 16), torch.zeros(4, dtype=torch.int32)
    loss = torch.zeros(1, dtype=torch.float64)
    with pytest.raises(ValueError):  # not on a GPU
        mg.linear_xent(h, w, y, loss=loss)
    for bad in (dict(W=torch.zeros(7, 16)), dict(W=w.double()), dict(labels=y.long()), dict(labels=y[:3]), dict(loss=loss.float()),
                dict(row_loss=torch.zeros(3)), dict(dH=torch.zeros(4, 9)), dict(dH=h.bfloat16()), dict(dW=torch.zeros(8, 15)),
                dict(labels=torch.zeros(8, dtype=torch.int32)[::2])):
        args = dict(H=h, W=w, labels=y, loss=loss)
        args.update(bad)
        with pytest.raises(ValueError):
            mg.linear_xent(**args)
    with pytest.raises(ValueError):
        mg.Checkpoint(torch.zeros(4, 40, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        mg.Checkpoint(torch.zeros(4, 40, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
    kept = mg.Checkpoint.empty(4, 40, "cpu")
    assert kept.shape == (4, 40) and kept.codes.stride(0) == 48
    with pytest.raises(ValueError):
        mg.checkpoint_unpack(kept, torch.zeros(4, 41))
    with pytest.raises(ValueError):
        mg.checkpoint_wgrad(kept, torch.zeros(4, 8), torch.zeros(40, 9))
    with pytest.raises(ValueError):
        mg.checkpoint_wgrad(kept, torch.zeros(4, 8), torch.zeros(40, 8), mask=torch.zeros(3, 1, dtype=torch.int32))


def test_workspaces_of_many_columns(lib):
    """A product that writes its result itself has no slabs in the workspace, many features shorten a block of rows so that no
    launch has 2^32 threads, and sizes that multiply past 64 bits are bad ones."""
    f = lib.mixgcn_linear_xent_workspace
    k, c = 1 << 12, 1 << 18
    assert f(0, 200, k, c, 1) < 1.05 * (4 * k * c) + (1 << 27) + 4 * 256 * (c + k * 2) + 8 * 256 * c // 64
    for dtype, planes in ((0, 2), (1, 1)):
        n, k = 1 << 19, 1 << 15
        assert f(dtype, n, k, 100, 1) < (1 << 17) * k * (2 * planes + 4) + (1 << 28)
    assert lib.mixgcn_checkpoint_wgrad_workspace(1, (1 << 28) + 1, 1) == -1
    assert lib.mixgcn_checkpoint_wgrad_workspace(1, 1 << 28, 0x7FFFFFFF) == (1 << 30) * 0x7FFFFFFF
