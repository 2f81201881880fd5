"""Layer normalisation and its gradients against numpy in 64 bits."""
import pytest
import torch

from tests import layer_refs as R

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def kb():
    from paper_2602_10016_amd import binding
    return binding


def both(kb, x, weight, bias, dtype, seed=5):
    D = x.shape[-1]
    y, rims = R.guarded(x.shape, dtype)
    got = kb.layer_norm_fwd(x, weight, bias, EPS, out=y)
    assert got[0] is y and R.untouched(rims)
    for name, t, (ref, bound), kind in zip(("y", "mean", "rstd"), got, R.norm_fwd(x, weight, bias, EPS), (dtype, torch.float32, torch.float32)):
        R.check(name, t, ref, bound, kind)
    dy = R.normal(x.shape, dtype, seed)
    outs = [R.guarded(s, dtype) for s in (x.shape, (D,), (D,))]
    grads = kb.layer_norm_bwd(x, weight, dy, got[1], got[2], out=[o for o, _ in outs])
    assert all(a is b for a, (b, _) in zip(grads, outs)) and all(R.untouched(r) for _, r in outs)
    for name, t, (ref, bound) in zip(("dx", "dw", "db"), grads, R.norm_bwd(x, weight, dy, got[1], got[2])):
        R.check(name, t.reshape(ref.shape), ref, bound, dtype)
    again = kb.layer_norm_bwd(x, weight, dy, got[1], got[2], want_dw=True, want_db=True)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))  # to the bit


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("rows", [1, 3, 261])
@pytest.mark.parametrize("D", [1, 2, 3, 7, 8, 9, 12, 40, 64, 100, 203, 256, 511, 512, 520, 1024, 1025, 2048, 2056, 4096, 4100, 8192, 8200, 16384])
def test_widths(kb, D, rows, dtype):
    both(kb, R.normal((rows, D), dtype, D) + 0.5, R.normal((D,), dtype, 1) + 1, R.normal((D,), dtype, 2), dtype)


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("D", [5, 96, 3000])
def test_without_weight_or_bias(kb, D, weight, bias):
    dtype = torch.bfloat16
    both(kb, R.normal((50, D), dtype, D), R.normal((D,), dtype, 1) if weight else None, R.normal((D,), dtype, 2) if bias else None, dtype)


@pytest.mark.parametrize("rows", [4000, 70_001])
def test_more_rows_than_lanes(kb, rows):
    dtype = torch.float32
    both(kb, R.normal((rows, 48), dtype, 0), R.normal((48,), dtype, 1), R.normal((48,), dtype, 2), dtype)


def test_a_large_mean_costs_no_digits(kb):
    x = R.normal((20, 1000), torch.float32, 0) + 4096
    both(kb, x, None, None, torch.float32)


def test_constant_rows(kb):
    x = torch.full((4, 100), 3.0, device="cuda")
    x[1], x[2] = 0, -1e30
    bias = R.normal((100,), torch.float32, 1)
    y, mean, rstd = kb.layer_norm_fwd(x, None, bias, EPS)
    assert torch.equal(y[:2], bias.expand(2, 100)) and torch.equal(mean[:2].cpu(), torch.tensor([3.0, 0.0]))
    R.check("rstd", rstd[:2], 1 / R.np.sqrt(R.np.full(2, float(R.np.float32(EPS)))), 3 * R.U * 316.3, torch.float32)


def test_infinities_stay_in_their_rows(kb):
    x = R.normal((6, 77), torch.bfloat16, 0)
    x[2, 5], x[4, 0] = float("nan"), float("inf")
    y, mean, rstd = kb.layer_norm_fwd(x, None, None, EPS)
    assert bool(y[[0, 1, 3, 5]].isfinite().all()) and bool(y[2].isnan().all()) and bool(y[4].isnan().any())
    dx, dw, db = kb.layer_norm_bwd(x, None, R.normal((6, 77), torch.bfloat16, 1), mean, rstd, want_dw=True)
    assert bool(dx[[0, 1, 3, 5]].isfinite().all()) and db is None


def test_shapes_and_what_is_wanted(kb):
    x, w = R.normal((3, 4, 24), torch.float32, 0), R.normal((24,), torch.float32, 1)
    y, mean, rstd = kb.layer_norm_fwd(x, w)
    assert y.shape == x.shape and mean.shape == rstd.shape == (3, 4)
    plain = kb.layer_norm_fwd(x, w, want_stats=False)
    assert torch.equal(plain[0], y) and plain[1] is None and plain[2] is None
    one = kb.layer_norm_fwd(x[1, 2], w)
    assert torch.equal(one[0], y[1, 2]) and one[1].shape == ()
    dy = R.normal(x.shape, torch.float32, 2)
    full = kb.layer_norm_bwd(x, w, dy, mean, rstd)
    for want in range(8):
        wants = dict(want_dx=bool(want & 1), want_dw=bool(want & 2), want_db=bool(want & 4))
        for g, f, on in zip(kb.layer_norm_bwd(x, w, dy, mean, rstd, **wants), full, wants.values()):
            assert g is None if not on else torch.equal(g, f)
    none = R.normal((0, 24), torch.float32, 0)
    y, mean, rstd = kb.layer_norm_fwd(none, w)
    assert y.shape == (0, 24) and mean.shape == (0,)
    dx, dw, db = kb.layer_norm_bwd(none, w, none, mean, rstd)
    assert dx.shape == (0, 24) and not dw.any() and not db.any()


def test_rows_beyond_32_bit_offsets(kb):
    rows, D = 300_000, 8192
    x = torch.zeros(rows, D, dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 131_072, 262_144, rows - 1], device="cuda")
    x[some] = R.normal((4, D), torch.bfloat16, 0)
    y, mean, rstd = kb.layer_norm_fwd(x)
    small = kb.layer_norm_fwd(x[some])
    assert torch.equal(y[some], small[0]) and torch.equal(mean[some], small[1]) and torch.equal(rstd[some], small[2])
    y[some] = 0
    assert not bool(y.any())
    dx, dw, _ = kb.layer_norm_bwd(x, None, x, mean, rstd, want_dw=True)
    small = kb.layer_norm_bwd(x[some], None, x[some], mean[some], rstd[some], want_dw=True)
    assert torch.equal(dx[some], small[0])
    dx[some] = 0
    assert not bool(dx.any())


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("D", [9, 256, 4097])
def test_tensors_that_start_anywhere(kb, D, dtype):
    """Views that begin one value into their memory: rows at any multiple of the value's size."""
    view = lambda n, seed: R.normal((n * D + 1,), dtype, seed)[1:].view(n, D)
    x, dy, w, b = view(13, 1), view(13, 2), view(1, 3)[0], view(1, 4)[0]
    y, mean, rstd = kb.layer_norm_fwd(x, w, b, EPS, out=view(13, 5))
    (ref, bound), *_ = R.norm_fwd(x, w, b, EPS)
    R.check("y", y, ref, bound, dtype)
    outs = view(13, 6), view(1, 7)[0], view(1, 8)[0]
    for name, t, (ref, bound) in zip(("dx", "dw", "db"), kb.layer_norm_bwd(x, w, dy, mean, rstd, out=outs), R.norm_bwd(x, w, dy, mean, rstd)):
        R.check(name, t, ref, bound, dtype)
