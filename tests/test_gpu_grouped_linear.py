"""Linear maps per group of rows against numpy in 64 bits."""
import numpy as np
import pytest
import torch

from tests import layer_refs as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kb():
    from paper_2602_10016_amd import binding
    return binding


def offsets_of(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")


def both(kb, sizes, K, N, dtype, rest=0):
    """Forward and gradients; `rest` rows behind the last group hold NaN and are left alone."""
    G, n = len(sizes), int(sum(sizes))
    off = offsets_of(sizes)
    x, w, dy = R.normal((n + rest, K), dtype, K), R.normal((G, K, N), dtype, N, K ** -0.5), R.normal((n + rest, N), dtype, G)
    x[n:], dy[n:] = float("nan"), float("nan")
    y, rims = R.guarded((n + rest, N), dtype)
    assert kb.grouped_linear_fwd(x, w, off, out=y) is y and R.untouched(rims) and bool(y[n:].isnan().all())
    R.check("y", y[:n], *R.grouped_fwd(x[:n], w, off), dtype)
    (dx, rx), (dw, rw) = R.guarded(x.shape, dtype), R.guarded(w.shape, dtype)
    got = kb.grouped_linear_bwd(x, w, dy, off, out=(dx, dw))
    assert got[0] is dx and got[1] is dw and R.untouched(rx) and R.untouched(rw) and bool(dx[n:].isnan().all())
    ref_x, ref_w = R.grouped_bwd(x[:n], w, dy[:n], off)
    R.check("dx", dx[:n], *ref_x, dtype)
    R.check("dw", dw, *ref_w, dtype)
    y2, (dx2, dw2) = kb.grouped_linear_fwd(x, w, off), kb.grouped_linear_bwd(x, w, dy, off)
    assert torch.equal(y2[:n], y[:n]) and torch.equal(dx2[:n], dx[:n]) and torch.equal(dw2, dw)  # to the bit
    assert not y2[n:].any() and not dx2[n:].any()


SIZES = {"one_row": [1], "one_group": [300], "empty_between": [0, 5, 0, 0, 130, 0], "single_rows": [1] * 9, "all_empty": [0, 0, 0],
         "mixed": [3, 64, 1, 257, 0, 128, 31], "many": [i % 7 for i in range(150)]}


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("K,N", [(8, 8), (64, 64), (24, 200), (256, 264), (136, 72)])
@pytest.mark.parametrize("sizes", SIZES)
def test_groups(kb, sizes, K, N, dtype):
    both(kb, SIZES[sizes], K, N, dtype, rest=3 if K == 24 else 0)


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("K,N", [(1024, 512), (512, 1032), (2056, 40), (40, 2056), (328, 328)])
def test_wide(kb, K, N, dtype):
    both(kb, [200, 0, 33, 513], K, N, dtype, rest=70)


@pytest.mark.parametrize("K,N", [(4, 4), (12, 20), (196, 100)])
def test_single_precision_in_fours(kb, K, N):
    both(kb, [7, 0, 70, 129], K, N, torch.float32, rest=1)


@pytest.mark.parametrize("dtype", R.DTYPES)
def test_long_groups(kb, dtype):
    both(kb, [9000, 1, 12_345, 0, 77], 96, 64, dtype, rest=9)


def test_more_groups_than_a_wave(kb):
    both(kb, [(i * 37) % 11 for i in range(4096)], 16, 8, torch.float32)


def test_infinities_stay_in_their_group(kb):
    sizes, K, N, dtype = [40, 70, 30], 72, 136, torch.bfloat16
    off = offsets_of(sizes)
    x, w, dy = R.normal((140, K), dtype, 0), R.normal((3, K, N), dtype, 1), R.normal((140, N), dtype, 2)
    clean = kb.grouped_linear_fwd(x, w, off), *kb.grouped_linear_bwd(x, w, dy, off)
    x[40:110], dy[40:110], w[1] = float("nan"), float("inf"), float("nan")
    y, dx, dw = kb.grouped_linear_fwd(x, w, off), *kb.grouped_linear_bwd(x, w, dy, off)
    keep = list(range(40)) + list(range(110, 140))
    assert torch.equal(y[keep], clean[0][keep]) and torch.equal(dx[keep], clean[1][keep]) and torch.equal(dw[[0, 2]], clean[2][[0, 2]])
    assert bool(y[40:110].isnan().all()) and bool(dw[1].isnan().all())


def test_infinities_stay_in_their_row_and_column(kb):
    K, N, dtype = 40, 88, torch.bfloat16  # a last tile that is partly outside both ways
    off = offsets_of([50])
    x, w, dy = R.normal((50, K), dtype, 0), R.normal((1, K, N), dtype, 1), R.normal((50, N), dtype, 2)
    x[7, 39], dy[9, 87] = float("inf"), float("inf")
    y, (dx, dw) = kb.grouped_linear_fwd(x, w, off), kb.grouped_linear_bwd(x, w, dy, off)
    rows = torch.arange(50, device="cuda")
    assert bool(y[rows != 7].isfinite().all()) and not bool(y[7].isfinite().any())
    assert bool(dx[rows != 9].isfinite().all()) and not bool(dx[9].isfinite().any())
    assert bool(dw[0, :39, :87].isfinite().all()) and not bool(dw[0, 39].isfinite().any()) and not bool(dw[0, :, 87].isfinite().any())


def test_empty_calls_and_what_is_wanted(kb):
    w, off = R.normal((3, 16, 24), torch.float32, 0), torch.zeros(4, dtype=torch.int32, device="cuda")
    x, dy = R.normal((0, 16), torch.float32, 0), R.normal((0, 24), torch.float32, 0)
    assert kb.grouped_linear_fwd(x, w, off).shape == (0, 24)
    dx, dw = kb.grouped_linear_bwd(x, w, dy, off)
    assert dx.shape == (0, 16) and dw.shape == w.shape and not dw.any()
    x, dy, off = R.normal((10, 16), torch.float32, 1), R.normal((10, 24), torch.float32, 2), offsets_of([4, 0, 6])
    full = kb.grouped_linear_bwd(x, w, dy, off)
    assert torch.equal(kb.grouped_linear_bwd(x, w, dy, off, want_dw=False)[0], full[0])
    dx, dw = kb.grouped_linear_bwd(x, w, dy, off, want_dx=False)
    assert dx is None and torch.equal(dw, full[1])
    assert kb.grouped_linear_bwd(x, w, dy, off, want_dx=False, want_dw=False) == (None, None)


def test_rows_and_weights_beyond_32_bit_offsets(kb):
    n, K, N, dtype = 300_000, 8192, 8, torch.bfloat16  # x: 4.9 GB
    x = torch.zeros(n, K, dtype=dtype, device="cuda")
    x[-5:] = R.normal((5, K), dtype, 0)
    w = R.normal((2, K, N), dtype, 1, K ** -0.5)
    off = offsets_of([n - 3, 3])
    y = kb.grouped_linear_fwd(x, w, off)
    small = offsets_of([2, 3])
    R.check("y", y[-5:], *R.grouped_fwd(x[-5:], w, small), dtype)
    assert not bool(y[:-5].any())
    dy = torch.zeros(n, N, dtype=dtype, device="cuda")
    dy[-5:] = R.normal((5, N), dtype, 2)
    dx, dw = kb.grouped_linear_bwd(x, w, dy, off)
    ref_x, ref_w = R.grouped_bwd(x[-5:], w, dy[-5:], small)
    R.check("dx", dx[-5:], *ref_x, dtype)
    R.check("dw", dw, *ref_w, dtype)
    assert not bool(dx[:-5].any())
    del x, dx
    w = torch.zeros(40, 8192, 8192, dtype=dtype, device="cuda")  # 2.7e9 values
    w[39] = R.normal((8192, 8192), dtype, 3, 8192 ** -0.5)
    x, dy, off = R.normal((3, 8192), dtype, 4), R.normal((3, 8192), dtype, 5), offsets_of([0] * 38 + [1, 2])
    y, (dx, dw) = kb.grouped_linear_fwd(x, w, off), kb.grouped_linear_bwd(x, w, dy, off)
    small = offsets_of([1, 2])
    ref = R.grouped_bwd(x, w[38:], dy, small)
    R.check("y", y, *R.grouped_fwd(x, w[38:], small), dtype)
    R.check("dx", dx, *ref[0], dtype)
    R.check("dw", dw[38:], *ref[1], dtype)
    assert not bool(dw[:38].any())


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("sizes,K,N", [([9000, 3, 0, 11_000, 700], 1000, 1032), ([20_000, 300], 264, 1000), ([70_000, 0, 513], 72, 520), ([33, 66_000], 256, 256),
                                       ([5000] * 8 + [17] * 8, 136, 392)])
def test_large(kb, sizes, K, N, dtype):
    """Against torch in 64 bits: the bounds of layer_refs with the magnitudes of a row's and a column's norms (Cauchy-Schwarz)."""
    n, rest = sum(sizes), 100
    off = offsets_of(sizes)
    x, w, dy = R.normal((n + rest, K), dtype, 1), R.normal((len(sizes), K, N), dtype, 2, K ** -0.5), R.normal((n + rest, N), dtype, 3)
    x[n:], dy[n:] = float("nan"), float("nan")
    (y, ry), (dx, rx), (dw, rw) = R.guarded((n + rest, N), dtype), R.guarded(x.shape, dtype), R.guarded(w.shape, dtype)
    kb.grouped_linear_fwd(x, w, off, out=y)
    kb.grouped_linear_bwd(x, w, dy, off, out=(dx, dw))
    assert R.untouched(ry) and R.untouched(rx) and R.untouched(rw) and bool(y[n:].isnan().all()) and bool(dx[n:].isnan().all())
    assert not kb.grouped_linear_fwd(x, w, off)[n:].any() and torch.equal(kb.grouped_linear_bwd(x, w, dy, off)[1], dw)
    for g, (a, b) in enumerate(zip(off.tolist(), off.tolist()[1:])):
        for got, left, right in ((y[a:b], x[a:b], w[g]), (dx[a:b], dy[a:b], w[g].t().contiguous()), (dw[g], x[a:b].t().contiguous(), dy[a:b])):
            left, right = left.double(), right.double()
            ref = left @ right
            bound = (left.shape[1] + 1) * R.U * left.norm(dim=1, keepdim=True) * right.norm(dim=0)
            limit = 1.01 * (bound + R.HALF_STEP[dtype] * (ref.abs() + bound)) + 1e-37
            assert bool(((got.double() - ref).abs() <= limit).all()), g
