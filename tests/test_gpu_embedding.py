"""Embedding lookup and its gradient against numpy in 64 bits."""
import numpy as np
import pytest
import torch

from tests import layer_refs as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kb():
    from paper_2602_10016_amd import binding
    return binding


def make_ids(kind, n, V, seed, dtype):
    rng = np.random.default_rng(seed)
    if kind == "same":
        x = np.full(n, V - 1)
    elif kind == "padding":
        x = np.full(n, -1)
    elif kind == "each":
        x = rng.permutation(np.arange(n) % V)
    elif kind == "outside":
        x = rng.integers(-3, V + 3, n)
    else:  # few ids in a large part of the rows
        x = (rng.random(n) ** 4 * V).astype(np.int64)
        x[rng.random(n) < 0.1] = -1
    return torch.from_numpy(x.astype(np.int64)).to(dtype).cuda()


WIDTHS = [1, 2, 3, 4, 7, 8, 9, 16, 40, 100, 203, 256, 511, 512, 520, 1024, 2056, 16384]


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(kb, D, dtype):
    n, V = (37, 11) if D > 600 else (301, 57)
    ids = make_ids("outside", n, V, D, torch.int32)
    table, d_out = R.normal((V, D), dtype, D), R.normal((n, D), dtype, D + 1)
    out, rims = R.guarded((n, D), dtype)
    assert kb.embedding_fwd(table, ids, 1.7, out=out) is out and R.untouched(rims)
    R.check("out", out, *R.embedding_fwd(table, ids, 1.7), dtype)
    grad, rims = R.guarded((V, D), dtype)
    assert kb.embedding_bwd(d_out, ids, V, 1.7, out=grad) is grad and R.untouched(rims)
    R.check("d_table", grad, *R.embedding_bwd(d_out, ids, V, 1.7), dtype)


@pytest.mark.parametrize("ids_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("kind", ["same", "padding", "each", "outside", "skewed"])
@pytest.mark.parametrize("n,V", [(1, 1), (2, 1), (7, 3), (8, 2), (9, 9), (64, 64), (65, 40), (513, 1000), (4097, 3), (20_000, 70_000), (150_000, 1000),
                                 (150_000, 1_048_575), (140_000, 1_048_576), (3000, 3_000_000)])
def test_ids(kb, n, V, kind, ids_dtype):
    D, dtype = 16, torch.float32
    ids = make_ids(kind, n, V, n + V, ids_dtype)
    table, d_out = R.normal((V, D), dtype, 1), R.normal((n, D), dtype, 2)
    R.check("out", kb.embedding_fwd(table, ids), *R.embedding_fwd(table, ids, 1.0), dtype)
    out, rims = R.guarded((V, D), dtype)
    kb.embedding_bwd(d_out, ids, V, 0.5, out=out)
    assert R.untouched(rims)
    R.check("d_table", out, *R.embedding_bwd(d_out, ids, V, 0.5), dtype)
    assert torch.equal(out, kb.embedding_bwd(d_out, ids, V, 0.5))  # to the bit


@pytest.mark.parametrize("D", [203, 256, 1024])
def test_one_id_in_most_rows_of_a_large_batch(kb, D):
    n, V, dtype = 300_001, 5000, torch.bfloat16
    ids = make_ids("skewed", n, V, 3, torch.int32)
    ids[torch.arange(n, device="cuda") % 3 > 0] = 17
    d_out = R.normal((n, D), dtype, 4)
    got = kb.embedding_bwd(d_out, ids, V, 2.0)
    ref = torch.zeros(V, D, dtype=torch.float64)
    size, ok = torch.zeros(V, D, dtype=torch.float64), (ids >= 0).cpu()
    d, i = d_out.cpu().double()[ok], ids.cpu().long()[ok]
    ref.index_add_(0, i, d)
    size.index_add_(0, i, d.abs())
    count = torch.bincount(i, minlength=V)[:, None]
    R.check("d_table", got, 2 * ref.numpy(), (2 * (count + 1) * R.U * size).numpy(), dtype)
    assert torch.equal(got, kb.embedding_bwd(d_out, ids, V, 2.0))


def test_shapes_and_empty_calls(kb):
    table = R.normal((5, 12), torch.float32, 0)
    ids = torch.tensor([[0, 4, -1], [2, 2, 1]], device="cuda")
    y = kb.embedding_fwd(table, ids)
    assert y.shape == (2, 3, 12) and torch.equal(y[1, 0], table[2]) and not y[0, 2].any()
    assert kb.embedding_bwd(y, ids, 5).shape == (5, 12)
    one = kb.embedding_fwd(table, torch.tensor(3, device="cuda"))
    assert one.shape == (12,) and torch.equal(one, table[3])
    assert kb.embedding_bwd(one, torch.tensor(3, device="cuda"), 5)[3].equal(table[3])
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert kb.embedding_fwd(table, none).shape == (0, 12)
    assert not kb.embedding_bwd(R.normal((0, 12), torch.float32, 0), none, 5, out=torch.full((5, 12), 7.0, device="cuda")).any()
    assert not kb.embedding_fwd(R.normal((0, 12), torch.float32, 0), ids).any()  # an empty table: every id is outside
    assert kb.embedding_bwd(y, ids, 0).shape == (0, 12)


def test_infinities_stay_in_their_rows(kb):
    table = R.normal((6, 20), torch.bfloat16, 0)
    table[1], table[2, 3] = float("inf"), float("nan")
    ids = torch.tensor([0, 1, -1, 2, 9, 5], device="cuda")
    y = kb.embedding_fwd(table, ids, 0.5)
    assert bool(y[1].isinf().all()) and bool(y[3, 3].isnan()) and not y[2].any() and not y[4].any()
    assert bool(y[[0, 2, 4, 5]].isfinite().all())
    d_out = R.normal((6, 20), torch.bfloat16, 1)
    d_out[2], d_out[4] = float("nan"), float("inf")  # of padding
    d_out[1] = float("inf")
    g = kb.embedding_bwd(d_out, ids, 6)
    assert bool(g[1].isinf().all()) and bool(g[[0, 2, 3, 4, 5]].isfinite().all())


def test_rows_beyond_32_bit_offsets(kb):
    V, D, dtype = 300_000, 8192, torch.bfloat16  # 4.9 GB, 2.4e9 values
    table = torch.zeros(V, D, dtype=dtype, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 2, V, 131_072, 262_144, V - 1], device="cuda")
    rows = R.normal((7, D), dtype, 0)
    table[ids.clamp(max=V - 1)[:6]] = rows[:6]
    table[V - 1] = rows[0]
    y = kb.embedding_fwd(table, ids, 1.0)
    want = rows.clone()
    want[3], want[6] = 0, rows[0]
    assert torch.equal(y, want)
    g = kb.embedding_bwd(y, ids, V)
    assert torch.equal(g[V - 1], (rows[0].float() * 2).to(dtype)) and torch.equal(g[262_144], rows[5]) and torch.equal(g[V - 2], rows[2])
    g[ids[ids < V]] = 0
    assert not bool(g.any())


def test_many_rows_of_one_value(kb):
    """Values at offsets beyond 32 bits in d_out, too."""
    n, D = 1_200_000, 2048
    d_out = torch.zeros(n, D, dtype=torch.bfloat16, device="cuda")
    d_out[-1], d_out[0], d_out[1_100_000] = 3, 2, 1
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ids[-1] = 1
    g = kb.embedding_bwd(d_out, ids, 3)
    assert bool((g[0] == 3).all()) and bool((g[1] == 3).all()) and not g[2].any()
    out = kb.embedding_fwd(g, ids)
    assert bool((out == 3).all())


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("D", [8, 203, 256])
def test_tensors_that_start_anywhere(kb, D, dtype):
    """Views that begin one value into their memory: rows at any multiple of the value's size."""
    view = lambda n, seed: R.normal((n * D + 1,), dtype, seed)[1:].view(n, D)
    table, d_out, ids = view(40, 1), view(90, 2), make_ids("skewed", 91, 40, 3, torch.int32)[1:]
    out, grad = view(90, 4), view(40, 5)
    kb.embedding_fwd(table, ids, 3.0, out=out)
    kb.embedding_bwd(d_out, ids, 40, 3.0, out=grad)
    R.check("out", out, *R.embedding_fwd(table, ids, 3.0), dtype)
    R.check("d_table", grad, *R.embedding_bwd(d_out, ids, 40, 3.0), dtype)


@pytest.mark.parametrize("V,D", [(270_000, 513), (1_100_000, 128)])
def test_tables_that_are_not_set_to_zero_first(kb, V, D):
    """Gradients above 256 MB: rows without ids are found among the sorted ids."""
    n, dtype = 6000, torch.bfloat16
    ids = make_ids("each", n, V, 1, torch.int64)
    ids[::7], ids[5::11] = V - 1, -1
    d_out = R.normal((n, D), dtype, 2)
    got = kb.embedding_bwd(d_out, ids, V, 1.0, out=torch.full((V, D), float("nan"), dtype=dtype, device="cuda"))
    named = torch.unique(ids[ids >= 0])
    small = torch.searchsorted(named, ids)
    small[ids < 0] = -1
    R.check("d_table", got[named], *R.embedding_bwd(d_out, small, len(named), 1.0), dtype)
    got[named] = 0
    assert not bool(got.any())
