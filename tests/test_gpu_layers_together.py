"""The operators in front of attention as a layer uses them: ids -> embedding -> layer norm -> projections by event type -> sliding-window
attention, forward and backward through autograd; captured into a graph; on another stream."""
import numpy as np
import pytest
import torch

from tests import layer_refs as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ka():
    from paper_2602_10016_amd import autograd
    return autograd


@pytest.fixture(scope="module")
def kb():
    from paper_2602_10016_amd import binding
    return binding


H, HD, D, V = 2, 32, 64, 50
LENGTHS = [[5, 0, 33], [1, 40, 17]]  # by event type, sequences packed one after another
SCALE = HD ** -0.5


def problem(dtype, seed=0):
    seqs = np.concatenate([[0], np.cumsum(sum(LENGTHS, []))])
    types = np.concatenate([[0], np.cumsum([sum(x) for x in LENGTHS])])
    off = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    n = int(seqs[-1])
    gen = torch.Generator().manual_seed(seed)
    ids = torch.randint(-1, V, (n,), generator=gen).cuda()
    return dict(ids=ids, sequences=off(seqs), types=off(types), table=R.normal((V, D), dtype, seed), weight=R.normal((D,), dtype, seed + 1, 0.2) + 1,
                bias=R.normal((D,), dtype, seed + 2, 0.2), w=R.normal((2, D, 3 * H * HD), dtype, seed + 3, D ** -0.5), d_o=R.normal((n, H, HD), dtype, seed + 4))


LEAVES = ["table", "weight", "bias", "w"]


def forward(ka, p):
    x = ka.embedding(p["table"], p["ids"], 8.0)
    qkv = ka.grouped_linear(ka.layer_norm(x, p["weight"], p["bias"]), p["w"], p["types"])
    q, k, v = (t.reshape(-1, H, HD).contiguous() for t in qkv.split(H * HD, dim=1))
    return ka.sliding_window_attention(q, k, v, p["sequences"], 9, 0, SCALE, max_len=40)


def plain(p):
    """The same in the type of p's tensors by torch on the host."""
    ids = p["ids"].cpu()
    x = p["table"][ids.clamp(min=0)] * 8.0 * (ids >= 0)[:, None]
    x = torch.nn.functional.layer_norm(x, (D,), p["weight"], p["bias"], 1e-5)
    types, seqs = p["types"].tolist(), p["sequences"].tolist()
    qkv = torch.cat([x[types[g]:types[g + 1]] @ p["w"][g] for g in range(2)])
    q, k, v = (t.reshape(-1, H, HD) for t in qkv.split(H * HD, dim=1))
    out = []
    for lo, hi in zip(seqs, seqs[1:]):
        t = torch.arange(hi - lo)
        seen = (t[None] <= t[:, None]) & (t[None] >= t[:, None] - 9)
        s = torch.einsum("qhd,khd->hqk", q[lo:hi], k[lo:hi]) * SCALE
        out.append(torch.einsum("hqk,khd->qhd", s.masked_fill(~seen, float("-inf")).softmax(-1), v[lo:hi]))
    return torch.cat(out)


def gradients(f, p, leaves):
    out = f(p)
    return [out.detach(), *torch.autograd.grad(out, [p[k] for k in leaves], p["d_o"])]


@pytest.mark.parametrize("dtype", R.DTYPES)
def test_forward_and_gradients_of_a_layer(ka, dtype):
    """fp32: against 64 bits, within 100 roundings of the largest value of each result (the longest path: five operators forward and five
    back, sums of at most 96 terms of either sign).  bf16: five roundings to bf16 forward and five back, each half a step of the
    largest value, and twice that for what products amplify."""
    p = problem(dtype)
    ref = {k: v.cpu().double().requires_grad_(k in LEAVES) if v.is_floating_point() else v for k, v in p.items()}
    for k in LEAVES:
        p[k].requires_grad_(True)
    got, want = gradients(lambda q: forward(ka, q), p, LEAVES), gradients(plain, ref, LEAVES)
    for name, g, w in zip(["out"] + LEAVES, got, want):
        limit = (100 * R.U if dtype == torch.float32 else 20 * R.HALF_STEP[dtype]) * w.abs().max()
        assert (g.cpu().double() - w).abs().max() <= limit, name


def test_gradients_against_differences(ka):
    """Directional derivatives in fp32 of <out, d_o>: central differences with step h have error h^2 from curvature and rounding / h."""
    p = problem(torch.float32, 3)
    leaves = LEAVES
    for k in leaves:
        p[k].requires_grad_(True)
    grads = gradients(lambda q: forward(ka, q), p, leaves)[1:]
    for name, grad in zip(leaves, grads):
        along = R.normal(p[name].shape, torch.float32, 11)
        along /= along.norm()
        h = 1e-2
        values = []
        with torch.no_grad():
            for sign in (1, -1):
                q = dict(p)
                q[name] = p[name] + sign * h * along
                values.append((forward(ka, q).double() * p["d_o"].double()).sum())
        slope, want = float((values[0] - values[1]) / (2 * h)), float((grad.double() * along.double()).sum())
        # value: 96 rows x 64 outputs of size about 1, errors of 100 roundings adding like a random walk, over 2 h; curvature: h^2 of the gradient's size
        noise = 100 * R.U * (96 * 64) ** 0.5 / h
        assert abs(slope - want) <= noise + 20 * h * h * float(grad.norm()), name


def parts(kb, p):
    x = kb.embedding_fwd(p["table"], p["ids"], 8.0)
    y, mean, rstd = kb.layer_norm_fwd(x, p["weight"], p["bias"])
    z = kb.grouped_linear_fwd(y, p["w"], p["types"])
    dy, dw = kb.grouped_linear_bwd(y, p["w"], z, p["types"])
    dx, dweight, dbias = kb.layer_norm_bwd(x, p["weight"], dy, mean, rstd)
    return [x, y, mean, rstd, z, dy, dw, dx, dweight, dbias, kb.embedding_bwd(dx, p["ids"], V, 8.0)]


@pytest.mark.parametrize("dtype", R.DTYPES)
def test_captured_and_replayed(kb, dtype):
    p, other = problem(dtype, 1), problem(dtype, 2)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        parts(kb, p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = parts(kb, p)
    original = {k: v.clone() for k, v in p.items()}
    for turn in range(4):
        for k in p:
            p[k].copy_(other[k] if turn % 2 else original[k])
        eager = parts(kb, p)
        torch.cuda.synchronize()
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), turn


class PythonOnly:
    def __getattr__(self, name):
        return lambda *args: None


@pytest.mark.parametrize("native", [True, False])
def test_on_another_stream(kb, monkeypatch, native):
    """The workspaces of calls on a busy stream are not handed out again before the stream has used them."""
    if not native:
        monkeypatch.setattr(kb, "_native", PythonOnly())
    p = problem(torch.bfloat16, 5)
    want = parts(kb, p)
    x, y, mean, rstd, z, dy, dw, dx, *_ = want
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)
    calls = [(lambda: kb.grouped_linear_bwd(y, p["w"], z, p["types"], stream=stream)[1], dw),
             (lambda: kb.layer_norm_bwd(x, p["weight"], dy, mean, rstd, stream=stream)[1], want[8]),
             (lambda: kb.embedding_bwd(dx, p["ids"], V, 8.0, stream=stream), want[10])]
    got, fills = [], []
    for call, _ in calls:
        got.append(call())
        fills += [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in (256, 4096, 65536, 1 << 20)]
    assert not stream.query(), "the stream was to be busy still"
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, (_, w) in zip(got, calls))


def test_native_and_python_give_the_same(kb, monkeypatch):
    p, native, taken = problem(torch.float32, 6), kb._native, []

    class Recorder:
        def __getattr__(self, name):
            def call(*args):
                done = getattr(native, name)(*args)
                assert done is not None, name
                taken.append(name)
                return done
            return call

    monkeypatch.setattr(kb, "_native", Recorder())
    a = parts(kb, p)
    assert len(set(taken)) == 6
    monkeypatch.setattr(kb, "_native", PythonOnly())
    assert all(torch.equal(x, y) for x, y in zip(a, parts(kb, p)))


def test_frozen_leaves_get_no_gradient(ka):
    p = problem(torch.float32, 7)
    p["w"].requires_grad_(True)
    forward(ka, p).backward(p["d_o"])
    assert p["w"].grad is not None and p["table"].grad is None
    q = problem(torch.float32, 7)
    q["bias"].requires_grad_(True)
    y = ka.layer_norm(q["table"], q["weight"], q["bias"])
    y.sum().backward()
    assert torch.allclose(q["bias"].grad, torch.full((D,), float(V), device="cuda"))


def test_wrong_offsets_are_found_where_they_are_looked_for(kb):
    x, w = R.normal((8, 16), torch.float32, 0), R.normal((2, 16, 8), torch.float32, 1)
    off = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    kb.verify_offsets(True)
    try:
        kb.grouped_linear_fwd(x, w, off(0, 3, 8))
        kb.grouped_linear_fwd(x, w, off(0, 3, 6))
        for bad in (off(0, 5, 4), off(1, 3, 8), off(0, 3, 9)):
            with pytest.raises(ValueError):
                kb.grouped_linear_fwd(x, w, bad)
            with pytest.raises(ValueError):
                kb.grouped_linear_bwd(x, w, x[:, :8].contiguous(), bad)
    finally:
        kb.verify_offsets(False)


def test_two_streams_at_once(kb):
    """Calls of two streams with workspaces of their own do not touch each other."""
    big = lambda seed: dict(problem(torch.bfloat16, seed), ids=torch.randint(-1, V, (96,), device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
    a, b = big(8), big(9)
    want = parts(kb, a), parts(kb, b)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [[], []]
    for _ in range(20):
        for k, (s, p) in enumerate(zip(streams, (a, b))):
            with torch.cuda.stream(s):
                got[k].append(parts(kb, p))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(x, y) for run in got[k] for x, y in zip(run, want[k]))
