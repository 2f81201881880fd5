"""Host-side checks of the operators in front of attention that need no GPU: exported symbols, statuses before any device is touched,
and what the Python entry points refuse."""
import os
import re

import pytest
import torch

from paper_2602_10016_amd import binding as kb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, INF = 0x1000, float("inf")
BIG = 1 << 40


def test_exports_match_header():
    header = open(os.path.join(ROOT, "include", "kunlun_layers.h")).read()
    declared = re.findall(r"^(?:int|size_t)\s+(kunlun_\w+)\(", header, flags=re.M)
    assert sorted(declared) == sorted(kb.LAYER_EXPORTS) and all(hasattr(kb.raw(), name) for name in declared)
    for name, value in (("CHANNELS", kb.MAX_CHANNELS), ("GROUPS", kb.MAX_GROUPS)):
        assert f"#define KUNLUN_MAX_{name} {value}" in header


def embedding(fwd, a=P, ids=P, out=P, n=5, rows=7, D=8, scale=1.0, id_bytes=4, dtype=0, ws=P, ws_bytes=BIG):
    if fwd:
        return kb.raw().kunlun_embedding_fwd(a, ids, out, n, rows, D, scale, id_bytes, dtype, None)
    return kb.raw().kunlun_embedding_bwd(a, ids, out, n, rows, D, scale, id_bytes, dtype, ws, ws_bytes, None)


def test_embedding_arguments():
    for fwd in (True, False):
        for bad in (dict(n=-1), dict(rows=-1), dict(D=0), dict(n=1 << 31), dict(rows=1 << 31)):
            assert embedding(fwd, **bad) == kb.ERR_SHAPE, bad
        for bad in (dict(D=kb.MAX_CHANNELS + 1), dict(scale=INF), dict(scale=float("nan")), dict(id_bytes=2), dict(dtype=2), dict(dtype=-1)):
            assert embedding(fwd, **bad) == kb.ERR_UNSUPPORTED, bad
        for bad in (dict(a=None), dict(ids=None), dict(out=None)):
            assert embedding(fwd, **bad) == kb.ERR_NULL, bad
        for bad in (dict(a=P + 1), dict(out=P + 2, dtype=1), dict(ids=P + 2), dict(ids=P + 4, id_bytes=8)):
            assert embedding(fwd, **bad) == kb.ERR_ALIGN, bad
    assert embedding(True, n=0, a=None, ids=None, out=None) == kb.OK
    assert embedding(False, rows=0, a=None, ids=None, out=None, ws=None) == kb.OK
    need = kb.embedding_bwd_workspace_bytes(5, 7, 8)
    assert need % 256 == 0 and embedding(False, ws_bytes=need - 1) == embedding(False, ws=None) == kb.ERR_WORKSPACE
    assert embedding(False, ws=P + 16) == kb.ERR_ALIGN
    assert kb.embedding_bwd_workspace_bytes(-1, 7, 8) == kb.embedding_bwd_workspace_bytes(1, 7, 0) == 0
    for dtype in (kb.BF16, kb.FP32):  # a kept workspace serves smaller calls
        sizes = [kb.embedding_bwd_workspace_bytes(n, 1000, 200, dtype) for n in (0, 1, 100, 5000, 131_072, 131_073, 300_000, 1 << 20, 3 << 20)]
        assert sizes == sorted(sizes)


def norm_fwd(x=P, weight=P, bias=P, y=P, mean=P, rstd=P, rows=3, D=8, eps=1e-5, dtype=0):
    return kb.raw().kunlun_layer_norm_fwd(x, weight, bias, y, mean, rstd, rows, D, eps, dtype, None)


def norm_bwd(x=P, weight=P, dy=P, mean=P, rstd=P, dx=P, dw=P, db=P, rows=3, D=8, dtype=0, ws=P, ws_bytes=BIG):
    return kb.raw().kunlun_layer_norm_bwd(x, weight, dy, mean, rstd, dx, dw, db, rows, D, dtype, ws, ws_bytes, None)


def test_layer_norm_arguments():
    for call in (norm_fwd, norm_bwd):
        for bad in (dict(rows=-1), dict(rows=1 << 31), dict(D=0)):
            assert call(**bad) == kb.ERR_SHAPE, bad
        for bad in (dict(D=kb.MAX_CHANNELS + 1), dict(dtype=3)):
            assert call(**bad) == kb.ERR_UNSUPPORTED, bad
        for bad in (dict(x=P + 1), dict(weight=P + 2, dtype=1), dict(mean=P + 2), dict(rstd=P + 2)):
            assert call(**bad) == kb.ERR_ALIGN, bad
    for eps in (-1e-5, INF, float("nan")):
        assert norm_fwd(eps=eps) == kb.ERR_UNSUPPORTED
    assert norm_fwd(x=None) == norm_fwd(y=None) == kb.ERR_NULL
    assert norm_fwd(bias=P + 1) == norm_fwd(y=P + 1) == kb.ERR_ALIGN
    assert norm_fwd(rows=0, x=None, y=None) == kb.OK
    for name in ("x", "dy", "mean", "rstd"):
        assert norm_bwd(**{name: None}) == kb.ERR_NULL
    for name in ("dy", "dx", "dw", "db"):
        assert norm_bwd(**{name: P + 1}) == kb.ERR_ALIGN
    need = kb.layer_norm_bwd_workspace_bytes(3, 8)
    assert norm_bwd(ws=None) == norm_bwd(ws_bytes=need - 1) == norm_bwd(ws=None, dw=None) == kb.ERR_WORKSPACE
    assert norm_bwd(ws=P + 64) == kb.ERR_ALIGN
    assert norm_bwd(dx=None, dw=None, db=None, ws=None) == norm_bwd(rows=0, dw=None, db=None, x=None, ws=None) == kb.OK
    assert kb.layer_norm_bwd_workspace_bytes(-1, 8) == kb.layer_norm_bwd_workspace_bytes(3, 0) == 0
    for D in (8, 200, 5000):
        sizes = [kb.layer_norm_bwd_workspace_bytes(rows, D) for rows in (0, 1, 7, 100, 3000, 1 << 20)]
        assert sizes == sorted(sizes)


def grouped_fwd(x=P, w=P, y=P, offsets=P, G=2, total=5, K=16, N=24, fill=0, dtype=0):
    return kb.raw().kunlun_grouped_linear_fwd(x, w, y, offsets, G, total, K, N, fill, dtype, None)


def grouped_bwd(x=P, w=P, dy=P, dx=P, dw=P, offsets=P, G=2, total=5, K=16, N=24, fill=0, dtype=0, ws=P, ws_bytes=BIG):
    return kb.raw().kunlun_grouped_linear_bwd(x, w, dy, dx, dw, offsets, G, total, K, N, fill, dtype, ws, ws_bytes, None)


def test_grouped_linear_arguments():
    for call in (grouped_fwd, grouped_bwd):
        for bad in (dict(G=0), dict(total=-1), dict(total=1 << 31), dict(K=0), dict(N=0)):
            assert call(**bad) == kb.ERR_SHAPE, bad
        for bad in (dict(G=kb.MAX_GROUPS + 1), dict(K=12), dict(N=20), dict(K=18, dtype=1), dict(N=kb.MAX_CHANNELS + 8), dict(K=kb.MAX_CHANNELS + 8),
                    dict(dtype=2)):
            assert call(**bad) == kb.ERR_UNSUPPORTED, bad
        for bad in (dict(x=P + 8), dict(w=P + 8), dict(offsets=P + 2)):
            assert call(**bad) == kb.ERR_ALIGN, bad
        assert call(offsets=None) == call(w=None) == call(x=None) == kb.ERR_NULL
    assert grouped_fwd(y=None) == kb.ERR_NULL and grouped_fwd(y=P + 8) == kb.ERR_ALIGN
    assert grouped_fwd(total=0, x=None, w=None, y=None, offsets=None) == kb.OK
    assert grouped_bwd(dy=None) == kb.ERR_NULL
    for name in ("dy", "dx", "dw"):
        assert grouped_bwd(**{name: P + 8}) == kb.ERR_ALIGN
    need = kb.grouped_linear_bwd_workspace_bytes(2, 5, 16, 24)
    assert grouped_bwd(ws=None) == grouped_bwd(ws_bytes=need - 1) == kb.ERR_WORKSPACE and grouped_bwd(ws=P + 16) == kb.ERR_ALIGN
    assert grouped_bwd(dx=None, dw=None, ws=None, offsets=None) == grouped_bwd(total=0, dw=None, offsets=None) == kb.OK
    assert kb.grouped_linear_bwd_workspace_bytes(0, 5, 16, 24) == kb.grouped_linear_bwd_workspace_bytes(2, 5, 16, 20) == 0


bf, f32 = torch.bfloat16, torch.float32
T = lambda *s, dtype=f32: torch.zeros(*s, dtype=dtype)
IDS = torch.zeros(3, dtype=torch.int64)
OFF = torch.tensor([0, 2, 5], dtype=torch.int32)

REFUSED = [
    (TypeError, lambda: kb.embedding_fwd(T(4, 8), IDS.float())),
    (TypeError, lambda: kb.embedding_fwd(T(4, 8), [0, 1])),
    (TypeError, lambda: kb.embedding_fwd(T(4, 8, dtype=torch.float16), IDS)),
    (TypeError, lambda: kb.embedding_fwd(None, IDS)),
    (ValueError, lambda: kb.embedding_fwd(T(4, 2, 8), IDS)),
    (ValueError, lambda: kb.embedding_fwd(T(8, 4).t(), IDS)),
    (ValueError, lambda: kb.embedding_fwd(T(4, 8), torch.zeros(6, dtype=torch.int64)[::2])),
    (ValueError, lambda: kb.embedding_fwd(T(4, 8), IDS, out=T(3, 9))),
    (TypeError, lambda: kb.embedding_fwd(T(4, 8), IDS, out=T(3, 8, dtype=bf))),
    (ValueError, lambda: kb.embedding_fwd(T(4, 8), IDS)),  # host tensors
    (ValueError, lambda: kb.embedding_bwd(T(3, 8), IDS, 4)),
    (ValueError, lambda: kb.embedding_bwd(T(2, 8), IDS, 4)),
    (ValueError, lambda: kb.embedding_bwd(T(3), IDS, 4)),
    (ValueError, lambda: kb.embedding_bwd(T(3, 8), IDS, -1)),
    (ValueError, lambda: kb.embedding_bwd(T(3, 8), IDS, 4, out=T(5, 8))),
    (TypeError, lambda: kb.embedding_bwd(T(3, 8), IDS, 4, workspace=T(100))),
    (TypeError, lambda: kb.layer_norm_fwd(T(3, 8, dtype=torch.float64))),
    (TypeError, lambda: kb.layer_norm_fwd(T(3, 8), T(8, dtype=bf))),
    (ValueError, lambda: kb.layer_norm_fwd(T(3, 8), T(9))),
    (ValueError, lambda: kb.layer_norm_fwd(T(3, 8), None, T(3, 8))),
    (ValueError, lambda: kb.layer_norm_fwd(torch.tensor(1.0))),
    (ValueError, lambda: kb.layer_norm_fwd(T(8, 3).t())),
    (ValueError, lambda: kb.layer_norm_fwd(T(3, 8), mean=T(8))),
    (TypeError, lambda: kb.layer_norm_fwd(T(3, 8, dtype=bf), rstd=T(3, dtype=bf))),
    (ValueError, lambda: kb.layer_norm_fwd(T(3, 8))),
    (ValueError, lambda: kb.layer_norm_bwd(T(3, 8), None, T(3, 9), T(3), T(3))),
    (TypeError, lambda: kb.layer_norm_bwd(T(3, 8), None, T(3, 8), None, T(3))),
    (ValueError, lambda: kb.layer_norm_bwd(T(3, 8), None, T(3, 8), T(3), T(4))),
    (ValueError, lambda: kb.layer_norm_bwd(T(3, 8), None, T(3, 8), T(3), T(3), out=(T(3, 8), T(3), None))),
    (ValueError, lambda: kb.layer_norm_bwd(T(3, 8), T(8), T(3, 8), T(3), T(3))),
    (ValueError, lambda: kb.grouped_linear_fwd(T(5, 8), T(2, 12, 8), OFF)),
    (ValueError, lambda: kb.grouped_linear_fwd(T(5, 2, 8), T(2, 8, 8), OFF)),
    (TypeError, lambda: kb.grouped_linear_fwd(T(5, 8), T(2, 8, 8, dtype=bf), OFF)),
    (ValueError, lambda: kb.grouped_linear_fwd(T(5, 8), T(3, 8, 8), OFF)),
    (TypeError, lambda: kb.grouped_linear_fwd(T(5, 8), T(2, 8, 8), OFF.long())),
    (ValueError, lambda: kb.grouped_linear_fwd(T(5, 8), T(2, 8, 12).transpose(1, 2).transpose(1, 2)[:, :, ::2], OFF)),
    (ValueError, lambda: kb.grouped_linear_fwd(T(5, 8), T(2, 8, 8), OFF, out=T(4, 8))),
    (ValueError, lambda: kb.grouped_linear_fwd(T(5, 8), T(2, 8, 8), OFF)),
    (ValueError, lambda: kb.grouped_linear_bwd(T(5, 8), T(2, 8, 8), T(5, 12), OFF)),
    (ValueError, lambda: kb.grouped_linear_bwd(T(5, 8), T(2, 8, 8), T(5, 8), OFF, out=(T(5, 8), T(8, 8)))),
    (ValueError, lambda: kb.grouped_linear_bwd(T(5, 8), T(2, 8, 8), T(5, 8), OFF)),
]


@pytest.mark.parametrize("number", range(len(REFUSED)))
def test_refused(number):
    error, call = REFUSED[number]
    with pytest.raises(error):
        call()


def test_another_device_than_the_current_one_is_refused(monkeypatch):
    monkeypatch.setattr(kb, "_on_device", lambda **t: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    with pytest.raises(ValueError, match="current device"):
        kb._on_current_device(None, x=T(2))
