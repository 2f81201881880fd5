"""The native marshalling of the operators in front of attention on the CPU: the module built for host tensors in front of stubs that note
their arguments (as tests/test_native_call_cpu.py does for attention)."""
import ctypes
import importlib.machinery
import importlib.util
import os
import re
import subprocess
import types

import pytest
import torch

from paper_2602_10016_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ENTRIES = ["embedding_fwd", "embedding_bwd", "layer_norm_fwd", "layer_norm_bwd", "grouped_linear_fwd", "grouped_linear_bwd"]
ATTENTION = ["gdpa_fwd", "gdpa_bwd", "seed_attn_fwd", "seed_attn_bwd", "swa_fwd", "swa_bwd", "sumkron_fwd", "sumkron_bwd"]
V, D, G, K, N, ROWS = 9, 12, 2, 16, 24, 6


def signature(name):
    header = open(os.path.join(ROOT, "include", "kunlun_layers.h")).read()
    return [p.replace("\n", " ").strip() for p in re.search(rf"^int kunlun_{name}\(([^)]*)\);", header, flags=re.M).group(1).split(",")]


class Stub:
    def __init__(self, folder):
        source, library, module = (os.path.join(folder, f) for f in ("stub.c", "libkunlun_layers_stub.so", "_torch_call.so"))
        code = ['#include "kunlun_layers.h"', "#include <stdio.h>", "char noted[4096]; int calls, status;",
                "size_t kunlun_embedding_bwd_workspace_bytes(int64_t n, int64_t rows, int D, int dtype) { return 1000; }",
                "size_t kunlun_layer_norm_bwd_workspace_bytes(int64_t rows, int D, int dtype) { return 2000; }",
                "size_t kunlun_grouped_linear_bwd_workspace_bytes(int G, int64_t total, int K, int N, int dtype) { return 3000; }"]
        for name in ENTRIES:
            formats, values = [], []
            for arg in signature(name):
                kind, var = arg.rsplit(" ", 1)
                var = var.lstrip("*")
                formats.append("%p" if "*" in arg else {"float": "%.9g"}.get(kind, "%lld"))
                values.append(f"(void*){var}" if "*" in arg else f"(double){var}" if kind == "float" else f"(long long){var}")
            code.append(f'int kunlun_{name}({", ".join(signature(name))}) {{ ++calls; snprintf(noted, sizeof noted, "{" ".join(formats)}", '
                        f'{", ".join(values)}); return status; }}')
        with open(source, "w") as f:
            f.write("\n".join(code))
        # the attention entry points, which the module needs to load
        more = os.path.join(folder, "more.c")
        with open(more, "w") as f:
            f.write("\n".join([f"int kunlun_{n}() {{ return -9; }}" for n in ATTENTION] +
                              [f"unsigned long kunlun_{n}() {{ return 0; }}" for n in ("workspace_bytes", "sumkron_batch_bytes", "sumkron_bwd_workspace_bytes")]))
        subprocess.run(["gcc", "-shared", "-fPIC", f"-I{ROOT}/include", source, more, "-o", library], check=True)
        build._build_torch_call(out=module, library=library, extra=["-O0", "-DKUNLUN_CALL_DEVICE=CPU"])
        loader = importlib.machinery.ExtensionFileLoader("_torch_call", module)
        self.native = importlib.util.module_from_spec(importlib.util.spec_from_loader("_torch_call", loader))
        self.lib = ctypes.CDLL(library)

    def reset(self, status=0):
        ctypes.c_int.in_dll(self.lib, "status").value = status
        ctypes.c_int.in_dll(self.lib, "calls").value = 0

    @property
    def calls(self):
        return ctypes.c_int.in_dll(self.lib, "calls").value

    @property
    def noted(self):
        return (ctypes.c_char * 4096).in_dll(self.lib, "noted").value.decode().split()


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    return Stub(str(tmp_path_factory.mktemp("native")))


@pytest.fixture
def stub(built):
    built.reset()
    return built


STREAM = types.SimpleNamespace(cuda_stream=0x5EED)


def arguments(name, dtype=torch.bfloat16, **change):
    r = lambda *s: torch.zeros(*s, dtype=dtype)
    stats = lambda: torch.zeros(2, 3)
    ids, off = torch.zeros(2, 3, dtype=torch.int64), torch.tensor([0, 2, 6], dtype=torch.int32)
    tail = dict(workspace=None, stream=STREAM)
    grouped = dict(x=r(ROWS, K), w=r(G, K, N))
    a = {"embedding_fwd": dict(table=r(V, D), ids=ids, scale=0.5, out=None, stream=STREAM),
         "embedding_bwd": dict(d_out=r(2, 3, D), ids=ids, rows=V, scale=0.5, out=None, **tail),
         "layer_norm_fwd": dict(x=r(2, 3, D), weight=r(D), bias=r(D), eps=0.25, out=None, mean=None, rstd=None, want_stats=True, stream=STREAM),
         "layer_norm_bwd": dict(x=r(2, 3, D), weight=r(D), dy=r(2, 3, D), mean=stats(), rstd=stats(), want_dx=True, want_dw=None, want_db=None, out=None,
                                **tail),
         "grouped_linear_fwd": dict(**grouped, offsets=off, out=None, stream=STREAM),
         "grouped_linear_bwd": dict(**grouped, dy=r(ROWS, N), offsets=off, want_dx=True, want_dw=True, out=None, **tail)}[name]
    assert set(change) <= set(a)
    a.update(change)
    return a


def results_of(name):
    return {"embedding_fwd": ["out"], "embedding_bwd": ["d_table"], "layer_norm_fwd": ["y", "mean", "rstd"], "layer_norm_bwd": ["dx", "dw", "db"],
            "grouped_linear_fwd": ["y"], "grouped_linear_bwd": ["dx", "dw"]}[name]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("name", ENTRIES)
def test_every_argument_arrives_in_its_place(stub, name, given, dtype):
    a = arguments(name, dtype)
    if given:
        r = lambda *s: torch.zeros(*s, dtype=dtype)
        outs = {"embedding_fwd": r(2, 3, D), "embedding_bwd": r(V, D), "layer_norm_fwd": r(2, 3, D), "layer_norm_bwd": [r(2, 3, D), r(D), r(D)],
                "grouped_linear_fwd": r(ROWS, N), "grouped_linear_bwd": (r(ROWS, K), r(G, K, N))}[name]
        a["out"] = outs
        if "workspace" in a:
            a["workspace"] = torch.zeros(5000, dtype=torch.uint8)
        if name == "layer_norm_fwd":
            a["mean"], a["rstd"] = torch.zeros(2, 3), torch.zeros(2, 3)
    result = getattr(stub.native, name)(*a.values())
    assert result is not None and stub.calls == 1
    flat = list(result) if isinstance(result, tuple) else [result]
    if given:
        mine = list(a["out"]) if isinstance(a["out"], (list, tuple)) else [a["out"]] + [a[k] for k in ("mean", "rstd") if k in a]
        assert all(x is y for x, y in zip(flat, mine))
    want = {k: v.data_ptr() for k, v in a.items() if isinstance(v, torch.Tensor)}
    want.update(zip(results_of(name), (t.data_ptr() for t in flat)))
    want.update(stream=0x5EED, dtype=int(dtype == torch.float32), D=D, G=G, K=K, N=N, total=ROWS, n=6, id_bytes=8, scale=0.5, eps=0.25,
                rows=V if name.startswith("embedding") else 6, fill_rest=int(not given))
    if "workspace" in a:
        want["workspace_bytes"] = 5000 if given else {"embedding_bwd": 1000, "layer_norm_bwd": 2000, "grouped_linear_bwd": 3000}[name]
    for arg, text in zip(signature(name), stub.noted):
        var = arg.rsplit(" ", 1)[1].lstrip("*")
        if var == "workspace" and not given:
            assert int(text, 16)
            continue
        value = 0 if text == "(nil)" else int(text, 16) if "*" in arg else float(text)
        assert value == want[var], (var, text, want[var])
    shapes = {"embedding_fwd": [(2, 3, D)], "embedding_bwd": [(V, D)], "layer_norm_fwd": [(2, 3, D), (2, 3), (2, 3)], "layer_norm_bwd": [(2, 3, D), (D,), (D,)],
              "grouped_linear_fwd": [(ROWS, N)], "grouped_linear_bwd": [(ROWS, K), (G, K, N)]}[name]
    assert [tuple(t.shape) for t in flat] == shapes


def test_what_is_not_wanted_is_not_allocated(stub):
    assert stub.native.layer_norm_fwd(*arguments("layer_norm_fwd", want_stats=False).values())[1:] == (None, None)
    got = stub.native.layer_norm_bwd(*arguments("layer_norm_bwd", weight=None).values())
    assert got[1:] == (None, None) and stub.noted[6:8] == ["(nil)", "(nil)"]
    got = stub.native.layer_norm_bwd(*arguments("layer_norm_bwd", want_dx=False, want_dw=False, want_db=True).values())
    assert got[:2] == (None, None) and got[2].shape == (D,)
    dw = torch.zeros(D, dtype=torch.bfloat16)
    got = stub.native.layer_norm_bwd(*arguments("layer_norm_bwd", out=(None, dw, None)).values())
    assert got[0] is None and got[1] is dw and got[2] is None
    got = stub.native.grouped_linear_bwd(*arguments("grouped_linear_bwd", want_dw=False).values())
    assert got[1] is None and stub.noted[4] == "(nil)"


b16 = torch.bfloat16
ODD = [("embedding_fwd", c) for c in (dict(table=None), dict(table=torch.zeros(V, D)[:, ::2]), dict(table=torch.zeros(V, 2, D)), dict(ids=torch.zeros(3)),
                                      dict(ids=torch.zeros(6, dtype=torch.int64)[::2]), dict(scale="x"), dict(out=torch.zeros(2, 3, D)), dict(stream=3))]
ODD += [("embedding_bwd", c) for c in (dict(d_out=torch.zeros(2, 2, D, dtype=b16)), dict(d_out=torch.zeros(D, dtype=b16)), dict(rows=-1), dict(rows=1 << 31),
                                       dict(rows=2.0), dict(out=torch.zeros(V + 1, D, dtype=b16)), dict(workspace=torch.zeros(9)))]
ODD += [("layer_norm_fwd", c) for c in (dict(x=torch.tensor(1.0)), dict(x=torch.zeros(3, 0)), dict(weight=torch.zeros(D)), dict(bias=torch.zeros(D + 1, dtype=b16)),
                                        dict(mean=torch.zeros(6)), dict(rstd=torch.zeros(2, 3, dtype=b16)), dict(want_stats=1), dict(eps=None))]
ODD += [("layer_norm_bwd", c) for c in (dict(dy=torch.zeros(2, 3, D)), dict(mean=None), dict(rstd=torch.zeros(2)), dict(want_dw=1), dict(out=(None, None)),
                                        dict(out=(None, None, torch.zeros(D))))]
ODD += [("grouped_linear_fwd", c) for c in (dict(x=torch.zeros(ROWS, K + 8, dtype=b16)), dict(w=torch.zeros(K, N, dtype=b16)), dict(out=torch.zeros(ROWS, N)),
                                            dict(offsets=torch.tensor([0, 6], dtype=torch.int32)), dict(offsets=torch.tensor([0, 2, 6])))]
ODD += [("grouped_linear_bwd", c) for c in (dict(dy=torch.zeros(ROWS, K, dtype=b16)), dict(want_dx=None, want_dw=2), dict(out=[None]),
                                            dict(out=[None, torch.zeros(K, N, dtype=b16)]))]


@pytest.mark.parametrize("number", range(len(ODD)))
def test_what_is_not_plain_is_left_to_the_python_code(stub, number):
    name, change = ODD[number]
    assert getattr(stub.native, name)(*arguments(name, **change).values()) is None and stub.calls == 0


@pytest.mark.parametrize("name", ENTRIES)
def test_a_refused_launch_raises_and_a_refused_argument_does_not(stub, name):
    from paper_2602_10016_amd import binding as kb
    stub.reset(kb.ERR_LAUNCH)
    with pytest.raises(kb.KunlunError):
        getattr(stub.native, name)(*arguments(name).values())
    for status in (kb.ERR_NULL, kb.ERR_SHAPE, kb.ERR_UNSUPPORTED, kb.ERR_ALIGN, kb.ERR_WORKSPACE):
        stub.reset(status)
        assert getattr(stub.native, name)(*arguments(name).values()) is None and stub.calls == 1
    with pytest.raises(TypeError):
        getattr(stub.native, name)(1)
