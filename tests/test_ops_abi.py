"""The operators' C ABI and binding without a GPU."""
import ctypes as C
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2606_03770_gb300 import build, ops
    build.build()
    return ops.load()


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "e2ops.h")).read(), flags=re.S)


def test_exports_every_declared_symbol(lib):
    from paper_2606_03770_gb300 import ops
    names = set(re.findall(r"\b(e2_[a-z_]+)\s*\(", header()))
    assert names == set(ops.SIGNATURES)
    for n in names:
        assert hasattr(lib, n), n


@pytest.mark.parametrize("name", ["e2_quant_weight", "e2_matmul_args", "e2_cache", "e2_append_args",
                                  "e2_attend_args", "e2_logprobs_args"])
def test_binding_structs_follow_the_header(name):
    from paper_2606_03770_gb300 import ops
    body = re.search(r"typedef struct \{([^}]*)\}\s*" + name + r"\s*;", header()).group(1)
    decl = []
    for stmt in body.split(";"):
        stmt = stmt.replace("const ", "").strip()
        if stmt:
            t, rest = stmt.split(None, 1)
            decl += [(t, v.strip()) for v in rest.split(",")]
    size = {"int32_t": 4, "int64_t": 8, "float": 4}
    mine = getattr(ops, name)._fields_
    assert [v.lstrip("* ") for _, v in decl] == [n for n, _ in mine]
    for (t, v), (n, ct) in zip(decl, mine):
        assert (ct is C.c_void_p) if v.startswith("*") else C.sizeof(ct) == size[t], n


def test_calls_refuse_without_arguments(lib):
    from paper_2606_03770_gb300 import e2ga
    assert lib.e2_quant_matmul(None, None, None, 0, None) == e2ga.E2_EINVAL
    assert lib.e2_ops_error() != b""
    assert lib.e2_cache_append(None, None, None) == e2ga.E2_EINVAL
    assert lib.e2_token_logprobs(None, None) == e2ga.E2_EINVAL


def test_host_tensors_are_refused():
    from paper_2606_03770_gb300 import ops
    z = torch.zeros
    with pytest.raises(ValueError, match="on the GPU"):
        ops.QuantWeight(z(4, 32, dtype=torch.uint8), z(4, 1, dtype=torch.float16))
    with pytest.raises(ValueError, match="on the GPU"):
        ops.Cache.empty(2, 16, 1, 64, device="cpu")
    with pytest.raises(ValueError, match="on the GPU"):
        ops.token_logprobs(z(2, 8))


def test_workspaces_are_sized_on_the_tensors_device(monkeypatch):
    """The plan goes by the current device's multiprocessors: the tensors' device is the current one then."""
    from paper_2606_03770_gb300 import ops
    current, asked = [0], []

    class Library:
        def __getattr__(self, name):
            return lambda *args: asked.append((name, args, current[0])) or 0

    class On:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, current[0] = current[0], self.device.index

        def __exit__(self, *error):
            current[0] = self.before

    monkeypatch.setattr(ops, "_lib", Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", On)
    for index in (0, 2):
        assert ops._workspace("e2_quant_matmul_workspace", torch.device("cuda", index), 5, 64, 1) is None
        assert asked.pop() == ("e2_quant_matmul_workspace", (5, 64, 1), index) and current == [0]


@pytest.mark.gpu
def test_calls_ask_for_workspaces_there(monkeypatch):
    from paper_2606_03770_gb300 import ops
    asked = []
    real = ops._workspace
    monkeypatch.setattr(ops, "_workspace", lambda name, device, *args: asked.append((name, device)) or real(name, device, *args))
    i32 = dict(dtype=torch.int32, device="cuda")
    w = ops.quantize_weight(torch.randn(64, 64, device="cuda"))
    ops.quant_matmul(torch.zeros(40, 64, device="cuda", dtype=torch.float16), w)
    cache = ops.Cache.empty(64, 64, 1, 64)
    ops.cache_attend(cache, torch.zeros(1, 8, 64, device="cuda", dtype=torch.float16), torch.zeros(1, 64, **i32),
                     torch.full((1,), 4096, **i32), torch.tensor([0, 1], **i32), max_new=1, max_len=4096)
    assert asked == [("e2_quant_matmul_workspace", w.device), ("e2_cache_attend_workspace", cache.device)]
