"""The C ABI and the binding of the operators for drafted tokens, without a GPU."""
import ctypes as C

import pytest
import torch

import drafts_reference as DR
from test_ops_abi import lib, test_binding_structs_follow_the_header as follows_the_header  # noqa: F401


@pytest.mark.parametrize("name", ["e2_verify_args", "e2_keep_args"])
def test_structs(name):
    follows_the_header(name)


def test_calls_refuse_without_arguments(lib):  # noqa: F811
    from paper_2606_03770_gb300 import e2ga
    assert lib.e2_verify_drafts(None, None) == e2ga.E2_EINVAL
    assert lib.e2_cache_keep(None, None, None) == e2ga.E2_EINVAL
    assert lib.e2_cache_layers(None, 1, None) == e2ga.E2_EINVAL
    assert lib.e2_cache_attend_tree_workspace(None, None) == 0
    assert b"" != lib.e2_ops_error()


def test_the_binding_leaves_what_is_not_plain(lib):  # noqa: F811
    """The compiled binding loads without a GPU, and goes by for anything but tensors on one."""
    from paper_2606_03770_gb300 import ops
    b, z, i32 = ops.binding(), torch.zeros, dict(dtype=torch.int32)
    assert b.verify(z(2, 8), z(2, **i32), z(2, **i32), z(2, **i32), z(2), None, None, 2) is None
    for f in (b.verify, b.attend_tree, b.keep):
        assert f() is None and f(None) is None


def test_host_tensors_are_refused():
    from paper_2606_03770_gb300 import ops
    z, i32 = torch.zeros, dict(dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        ops.verify_drafts(z(2, 8), z(2, **i32), z(2, **i32), z(2, **i32), z(2))
    with pytest.raises(ValueError, match="Cache objects"):
        ops.CacheLayers([])
    with pytest.raises(ValueError, match="Cache objects"):
        ops.CacheLayers([z(1)])
    with pytest.raises(ValueError, match="CacheLayers"):
        ops.cache_keep(None, z(1, 1, **i32), z(1, **i32), z(2, **i32), z(1, 1, **i32), z(1, **i32))


def test_reference_answers_with_the_targets_probabilities():
    """Two children drawn from the draft, then the walk: summed over the draws and over the intervals in
    which the random numbers decide alike, the token after node 0 has the target's probabilities."""
    V = 4
    logits, draft = torch.tensor([[0.2, 1.0, -0.5, 0.4]] * 3), torch.tensor([[1.1, 0.0, 0.3, -2.0]] * 3)
    p, q = DR.probabilities(logits[0], 1.0), DR.probabilities(draft[0], 1.0)
    got = torch.zeros(V, dtype=torch.float64)
    parents, starts = torch.tensor([-1, 0, 0]), [0, 3]
    pieces = lambda edge: [(0.0, edge), (edge, 1.0)] if edge < 1 else [(0.0, 1.0)]
    for a in range(V):
        for b in range(V):
            rest = [p]
            for _ in range(2):
                rest.append((rest[-1] - q).clamp_min(0))
                rest[-1] = rest[-1] / rest[-1].sum()
            for lo1, hi1 in pieces(float(p[a] / q[a])):
                for lo2, hi2 in pieces(float(rest[1][b] / q[b])):
                    edges = [0.0] + torch.cumsum(rest[2], 0).tolist()
                    for lo0, hi0 in zip(edges, edges[1:]):
                        if hi0 - lo0 < 1e-9 or hi2 - lo2 < 1e-9:
                            continue
                        u = torch.tensor([(lo0 + hi0) / 2, (lo1 + hi1) / 2, (lo2 + hi2) / 2])
                        _, _, answer = DR.verify(logits, torch.tensor([0, a, b]), parents, starts, u, draft, None, 3)
                        got[answer[0][0]] += float(q[a] * q[b]) * (hi1 - lo1) * (hi2 - lo2) * (hi0 - lo0)
    assert float((got - p).abs().max()) < 1e-7         # (64 draws, and pieces below 1e-9 left out)
