"""Host-side checks of the orthogonalised update and of the stateless operators that need no GPU."""
import ctypes

import pytest

from paper_2412_05270_b200 import binding as B
from paper_2412_05270_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(steps=0), dict(steps=33), dict(momentum=1.0), dict(momentum=-0.1), dict(scale=3), dict(eps=0.0),
    dict(eps=float("nan")), dict(workspace_mb=-1), dict(coef=(float("inf"), 0, 0)),
    dict(coef=(9.0, 0.0, 0.0)),                       # leaves |x| <= 8 in the first step
    dict(coef=(3.4445, 4.7750, 2.0315)),              # a sign lost: diverges within the steps
])
def test_muon_configurations_that_are_refused(kw):
    with pytest.raises(B.ApolloError) as e:
        B.muon_workspace_bytes([(64, 64)], B.make_muon_config(**kw))
    assert e.value.code == B.ERR_INVALID_ARG


@pytest.mark.parametrize("shapes,code", [
    ([], B.ERR_INVALID_ARG), ([(0, 4)], B.ERR_SHAPE), ([(4, -1)], B.ERR_SHAPE), ([(2 ** 20 + 1, 4)], B.ERR_SHAPE),
])
def test_muon_shapes_that_are_refused(shapes, code):
    with pytest.raises(B.ApolloError) as e:
        B.muon_workspace_bytes(shapes, B.make_muon_config())
    assert e.value.code == code


def test_muon_workspace_holds_one_group():
    one = B.muon_workspace_bytes([(4096, 4096)], B.make_muon_config())
    iterates = (2 + 3) * 4096 * 4096 * 2
    assert iterates <= one < iterates + (1 << 20)
    pairs = B.muon_workspace_bytes([(4096, 4096)], B.make_muon_config(dtype=B.DT_F32))
    assert 2 * iterates <= pairs < 2 * iterates + (1 << 20)
    # as many matrices as fit are in flight together, not the whole list
    many = B.muon_workspace_bytes([(4096, 4096)] * 100, B.make_muon_config(workspace_mb=512))
    assert 3 * iterates <= many < (512 << 20) + (4 << 20)
    assert B.muon_workspace_bytes([(4096, 4096)] * 100, B.make_muon_config(workspace_mb=1)) < one + (4 << 20)


def test_null_pointers_are_refused():
    lib = B.load()
    cfg, shapes = B.make_muon_config(), B._shape_array([(8, 8)])
    assert lib.apollo_muon_workspace_bytes(shapes, 1, None, None) == B.ERR_INVALID_ARG
    out = ctypes.c_size_t(0)
    assert lib.apollo_muon_workspace_bytes(None, 1, ctypes.byref(cfg), ctypes.byref(out)) == B.ERR_INVALID_ARG
    ctx = ctypes.c_void_p()
    assert lib.apollo_muon_create(ctypes.byref(ctx), shapes, 1, ctypes.byref(cfg), None, 1 << 30) == B.ERR_INVALID_ARG
    assert lib.apollo_muon_create(ctypes.byref(ctx), shapes, 1, ctypes.byref(cfg), 256, 16) == B.ERR_WORKSPACE
    assert lib.apollo_muon_create(ctypes.byref(ctx), shapes, 1, ctypes.byref(cfg), 128, 1 << 30) == B.ERR_WORKSPACE
    assert not ctx
    assert lib.apollo_muon_destroy(None) == B.ERR_INVALID_ARG
    assert lib.apollo_muon_step(None, None, None, None, 0.1, 0.0, None) == B.ERR_INVALID_ARG
    assert lib.apollo_embedding(None, 4, 4, B.DT_F32, None, B.INDEX_I64, 3, 1.0, None, 4, None) == B.ERR_INVALID_ARG
    assert lib.apollo_embedding(None, 4, 4, B.DT_F32, None, 7, 3, 1.0, None, 4, None) == B.ERR_INVALID_ARG
    assert lib.apollo_embedding(None, 4, 4, B.DT_F32, None, B.INDEX_I64, 3, 1.0, None, 3, None) == B.ERR_SHAPE
    assert lib.apollo_embedding(None, 4, 4, B.DT_F32, None, B.INDEX_I64, 0, 1.0, None, 4, None) == B.OK
    assert lib.apollo_token_logprobs(None, 4, 2, 4, B.DT_F32, None, B.INDEX_I64, 1.0, 0, None, None, None, None, None, None) == B.ERR_INVALID_ARG
    assert lib.apollo_token_logprobs(None, 3, 2, 4, B.DT_F32, None, B.INDEX_I64, 1.0, 0, None, None, None, None, None, None) == B.ERR_SHAPE
    assert lib.apollo_token_logprobs_grad(None, 4, 2, 4, B.DT_F32, None, B.INDEX_I64, 1.0, None, None, None, None, None, 4, None) == B.ERR_INVALID_ARG
    assert lib.apollo_embedding_grad(None, 4, None, B.INDEX_I64, 3, 4, 4, B.DT_F32, 1.0, 2, 16, None, 0, None) == B.ERR_INVALID_ARG


def test_embedding_grad_workspace_covers_the_sort_and_the_pieces():
    n, dim = 10000, 100
    windows = (n + 31) // 32
    need = 2 * 8 * n + windows * 2 * dim * 4
    assert need <= B.embedding_grad_workspace_bytes(n, 500, dim) < need + 4096
    assert B.embedding_grad_workspace_bytes(0, 500, dim) > 0
