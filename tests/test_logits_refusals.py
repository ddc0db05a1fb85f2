"""What the calls on rows of logits refuse, on the host and before any launch: no GPU.  The addresses are never touched."""
import ctypes

import pytest

from paper_2503_23367_b200 import binding as fv
from paper_2503_23367_b200 import build as fv_build

A = 0x10000            # some address, aligned to everything
INVALID, CAPACITY, UNSUPPORTED = 1, 3, 4
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    fv_build.build()
    return fv.lib()


def call(f, defaults, **change):
    unknown = set(change) - set(defaults)
    assert not unknown, unknown
    return f(*{**defaults, **change}.values())


TOKEN = dict(logits=A, dtype=0, ld=100, rows=4, V=100, tau=1.0, ids=A, n_alt=2, logprob=A, stats=A, entropy=A, alt_ids=A, alt_logprob=A, status=None, stream=None)
GRAD = dict(logits=A, dtype=0, ld=100, rows=4, V=100, tau=1.0, ids=A, stats=A, entropy=A, g_logprob=A, g_entropy=A, dlogits=2 * A, ld_out=100, status=None, stream=None)
DISTILL = dict(logits=A, dtype=0, ld=100, rows=4, V=100, tau=1.0, t_ids=A, t_logits=A, K=8, g=A, loss=A, stats=A, dlogits=2 * A, ld_out=100, status=None, stream=None)
DGRAD = dict(logits=A, dtype=0, ld=100, rows=4, V=100, tau=1.0, t_ids=A, t_logits=A, K=8, stats=A, g=A, dlogits=2 * A, ld_out=100, status=None, stream=None)
LINEAR = dict(a=A, w=A, bias=A, rows=4, C=64, V=104, tau=1.0, ids=A, logprob=A, stats=A, entropy=A, workspace=A, bytes=1 << 30, status=None, stream=None)

ROWS = [dict(logits=None), dict(dtype=2), dict(dtype=-1), dict(ld=99), dict(rows=0), dict(rows=-1), dict(V=0), dict(V=-5), dict(tau=0.0), dict(tau=-1.0), dict(tau=NAN),
        dict(tau=INF), dict(tau=1e-7), dict(tau=1e7), dict(logits=A + 2), dict(dtype=1, logits=A + 1)]


@pytest.mark.parametrize("bad", ROWS + [dict(n_alt=-1), dict(n_alt=65), dict(n_alt=0), dict(alt_ids=None), dict(alt_logprob=None), dict(ids=None), dict(logprob=None),
                                        dict(stats=A + 4), dict(n_alt=0, alt_ids=None, alt_logprob=None, ids=None, logprob=None, stats=None, entropy=None)])
def test_token_logprobs(lib, bad):
    assert call(lib.fv_token_logprobs, TOKEN, **bad) == INVALID


@pytest.mark.parametrize("bad", ROWS + [dict(stats=None), dict(stats=A + 4), dict(dlogits=None), dict(dlogits=2 * A + 2), dict(ld_out=99), dict(ids=None), dict(g_logprob=None),
                                        dict(entropy=None), dict(ids=None, g_logprob=None, g_entropy=None), dict(dlogits=A, ld_out=104)])
def test_token_logprobs_grad(lib, bad):
    assert call(lib.fv_token_logprobs_grad, GRAD, **bad) == INVALID


@pytest.mark.parametrize("bad", ROWS + [dict(t_ids=None), dict(t_logits=None), dict(K=0), dict(K=129), dict(loss=None), dict(stats=A + 4), dict(dlogits=None), dict(ld_out=50),
                                        dict(dlogits=2 * A + 1), dict(dlogits=A, ld_out=104)])
def test_distill_topk(lib, bad):
    assert call(lib.fv_distill_topk, DISTILL, **bad) == INVALID          # (dlogits None with g_loss given)


@pytest.mark.parametrize("bad", ROWS + [dict(t_ids=None), dict(t_logits=None), dict(K=0), dict(K=129), dict(stats=None), dict(stats=A + 4), dict(dlogits=None), dict(ld_out=99),
                                        dict(dlogits=A, ld_out=104)])
def test_distill_topk_grad(lib, bad):
    assert call(lib.fv_distill_topk_grad, DGRAD, **bad) == INVALID


@pytest.mark.parametrize("f,args", [("fv_token_logprobs", TOKEN), ("fv_token_logprobs_grad", GRAD), ("fv_distill_topk", DISTILL), ("fv_distill_topk_grad", DGRAD)])
def test_rows_that_are_too_long_or_too_many(lib, f, args):
    more = {"ld_out": 1 << 20} if "ld_out" in args else {}
    assert call(getattr(lib, f), args, V=393217, ld=1 << 20, **more) == UNSUPPORTED
    assert call(getattr(lib, f), args, dtype=1, V=786433, ld=1 << 20, **more) == UNSUPPORTED
    assert call(getattr(lib, f), args, rows=(1 << 28) + 1) == UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(a=None), dict(w=None), dict(a=A + 8), dict(w=A + 8), dict(bias=A + 2), dict(rows=0), dict(C=0), dict(C=60), dict(V=0), dict(V=100), dict(tau=0.0), dict(tau=NAN),
                                 dict(ids=None), dict(logprob=None), dict(stats=A + 4), dict(workspace=None), dict(workspace=A + 128),
                                 dict(ids=None, logprob=None, stats=None, entropy=None)])
def test_linear_logprobs(lib, bad):
    assert call(lib.fv_linear_logprobs, LINEAR, **bad) == INVALID


def test_linear_logprobs_workspace(lib):
    size = lib.fv_linear_logprobs_workspace_bytes
    assert size(0, 8) == 0 and size(8, 0) == 0 and size(-1, 8) == 0
    for rows, V in ((1, 8), (48, 4096), (49, 4096), (8192, 4096), (300, 65536)):
        need = size(rows, V)
        assert 0 < need < 4 * rows * V + (1 << 20)                       # never more than the logits it does without
        assert call(lib.fv_linear_logprobs, LINEAR, rows=rows, V=V, bytes=need - 1) == CAPACITY
    assert size(8192, 131072) < 8192 * 131072 // 4
