"""Rows of logits, statistics, tokens, weights and biases that a kernel of the library has just written on the stream: the calls on rows of logits read them
behind their dependency wait.  (W of the head is the one exception, a constant of the stream.)"""
import pytest
import torch

from paper_2503_23367_b200 import binding as fv
from test_gpu_stream_order import DEV, _check_in_order, _LongGemm, _randn

pytestmark = pytest.mark.gpu


def _teacher(rows, V, K):
    g = torch.Generator(device=DEV).manual_seed(V)
    return torch.randint(0, V, (rows, K), device=DEV, generator=g).to(torch.int32), torch.randn(rows, K, device=DEV, generator=g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V", [(4, 1024), (1300, 1024), (64, 16384), (2, 65536)])       # a warp, many warps, a CTA, clusters
def test_logits_written_by_the_kernel_before(rows, V, dtype):
    x = _LongGemm(rows, V, dtype, K=2048)
    ids = torch.arange(rows, dtype=torch.int32, device=DEV) % V
    t_ids, t_logits = _teacher(rows, V, 10)
    g = torch.rand(rows, device=DEV)
    stats = torch.tensor([[10.0, 3.0]], device=DEV).repeat(rows, 1)
    out = torch.empty(rows, V, dtype=dtype, device=DEV)
    _check_in_order(x, lambda: list(fv.fv_token_logprobs(x.out, ids, n_alt=6, want_entropy=True).values()), x.renew)
    _check_in_order(x, lambda: list(fv.fv_token_logprobs(x.out, ids).values()), x.renew)
    _check_in_order(x, lambda: list(fv.fv_distill_topk(x.out, t_ids, t_logits).values()), x.renew)
    _check_in_order(x, lambda: list(fv.fv_distill_topk(x.out, t_ids, t_logits, g_loss=g, want_grad=True).values()), x.renew)
    _check_in_order(x, lambda: fv.fv_token_logprobs_grad(x.out, ids, stats, g, out=out).clone(), x.renew)
    _check_in_order(x, lambda: fv.fv_distill_topk_grad(x.out, t_ids, t_logits, stats, g, out=out).clone(), x.renew)


@pytest.mark.parametrize("rows,V", [(8, 1024), (8, 16384)])
def test_small_inputs_written_by_the_kernel_before(rows, V):
    """Teacher, statistics, entropies and weights out of one produced buffer; tokens by the library's token choice."""
    K = 8
    made = _LongGemm(rows, 64, torch.float32)
    x = _randn(3, rows, V)
    stats = torch.empty(rows, 2, device=DEV)
    t_ids = _teacher(rows, V, K)[0]
    col = lambda i: made.out.view(-1)[rows * i:rows * (i + 1)]
    _check_in_order(made, lambda: list(fv.fv_distill_topk(x, t_ids, made.out.view(-1)[:rows * K].view(rows, K), g_loss=col(60), want_grad=True).values()), made.renew)
    _check_in_order(made, lambda: list(fv.fv_distill_topk(x, t_ids, made.out.view(-1)[:rows * K].view(rows, K)).values()), made.renew)
    s = made.out.view(-1)[:rows * 2].view(rows, 2)
    _check_in_order(made, lambda: fv.fv_distill_topk_grad(x, t_ids, made.out.view(-1)[rows * 8:rows * 16].view(rows, K), s, col(60)), made.renew)
    ids = torch.zeros(rows, dtype=torch.int32, device=DEV)
    _check_in_order(made, lambda: fv.fv_token_logprobs_grad(x, ids, s, col(40), entropy=col(41), g_entropy=col(42)), made.renew)
    src = _LongGemm(rows, V, torch.float32, K=2048)

    def tokens():
        chosen = fv.fv_argmax_rows(src.out)
        return [chosen, *fv.fv_token_logprobs(x, chosen).values()]
    _check_in_order(src, tokens, src.renew)


@pytest.mark.parametrize("rows,C,V", [(1, 1024, 4096), (40, 2048, 4096), (300, 1024, 4096), (4000, 512, 2048)])
def test_rows_and_bias_of_the_head_written_by_the_kernel_before(rows, C, V):
    w = _randn(4, V, C, std=0.02, dtype=torch.bfloat16)
    ids = torch.zeros(rows, dtype=torch.int32, device=DEV)
    a = _LongGemm(rows, C, torch.bfloat16)
    b = _randn(5, V, dtype=torch.bfloat16)
    _check_in_order(a, lambda: list(fv.fv_linear_logprobs(a.out, w, b, ids, want_entropy=True).values()), a.renew)
    bias, rest = _LongGemm(8, V, torch.bfloat16), _randn(6, rows, C, dtype=torch.bfloat16)
    _check_in_order(bias, lambda: list(fv.fv_linear_logprobs(rest, w, bias.out[0], ids, want_entropy=True).values()), bias.renew)
    src = _LongGemm(rows, V, torch.float32, K=2048)

    def tokens():
        chosen = fv.fv_argmax_rows(src.out)
        return [chosen, *fv.fv_linear_logprobs(rest, w, b, chosen, want_entropy=True).values()]
    _check_in_order(src, tokens, src.renew)
