"""Where the binding puts a gradient of logits when it is given no place: rows at the logits' offsets from a 16-byte boundary, and no more memory than that takes.  Host code, no GPU."""
import pytest
import torch

from paper_2503_23367_b200 import binding as fv


def _storage(t):
    return t.untyped_storage().nbytes()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V,ld,shift", [(4, 1000, 1000, 0), (4, 1001, 1001, 0), (3, 1001, 1004, 1), (2, 500, 64 * 500, 63 * 500), (5, 333, 9 * 333, 4 * 333), (3, 50021, 50048, 0), (7, 1, 40, 3), (1, 77, 77, 5)])
def test_rows_of_a_new_gradient(rows, V, ld, shift, dtype):
    x = torch.zeros(shift + rows * ld, dtype=dtype)[shift:shift + (rows - 1) * ld + V].as_strided((rows, V), (ld, 1))
    es = x.element_size()
    out, address, ldo = fv._grad_out(x, ld, -1, None)
    assert out.shape == x.shape and out.dtype == dtype and out.stride() == (ldo, 1) and address == out.data_ptr() and ldo >= V
    assert (address - x.data_ptr()) % 16 == 0 and (ldo - ld) * es % 16 == 0        # every row at its logits' offset
    assert _storage(out) <= (rows * V * es) + (rows + 1) * 16
    if ld == V:
        assert out.is_contiguous() and ldo == V


def test_the_last_position_of_long_sequences():
    """[B, T, V] logits of which one position counts: the gradient takes B x V elements, not B x T x V."""
    x = torch.zeros(2, 300, 1024)[:, -1, :]
    out, _, _ = fv._grad_out(x, x.stride(0), -1, None)
    assert _storage(out) == 2 * 1024 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1024, 1001])
def test_gradients_of_the_last_position_of_long_sequences(dtype, V):
    """The same bits as for a copy of those rows, and no more memory than they take."""
    whole = torch.randn(6, 50, V, device="cuda:0").to(dtype)
    x, own = whole[:, -1, :], whole[:, -1, :].contiguous()
    ids = torch.arange(6, dtype=torch.int32, device="cuda:0")
    g = torch.rand(6, device="cuda:0")
    t_ids, t_logits = torch.randint(0, V, (6, 9), device="cuda:0").to(torch.int32), torch.randn(6, 9, device="cuda:0")
    f = fv.fv_token_logprobs(own, ids, want_entropy=True)
    for call in (lambda y: fv.fv_token_logprobs_grad(y, ids, f["stats"], g, entropy=f["entropy"], g_entropy=g),
                 lambda y: fv.fv_distill_topk_grad(y, t_ids, t_logits, f["stats"], g)):
        a, b = call(x), call(own)
        assert torch.equal(a, b) and _storage(a) < 7 * V * x.element_size() + 256
    a, b = (fv.fv_distill_topk(y, t_ids, t_logits, g_loss=g, want_grad=True)["dlogits"].float() for y in (x, own))
    torch.testing.assert_close(a, b, rtol=2.0 ** -7, atol=1e-6)          # (rows at another offset add in another order: the last bit)
    assert _storage(fv.fv_distill_topk(x, t_ids, t_logits, want_grad=True)["dlogits"]) < 7 * V * x.element_size() + 256
