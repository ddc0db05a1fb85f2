"""What the header promises for rows of logits beyond ordinary ones: rows that hold a NaN or +inf, teachers that do, alternatives of another temperature as a teacher."""
import pytest
import torch

from paper_2503_23367_b200 import binding as fv
from test_gpu_logits import BF16, DEV, F32, INF, LN, U, check_distill, near, rows_of

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(3, 900), (1300, 900), (3, 30000), (3, 150000)])
def test_largest_logit_and_missing_tokens_of_rows_with_nan_or_infinity(rows, V, dtype):
    """m passes over NaN and is +inf where the row holds one; a row without a token has log probability 0, one without entries loss 0 and gradient 0, whatever its logits are."""
    x, _ = rows_of(rows, V, dtype, 5)
    one = torch.ones(rows, device=DEV)
    for bad, both in ((NAN, False), (INF, False), (NAN, True)):
        y = x.clone()
        y[1, V // 3] = bad
        if both:
            y[1, V // 2] = INF
        want = INF if both or bad == INF else float(torch.cat([x[1, :V // 3], x[1, V // 3 + 1:]]).max())
        ids = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
        r = fv.fv_token_logprobs(y, ids, n_alt=3, want_entropy=True)
        assert float(r["stats"][1, 0]) == want and torch.isnan(r["stats"][1, 1]) and torch.isnan(r["entropy"][1])
        assert torch.isnan(r["alt_logprob"][1]).all() and (r["alt_ids"][1] == -1).all()
        assert (r["logprob"] == 0).all()
        assert (fv.fv_token_logprobs_grad(y, ids, r["stats"], one) == 0).all()
        t_ids = torch.full((rows, 2), -1, dtype=torch.int32, device=DEV)
        t_logits = torch.zeros(rows, 2, device=DEV)
        for grad in (False, True):
            d = fv.fv_distill_topk(y, t_ids, t_logits, want_grad=grad)
            assert float(d["stats"][1, 0]) == want and (d["loss"] == 0).all()
        assert (d["dlogits"] == 0).all() and (fv.fv_distill_topk_grad(y, t_ids, t_logits, d["stats"]) == 0).all()


@pytest.mark.parametrize("rows", [5, 300])
def test_largest_logit_of_the_heads_rows_with_nan_or_infinity(rows):
    g = torch.Generator(device=DEV).manual_seed(1)
    a = torch.randn(rows, 64, device=DEV, generator=g).bfloat16()
    w = torch.randn(1000, 64, device=DEV, generator=g).bfloat16()
    ids = torch.zeros(rows, dtype=torch.int32, device=DEV)
    ids[0] = -1
    clean = fv.fv_linear_logprobs(a, w, None, ids, want_entropy=True)
    for bad in (NAN, INF):
        b = torch.zeros(1000, device=DEV).bfloat16()
        b[777] = bad
        r = fv.fv_linear_logprobs(a, w, b, ids, want_entropy=True)
        assert torch.isnan(r["stats"][:, 1]).all() and torch.isnan(r["entropy"]).all()
        assert float(r["logprob"][0]) == 0 and torch.isnan(r["logprob"][1:]).all()
        if bad == INF:
            assert (r["stats"][:, 0] == INF).all()
        else:
            x = fv.fv_gemm_bf16(a, w, None, 4, out=torch.empty(rows, 1000, device=DEV))
            x[:, 777] = -INF
            near(r["stats"][:, 0], x.max(1).values, 64 * U * 64)       # the same products, summed in another order: sums of 64 terms of a few units
    assert torch.isfinite(clean["stats"]).all()


@pytest.mark.parametrize("V", [900, 40000])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_a_teacher_with_nan_or_infinity(V, bad):
    """Its row's loss is NaN, and the gradient at the tokens of its entries; an entry without a token holds anything."""
    x, _ = rows_of(3, V, F32, 9)
    t_ids = torch.tensor([[5, 70, 800, -1]] * 3, dtype=torch.int32, device=DEV)
    t_logits = torch.randn(3, 4, device=DEV)
    t_logits[0, 3] = bad
    t_logits[1, 1] = bad
    good = t_logits.clone()
    good[0, 3] = 0.0
    d = fv.fv_distill_topk(x, t_ids, t_logits, want_grad=True)
    late = fv.fv_distill_topk_grad(x, t_ids, t_logits, d["stats"])
    clean = fv.fv_distill_topk(x, t_ids, good, want_grad=True)
    assert torch.isnan(d["loss"][1]) and torch.isnan(d["dlogits"][1, [5, 70, 800]]).all() and torch.isnan(late[1, [5, 70, 800]]).all()
    for r in (0, 2):
        assert torch.equal(d["loss"][r], clean["loss"][r]) and torch.equal(d["dlogits"][r], clean["dlogits"][r]) and torch.isfinite(late[r]).all()


@pytest.mark.parametrize("tau", [2.0, 0.6])
def test_alternatives_of_another_temperature_as_a_teacher(tau):
    """ln p at temperature tau is the logit over tau and a constant of the row, so tau ln p serves as the teacher's logits: what is a multiple of
    tau apart rounds by 2 u of ln p tau, which the loss divides by tau again."""
    x, _ = rows_of(200, 5000, F32, 13)
    teacher, _ = rows_of(200, 5000, F32, 14)
    alt = fv.fv_token_logprobs(teacher, n_alt=20, tau=tau)
    raw = teacher.gather(1, alt["alt_ids"].long())
    a = fv.fv_distill_topk(x, alt["alt_ids"], tau * alt["alt_logprob"], tau=tau)["loss"]
    b = fv.fv_distill_topk(x, alt["alt_ids"], raw, tau=tau)["loss"]
    off = 4 * U * (alt["alt_logprob"].abs().amax(1).double() + raw.abs().amax(1).double() / tau) + LN
    near(a, b, 2 * off * (1 + b.double().abs()))
    check_distill(x, alt["alt_ids"], (tau * alt["alt_logprob"]).contiguous(), None, tau)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [900, 40000])
def test_log_probabilities_beyond_the_range_of_fp32(V, dtype):
    """The lowest logit over a temperature of 0.5: -inf, the loss over it +inf however little it weighs, gradients finite."""
    x, _ = rows_of(3, V, dtype, 15)
    x[1, 7] = torch.finfo(dtype).min
    ids = torch.full((3,), 7, dtype=torch.int32, device=DEV)
    r = fv.fv_token_logprobs(x, ids, tau=0.5, want_entropy=True)
    assert float(r["logprob"][1]) == -INF and torch.isfinite(r["logprob"][[0, 2]]).all() and torch.isfinite(r["entropy"]).all()
    t_ids = torch.tensor([[7, 3]] * 3, dtype=torch.int32, device=DEV)
    t_logits = torch.tensor([[0.0, 2.0]] * 3, device=DEV)
    for grad in (False, True):
        d = fv.fv_distill_topk(x, t_ids, t_logits, tau=0.5, want_grad=grad)
        assert float(d["loss"][1]) == INF and torch.isfinite(d["loss"][[0, 2]]).all()
    late = fv.fv_distill_topk_grad(x, t_ids, t_logits, d["stats"], tau=0.5)
    one = torch.ones(3, device=DEV)
    token = fv.fv_token_logprobs_grad(x, ids, r["stats"], one, tau=0.5, entropy=r["entropy"], g_entropy=one)
    assert all(torch.isfinite(t.float()).all() for t in (d["dlogits"], late, token))
