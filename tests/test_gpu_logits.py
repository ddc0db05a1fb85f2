"""Rows of logits through the C ABI against their definition in float64: log probabilities of given tokens, entropy, alternatives, the
distillation loss, the gradients of both, the head that keeps no logits.

Tolerances come from the roundings on the way (u = 2^-24).  An exponent (x - m) / tau carries the rounding of its scale and of one fused
multiply-add, 2 u |d|; the power of two 4 u; a thread adds at most 100 terms in a row and the group's sums another 30, each u of a
sum of positive terms.  So ln s is within u (134 + 2 D) of its value, D = sum p |d| <= 20 for every row here that is compared, a log probability
within that + 4 u |d|, and a probability relatively within u (2 |d| + 8) more."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2503_23367_b200 import binding as fv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
INF = float("inf")
F32, BF16 = torch.float32, torch.bfloat16
LN = U * (134 + 40)          # ln s


def rows_of(rows, V, dtype, seed, pad=0, shift=0, spread=2.5, offset=4.0):
    """[rows, V] logits inside a wider buffer, the first row `shift` elements into it; and the buffer."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    ld = V + pad
    x = torch.randn(rows, V, device=DEV, generator=g) * spread + torch.randn(rows, 1, device=DEV, generator=g) * offset
    buf = torch.full((shift + rows * ld,), 77.0, device=DEV, dtype=dtype)
    v = buf.as_strided((rows, V), (ld, 1), shift)
    v.copy_(x)
    return v, buf


class Ref:
    """The definition in float64."""

    def __init__(self, x, tau):
        self.x = x.double()
        self.tau = tau
        z = self.x / tau
        self.some = ~torch.isinf(z).all(1) | (z == INF).any(1)
        self.m = self.x.max(1).values
        m0 = torch.where(self.some, self.m, torch.zeros_like(self.m))[:, None]
        self.d = (self.x - m0) / tau
        e = self.d.exp()
        self.L = e.sum(1).log()
        self.logp = torch.where(self.some[:, None], self.d - self.L[:, None], torch.full_like(z, -INF))
        self.p = self.logp.exp()
        self.plogp = torch.where(self.p == 0, torch.zeros_like(z), self.p * self.logp.clamp(min=-1e300))
        self.H = -self.plogp.sum(1)

    def logprob(self, ids):
        lp = self.logp.gather(1, ids.long().clamp(min=0)[:, None])[:, 0]
        return torch.where(ids < 0, torch.zeros_like(lp), lp)

    def alternatives(self, n):
        n1 = min(n, self.x.shape[1])
        order = torch.sort(self.x, dim=1, descending=True, stable=True)
        ids = torch.where(order.values[:, :n1] == -INF, torch.full_like(order.indices[:, :n1], -1), order.indices[:, :n1])
        lp = torch.where(ids < 0, torch.full_like(ids, 0, dtype=torch.float64) - INF, self.logp.gather(1, ids.clamp(min=0)))
        more = n - n1
        return torch.nn.functional.pad(ids, (0, more), value=-1), torch.nn.functional.pad(lp, (0, more), value=-INF)

    def grad(self, ids, gl, ge):
        dx = torch.zeros_like(self.x)
        if gl is not None:
            g = torch.where((ids >= 0) & self.some, gl.double(), torch.zeros_like(self.L))
            dx -= g[:, None] * self.p
            dx[torch.arange(len(g), device=DEV), ids.long().clamp(min=0)] += g
        if ge is not None:
            dx -= ge.double()[:, None] * (self.plogp + self.p * self.H[:, None])
        return dx / self.tau

    def teacher(self, t_ids, t_logits):
        t = torch.where(t_ids < 0, torch.full_like(t_logits, -INF), t_logits).double() / self.tau
        tl = torch.logsumexp(t, 1, keepdim=True)
        some = tl > -INF
        logq = t - torch.where(some, tl, torch.zeros_like(tl))
        return logq, logq.exp(), some

    def loss(self, t_ids, t_logits):
        logq, q, _ = self.teacher(t_ids, t_logits)
        lp = self.logp.gather(1, t_ids.long().clamp(min=0))
        return torch.where(q > 0, q * (logq - lp), torch.zeros_like(q)).sum(1)

    def loss_grad(self, t_ids, t_logits, g):
        _, q, some = self.teacher(t_ids, t_logits)
        dx = self.p * some
        dx.scatter_add_(1, t_ids.long().clamp(min=0), torch.where(self.some[:, None], -q, torch.zeros_like(q)))
        return dx * (1.0 if g is None else g.double()[:, None]) / self.tau


def near(got, ref, tol):
    """Within tol, the same infinities and NaN."""
    got = got.double()
    ref = ref.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)])
    tol = tol if torch.is_tensor(tol) else torch.full_like(ref, tol)
    # a value within its tolerance of the largest float may round to infinity: where every token of a teacher has the lowest logit, the
    # weights' sum of 1 + u times that logit is past the largest float
    top = (ref.abs() + tol > torch.finfo(F32).max) & (got.abs() == INF) & (torch.sign(got) == torch.sign(ref))
    fine &= ~top
    off = (got - ref).abs()[fine] - tol.expand_as(ref)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, f"off by {float((got - ref).abs()[fine].max()):.3e}"


def check_forward(x, ids, tau, n_alt):
    r = fv.fv_token_logprobs(x, ids, tau=tau, n_alt=n_alt, want_entropy=True)
    ref = Ref(x, tau)
    assert torch.equal(r["stats"][:, 0].double(), ref.m)
    near(r["stats"][:, 1], ref.L, LN)
    d = ref.logprob(ids).abs()
    near(r["logprob"], ref.logprob(ids), LN + 4 * U * torch.where(torch.isfinite(d), d + ref.L.abs(), torch.zeros_like(d)))
    # H = L - sum p d: the exponents' errors once more, the quotient, the sum of terms of one sign
    near(r["entropy"], ref.H, 2 * LN + U * 200 * ref.H.abs())
    if n_alt:
        ids_ref, lp_ref = ref.alternatives(n_alt)
        assert torch.equal(r["alt_ids"].long(), ids_ref)
        a = lp_ref.abs()
        near(r["alt_logprob"], lp_ref, LN + 4 * U * torch.where(torch.isfinite(a), a + ref.L[:, None].abs(), torch.zeros_like(a)))
    return r, ref


# rows x V: a warp per row, one CTA, clusters of 2, 4 and 8; odd sizes, rows that start anywhere
SHAPES = [(1, 1, 0, 0), (3, 2, 5, 1), (5, 7, 0, 3), (2, 33, 1, 0), (4, 200, 0, 1), (1300, 200, 3, 1), (1300, 1000, 0, 0), (1185, 4089, 0, 5), (1200, 2047, 1, 0), (70, 4096, 0, 0),
          (300, 4097, 0, 1), (40, 16411, 5, 2), (7, 50021, 0, 0), (1, 65536, 0, 0), (161, 50021, 27, 1), (3, 131072, 0, 0), (2, 262147, 0, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V,pad,shift", SHAPES)
def test_forward_matches_the_definition(rows, V, pad, shift, dtype):
    x, buf = rows_of(rows, V, dtype, 7 * rows + V, pad, shift)
    before = buf.clone()
    g = torch.Generator(device=DEV).manual_seed(V)
    ids = torch.randint(-1, V, (rows,), device=DEV, generator=g).to(torch.int32)
    for n_alt, tau in ((0, 1.0), (1, 0.7), (5, 1.0), (20, 1.0), (24, 2.5), (25, 1.0), (33, 0.9), (64, 1.0)):
        check_forward(x, ids, tau, n_alt)
    assert torch.equal(buf, before)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(3, 900), (1300, 900), (5, 40007)])
@pytest.mark.parametrize("tau", [1e-6, 0.01, 50.0, 1e6])
def test_temperatures_far_from_one(rows, V, dtype, tau):
    """Exponents of up to 2e7 (all but the largest vanish) and of almost 0 (everything is equally likely)."""
    x, _ = rows_of(rows, V, dtype, 17)
    ids = torch.randint(0, V, (rows,), device=DEV).to(torch.int32)
    r, ref = check_forward(x, ids, tau, 3)
    t_ids, t_logits = teacher_of(rows, V, 6, 4)
    d = fv.fv_distill_topk(x, t_ids, t_logits, tau=tau, want_grad=True)
    want = ref.loss(t_ids, t_logits)
    near(d["loss"], want, LN + U * 400 * (want.abs() + 1))
    want = ref.loss_grad(t_ids, t_logits, None)
    # p and q carry the rounding of their exponents, u times up to 150 where they are not 0, twice for the two subtractions
    near(d["dlogits"], want, (torch.finfo(dtype).eps / 2 if dtype != F32 else 0) * want.abs() + (LN + 600 * U) / tau)


@pytest.mark.parametrize("dtype,V", [(F32, 393216), (BF16, 786432), (BF16, 786431)])
def test_the_longest_rows(dtype, V):
    x, _ = rows_of(2, V, dtype, 3)
    ids = torch.tensor([V - 1, -1], dtype=torch.int32, device=DEV)
    for n_alt in (3, 64):
        check_forward(x, ids, 1.0, n_alt)
    g = torch.tensor([0.5, -1.0], device=DEV)
    check_token_grad(x, ids, g, g, 1.0)
    check_distill(x, *teacher_of(2, V, 100, 5), g, 1.0)


def test_many_rows_of_32_kb():
    """Enough rows that a warp takes each, of a length that fewer rows give to a CTA."""
    x, _ = rows_of(3600, 8190, F32, 19)
    ids = torch.randint(0, 8190, (3600,), device=DEV).to(torch.int32)
    for n_alt in (0, 8, 30):
        check_forward(x, ids, 1.0, n_alt)


def test_large_values_in_one_part_of_a_row():
    """The alternatives lie side by side in one CTA's part of the row, and at its ends."""
    for rows, V in ((1, 131072), (3, 262144), (1300, 4096)):
        x, _ = rows_of(rows, V, F32, 23)
        x[:, 1000:1100] += 20.0
        x[:, -40:] += 30.0
        x[:, :3] += 40.0
        ids = torch.zeros(rows, dtype=torch.int32, device=DEV)
        for n_alt in (10, 24, 64):
            check_forward(x, ids, 1.0, n_alt)


def test_refusals_of_the_binding():
    x = torch.randn(4, 100, device=DEV); ids = torch.zeros(4, dtype=torch.int32, device=DEV)
    f = fv.fv_token_logprobs(x, ids, want_entropy=True)
    t_ids = torch.zeros(4, 3, dtype=torch.int32, device=DEV); t_logits = torch.zeros(4, 3, device=DEV)
    bad = [lambda: fv.fv_token_logprobs(x[0]), lambda: fv.fv_token_logprobs(x.half()), lambda: fv.fv_token_logprobs(x.t()), lambda: fv.fv_token_logprobs(x, ids.long()),
           lambda: fv.fv_token_logprobs(x, ids[:3]), lambda: fv.fv_token_logprobs(x, ids.cpu()), lambda: fv.fv_token_logprobs(x.cpu(), ids),
           lambda: fv.fv_token_logprobs_grad(x, ids, f["stats"][:3], ids.float()), lambda: fv.fv_token_logprobs_grad(x, ids, f["stats"], ids),
           lambda: fv.fv_token_logprobs_grad(x, ids, f["stats"], ids.float(), out=x.bfloat16()), lambda: fv.fv_token_logprobs_grad(x, ids, f["stats"], ids.float(), out=x[:3]),
           lambda: fv.fv_distill_topk(x, t_ids, t_logits[:, :2]), lambda: fv.fv_distill_topk(x, t_ids.long(), t_logits), lambda: fv.fv_distill_topk(x, t_ids, t_logits.bfloat16()),
           lambda: fv.fv_linear_logprobs(x, x, None), lambda: fv.fv_linear_logprobs(x.bfloat16(), x[:, :96].bfloat16(), None)]
    for call in bad:
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(fv.FvError) as e:
        fv.fv_token_logprobs(x, ids, n_alt=65)
    assert e.value.code == 1
    with pytest.raises(fv.FvError) as e:
        fv.fv_token_logprobs(torch.zeros(1, 400000, device=DEV))
    assert e.value.code == 4


def test_each_output_alone_is_the_same():
    x, _ = rows_of(37, 5000, BF16, 3)
    ids = torch.randint(0, 5000, (37,), device=DEV).to(torch.int32)
    full = fv.fv_token_logprobs(x, ids, n_alt=9, want_entropy=True)
    assert set(fv.fv_token_logprobs(x)) == {"stats"}
    assert torch.equal(fv.fv_token_logprobs(x)["stats"], full["stats"])
    assert torch.equal(fv.fv_token_logprobs(x, ids)["logprob"], full["logprob"])
    assert torch.equal(fv.fv_token_logprobs(x, want_entropy=True)["entropy"], full["entropy"])
    r = fv.fv_token_logprobs(x, n_alt=9)
    assert torch.equal(r["alt_ids"], full["alt_ids"]) and torch.equal(r["alt_logprob"], full["alt_logprob"])


def special_rows(V, dtype):
    """Rows that go wrong easily, by name."""
    low = torch.finfo(dtype).min
    g = torch.Generator(device=DEV).manual_seed(V)
    n = lambda: torch.randn(V, device=DEV, generator=g)
    r = {"all forbidden": torch.full((V,), -INF, device=DEV), "all equal": torch.full((V,), 3.25, device=DEV), "all zero": torch.zeros(V, device=DEV),
         "both zeros": torch.where(n() > 0, 0.0, -0.0), "all lowest": torch.full((V,), low, device=DEV)}
    one = torch.full((V,), -INF, device=DEV); one[V // 2] = -5.0; r["one left"] = one
    one = torch.full((V,), low, device=DEV); one[V // 3] = 1.0; r["lowest but one"] = one
    r["half lowest"] = torch.where(n() > 0, n(), torch.full((V,), low, device=DEV))
    r["half forbidden"] = torch.where(torch.arange(V, device=DEV) < V // 2, torch.full((V,), -INF, device=DEV), n())
    r["lowest and forbidden"] = torch.where(n() > 0, torch.full((V,), low, device=DEV), torch.full((V,), -INF, device=DEV))
    r["ascending"] = torch.arange(V, device=DEV) / 64.0
    r["descending"] = -torch.arange(V, device=DEV) / 64.0
    r["two values"] = torch.where(n() > 0, 1.0, 2.0)
    r["far up"] = n() + 3000.0
    r["far down"] = n() - 3000.0
    r["peaked"] = torch.where(torch.arange(V, device=DEV) == V - 1, 60.0, 0.0)
    return {k: v.to(dtype) for k, v in r.items()}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,copies", [(5, 1), (600, 1), (600, 100), (4096, 1), (4096, 80), (20011, 1), (70001, 1)])
def test_rows_that_go_wrong_easily(V, copies, dtype):
    rows = special_rows(V, dtype)
    x = torch.stack(list(rows.values()) * copies)
    ids = torch.randint(0, V, (len(x),), device=DEV).to(torch.int32)
    for n_alt in (1, 20, 64):
        # far-off rows: m is exact and subtracted from the logits, so their size adds no error
        r, ref = check_forward(x, ids, 1.0, n_alt)
    names = list(rows)
    assert float(r["entropy"][names.index("all forbidden")]) == 0.0
    t_ids = torch.stack([torch.randint(0, V, (9,), device=DEV) for _ in range(len(x))]).to(torch.int32)
    t_logits = torch.randn(len(x), 9, device=DEV)
    check_distill(x, t_ids, t_logits, None, 1.0)
    g = torch.rand(len(x), device=DEV) + 0.5
    check_token_grad(x, ids, g, g, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(2, 900), (1300, 900), (2, 30000), (2, 150000)])
def test_rows_with_nan_or_infinity(rows, V, dtype):
    """Every result of such a row is NaN, its alternatives -1; its neighbours are what they are without it."""
    x, _ = rows_of(rows, V, dtype, 5)
    ids = torch.zeros(rows, dtype=torch.int32, device=DEV)
    clean = fv.fv_token_logprobs(x, ids, n_alt=6, want_entropy=True)
    t_ids, t_logits = clean["alt_ids"].clone(), clean["alt_logprob"].clone()
    clean_d = fv.fv_distill_topk(x, t_ids, t_logits, want_grad=True)
    for bad in (float("nan"), INF):
        for at in (0, V // 2, V - 1):
            y = x.clone()
            y[1, at] = bad
            r = fv.fv_token_logprobs(y, ids, n_alt=6, want_entropy=True)
            for k in ("logprob", "entropy", "alt_logprob"):
                assert torch.isnan(r[k][1]).all(), k
            assert torch.isnan(r["stats"][1, 1]) and (r["alt_ids"][1] == -1).all()
            d = fv.fv_distill_topk(y, t_ids, t_logits, want_grad=True)
            assert torch.isnan(d["loss"][1]) and torch.isnan(d["dlogits"][1].float()).all()
            dx = fv.fv_token_logprobs_grad(y, ids, r["stats"], torch.ones(rows, device=DEV))
            assert torch.isnan(dx[1].float()).all()
            rest = [i for i in range(rows) if i != 1]
            for k in clean:
                assert torch.equal(r[k][rest], clean[k][rest]), k
            assert torch.equal(d["loss"][rest], clean_d["loss"][rest]) and torch.equal(d["dlogits"][rest], clean_d["dlogits"][rest])


# ------------------------------------------------------------------------------------------------------ gradients
def grad_tol(ref_dx, ref, scale, dtype):
    """p's relative error times p, the sum of its terms, and the one rounding of the result to its type (half a step)."""
    scale = scale.abs()[:, None] / ref.tau
    d = torch.where(ref.p > 0, ref.logp.abs().clamp(max=200), torch.zeros_like(ref.p))
    p = ref.p * (LN + U * (3 * (d + ref.L.abs().clamp(max=200)[:, None]) + 12)) * (1 + d + ref.H[:, None].abs())
    own = torch.finfo(dtype).eps / 2 * ref_dx.abs() if dtype != F32 else 0
    return scale * (2 * p + 6 * U) + own + 2.0 ** -126 * 4


def check_token_grad(x, ids, gl, ge, tau, out=None):
    f = fv.fv_token_logprobs(x, ids, tau=tau, want_entropy=True)
    ref = Ref(x, tau)
    want = ref.grad(ids, gl, ge)
    got = fv.fv_token_logprobs_grad(x, ids, f["stats"], gl, tau=tau, entropy=f["entropy"], g_entropy=ge, out=out)
    scale = (gl.abs() if gl is not None else 0) + (ge.abs() if ge is not None else 0)
    near(got, want, grad_tol(want, ref, scale.double(), x.dtype))
    return got


def check_distill(x, t_ids, t_logits, g, tau, out=None):
    ref = Ref(x, tau)
    loss = ref.loss(t_ids, t_logits)
    r = fv.fv_distill_topk(x, t_ids, t_logits, tau=tau)
    # the loss: q carries the errors of an exponent and of its sum, each entry those of two log probabilities
    logq, q, _ = ref.teacher(t_ids, t_logits)
    lp = ref.logp.gather(1, t_ids.long().clamp(min=0))
    size = torch.where((q > 0) & torch.isfinite(lp), q * (logq.abs() + lp.abs()), torch.zeros_like(q)).sum(1)
    want = ref.loss_grad(t_ids, t_logits, g)
    scale = torch.ones_like(loss) if g is None else g.double()
    tol = grad_tol(want, ref, scale, x.dtype) + (scale.abs() / tau * U * 170)[:, None] * (torch.zeros_like(want).scatter_add_(1, t_ids.long().clamp(min=0), q))
    fused = fv.fv_distill_topk(x, t_ids, t_logits, tau=tau, g_loss=g, want_grad=True)
    for one in (r, fused):               # (the loss alone and the loss with its gradient add in another order)
        assert torch.equal(one["stats"][:, 0].double(), ref.m)
        near(one["stats"][:, 1], ref.L, LN)
        near(one["loss"], loss, LN + U * 170 * (size + 1))
    near(fused["dlogits"], want, tol)
    late = fv.fv_distill_topk_grad(x, t_ids, t_logits, r["stats"], g, tau=tau, out=out)
    near(late, want, tol)
    return fused, late


def teacher_of(rows, V, K, seed, holes=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(0, V, (rows, K), device=DEV, generator=g)            # small V: the same token more than once
    logits = torch.randn(rows, K, device=DEV, generator=g) * 2
    if holes:
        ids = torch.where(torch.rand(rows, K, device=DEV, generator=g) < 0.1, torch.full_like(ids, -1), ids)
        logits = torch.where(torch.rand(rows, K, device=DEV, generator=g) < 0.05, torch.full_like(logits, -INF), logits)
        ids[0] = -1                                                          # a row without entries
    return ids.to(torch.int32), logits


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V,pad,shift", SHAPES)
def test_gradients_match_the_formulas(rows, V, pad, shift, dtype):
    x, buf = rows_of(rows, V, dtype, 5 * rows + V, pad, shift)
    before = buf.clone()
    g = torch.Generator(device=DEV).manual_seed(V)
    ids = torch.randint(-1, V, (rows,), device=DEV, generator=g).to(torch.int32)
    gl, ge = (torch.randn(rows, device=DEV, generator=g) for _ in range(2))
    gl[rows // 2] = 0.0
    for tau, a, b in ((1.0, gl, ge), (0.6, gl, None), (1.7, None, ge)):
        check_token_grad(x, ids if a is not None else None, a, b, tau) if a is not None else check_entropy_grad(x, b, tau)
    for K, tau, w in ((1, 1.0, None), (16, 2.0, gl), (100, 0.8, gl), (128, 1.0, gl)):
        check_distill(x, *teacher_of(rows, V, K, V + K), w, tau)
    assert torch.equal(buf, before)


def check_entropy_grad(x, ge, tau):
    f = fv.fv_token_logprobs(x, None, tau=tau, want_entropy=True)
    ref = Ref(x, tau)
    want = ref.grad(None, None, ge)
    got = fv.fv_token_logprobs_grad(x, None, f["stats"], None, tau=tau, entropy=f["entropy"], g_entropy=ge)
    near(got, want, grad_tol(want, ref, ge.double(), x.dtype))


def test_gradients_match_differences():
    """Against central differences of the definition in float64 (h 1e-4: their own error is below 1e-7 here)."""
    rows, V, tau, K = 3, 40, 1.3, 7
    x, _ = rows_of(rows, V, F32, 11, spread=1.0, offset=0.5)
    ids = torch.tensor([4, 0, 39], dtype=torch.int32, device=DEV)
    t_ids, t_logits = teacher_of(rows, V, K, 3, holes=False)
    gl = torch.tensor([0.7, -1.1, 0.4], device=DEV); ge = torch.tensor([-0.3, 0.9, 1.2], device=DEV)
    f = fv.fv_token_logprobs(x, ids, tau=tau, want_entropy=True)
    got_t = fv.fv_token_logprobs_grad(x, ids, f["stats"], gl, tau=tau, entropy=f["entropy"], g_entropy=ge).double()
    got_d = fv.fv_distill_topk(x, t_ids, t_logits, tau=tau, g_loss=gl, want_grad=True)["dlogits"].double()

    def value(y):
        ref = Ref(y, tau)
        return gl.double() * ref.logprob(ids) + ge.double() * ref.H, gl.double() * ref.loss(t_ids, t_logits)
    for j in range(V):
        up, down = x.double().clone(), x.double().clone()
        up[:, j] += 1e-4; down[:, j] -= 1e-4
        (a, b), (c, d) = value(up), value(down)
        near(got_t[:, j], (a - c) / 2e-4, 2e-6)
        near(got_d[:, j], (b - d) / 2e-4, 2e-6)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V,pad,shift", [(4, 37, 3, 1), (1300, 333, 0, 1), (30, 9001, 2, 3), (5, 100003, 0, 1)])
def test_gradients_in_place_and_in_other_layouts(rows, V, pad, shift, dtype):
    """In place, and into rows that start elsewhere than the logits' do: the same bits as into a tensor of their own, and what lies
    between the rows stays."""
    x, _ = rows_of(rows, V, dtype, 21, pad, shift)
    g = torch.Generator(device=DEV).manual_seed(2)
    ids = torch.randint(0, V, (rows,), device=DEV, generator=g).to(torch.int32)
    gl = torch.randn(rows, device=DEV, generator=g)
    t_ids, t_logits = teacher_of(rows, V, 20, 8)
    f = fv.fv_token_logprobs(x, ids, want_entropy=True)
    calls = [lambda y, out: fv.fv_token_logprobs_grad(y, ids, f["stats"], gl, entropy=f["entropy"], g_entropy=gl, out=out),
             lambda y, out: fv.fv_distill_topk(y, t_ids, t_logits, g_loss=gl, want_grad=True, out=out)["dlogits"],
             lambda y, out: fv.fv_distill_topk_grad(y, t_ids, t_logits, f["stats"], gl, out=out)]
    for call in calls:
        own = call(x, None).clone()
        for opad, oshift in ((0, 0), (5, 2), (1, 1)):
            ld = V + opad
            buf = torch.full((oshift + rows * ld,), 55.0, dtype=dtype, device=DEV)
            out = buf.as_strided((rows, V), (ld, 1), oshift)
            call(x, out)
            assert torch.equal(out, own)
            between = torch.ones_like(buf, dtype=torch.bool)
            between.as_strided((rows, V), (ld, 1), oshift).fill_(False)
            assert (buf[between] == 55.0).all()
        y, ybuf = rows_of(rows, V, dtype, 21, pad, shift)
        call(y, y)
        assert torch.equal(y, own)
        between = torch.ones_like(ybuf, dtype=torch.bool)
        between.as_strided((rows, V), (V + pad, 1), shift).fill_(False)
        assert (ybuf[between] == 77.0).all()


def test_ids_that_are_none_or_outside():
    x, _ = rows_of(6, 900, F32, 4)
    ref = Ref(x, 1.0)
    ids = torch.tensor([-1, 5, 900, -2, 899, 0], dtype=torch.int32, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    lp = fv.fv_token_logprobs(x, ids, status=st)["logprob"]
    assert int(st) == 40
    assert float(lp[0]) == 0 and torch.isnan(lp[2]) and torch.isnan(lp[3])
    good = torch.tensor([1, 4, 5], device=DEV)
    near(lp[good], ref.logprob(ids.clamp(-1, 899))[good], LN + 100 * U)
    st.zero_()
    stats = fv.fv_token_logprobs(x)["stats"]
    dx = fv.fv_token_logprobs_grad(x, ids, stats, torch.ones(6, device=DEV), status=st)
    assert int(st) == 40 and (dx[[0, 2, 3]] == 0).all()
    st.zero_()
    fv.fv_token_logprobs(x, torch.tensor([-1, 0, 1, 2, 3, 899], dtype=torch.int32, device=DEV), status=st)
    assert int(st) == 0
    t_ids = torch.zeros(6, 4, dtype=torch.int32, device=DEV); t_logits = torch.zeros(6, 4, device=DEV)
    t_ids[1, 2] = 900
    r = fv.fv_distill_topk(x, t_ids, t_logits, want_grad=True, status=st)
    assert int(st) == 40 and torch.isnan(r["loss"][1]) and not torch.isnan(r["loss"][[0, 2, 3, 4, 5]]).any()
    assert torch.isfinite(r["dlogits"]).all()
    st.zero_()
    late = fv.fv_distill_topk_grad(x, t_ids, t_logits, r["stats"], status=st)
    assert int(st) == 40
    near(late, r["dlogits"], 1e-6)


def test_a_student_that_forbids_a_teachers_token():
    """Its loss is infinite, its gradient finite: -q at that token."""
    x, _ = rows_of(2, 600, F32, 4)
    x[1, 17] = -INF
    t_ids = torch.tensor([[17, 3]] * 2, dtype=torch.int32, device=DEV); t_logits = torch.zeros(2, 2, device=DEV)
    r = fv.fv_distill_topk(x, t_ids, t_logits, want_grad=True)
    assert torch.isfinite(r["loss"][0]) and float(r["loss"][1]) == INF
    assert torch.isfinite(r["dlogits"]).all() and float(r["dlogits"][1, 17]) == -0.5


# ------------------------------------------------------------------------------------------------------------ head
@pytest.mark.parametrize("rows,Cw,V", [(1, 64, 8), (2, 256, 64), (169, 1024, 4096), (130, 136, 1000), (300, 2048, 4096), (33, 512, 16400), (1000, 72, 264), (5, 8, 100000)])
@pytest.mark.parametrize("bias,tau", [(True, 1.0), (False, 0.6)])
def test_linear_logprobs_match_the_definition(rows, Cw, V, bias, tau):
    """Products of bf16 are exact in fp32; a sum of C of them is within C u sum |a w| at worst, and 8 u sqrt(C) of it is far beyond
    what sums of signs at random come to.  It moves ln p by twice as much / tau, and H by that times the spread of ln p."""
    g = torch.Generator(device=DEV).manual_seed(rows + V)
    a = torch.randn(rows, Cw, device=DEV, generator=g).bfloat16()
    w = (torch.randn(V, Cw, device=DEV, generator=g) * 2.5 / Cw ** 0.5).bfloat16()
    b = (torch.randn(V, device=DEV, generator=g) * 0.1).bfloat16() if bias else None
    ids = torch.randint(-1, V, (rows,), device=DEV, generator=g).to(torch.int32)
    x = a.double() @ w.double().t() + (b.double() if bias else 0)
    ref = Ref(x, tau)
    size = float((a.double().abs() @ w.double().abs().t()).max())
    e = 8 * U * Cw ** 0.5 * max(1.0, size / Cw ** 0.5) / tau
    r = fv.fv_linear_logprobs(a, w, b, ids, tau=tau, want_entropy=True)
    near(r["stats"][:, 0], ref.m, e * tau)
    near(r["stats"][:, 1], ref.L, 2 * e + LN)
    near(r["logprob"], ref.logprob(ids), 2 * e + LN + 200 * U)
    near(r["entropy"], ref.H, 40 * e + 2 * LN + 200 * U * ref.H.abs())


def test_linear_logprobs_with_forbidden_tokens():
    """A bias of -inf forbids a token: p = 0, and where it forbids all, every statistic is -inf and the entropy 0."""
    g = torch.Generator(device=DEV).manual_seed(3)
    for rows in (7, 300):                # the few-row route and the tiles
        a = torch.randn(rows, 128, device=DEV, generator=g).bfloat16()
        w = (torch.randn(1024, 128, device=DEV, generator=g) * 0.2).bfloat16()
        b = torch.where(torch.rand(1024, device=DEV, generator=g) < 0.7, -INF, 0.1).bfloat16()
        ids = torch.randint(-1, 1024, (rows,), device=DEV, generator=g).to(torch.int32)
        ref = Ref(a.double() @ w.double().t() + b.double(), 1.0)
        r = fv.fv_linear_logprobs(a, w, b, ids, want_entropy=True)
        near(r["stats"][:, 1], ref.L, 1e-5)
        near(r["logprob"], ref.logprob(ids), 1e-5)
        near(r["entropy"], ref.H, 1e-4)
        r = fv.fv_linear_logprobs(a, w, torch.full_like(b, -INF), ids, want_entropy=True)
        assert (r["stats"] == -INF).all() and (r["entropy"] == 0).all()
        assert (r["logprob"] == torch.where(ids < 0, 0.0, -INF)).all()


def test_linear_logprobs_ids_none_or_outside():
    a = torch.randn(70, 64, device=DEV).bfloat16(); w = torch.randn(256, 64, device=DEV).bfloat16()
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for rows in (3, 70):
        ids = torch.zeros(rows, dtype=torch.int32, device=DEV)
        ids[0], ids[1] = -1, 256
        st.zero_()
        r = fv.fv_linear_logprobs(a[:rows], w, None, ids, status=st)
        assert int(st) == 40 and float(r["logprob"][0]) == 0 and torch.isnan(r["logprob"][1]) and torch.isfinite(r["logprob"][2:]).all()
        assert set(fv.fv_linear_logprobs(a[:rows], w, None)) == {"stats"}


# ------------------------------------------------------------------------------------------------ streams and graphs
def test_another_stream_and_a_captured_call():
    x, _ = rows_of(600, 20011, BF16, 31)
    ids = torch.randint(0, 20011, (600,), device=DEV).to(torch.int32)
    t_ids, t_logits = teacher_of(600, 20011, 12, 5)
    gl = torch.rand(600, device=DEV)
    a = torch.randn(600, 256, device=DEV).bfloat16(); w = torch.randn(1024, 256, device=DEV).bfloat16()
    lids = (ids % 1024).contiguous()

    def calls():
        f = fv.fv_token_logprobs(x, ids, n_alt=20, want_entropy=True)
        d = fv.fv_distill_topk(x, t_ids, t_logits, g_loss=gl, want_grad=True)
        return [*f.values(), *d.values(), fv.fv_token_logprobs_grad(x, ids, f["stats"], gl, entropy=f["entropy"], g_entropy=gl),
                fv.fv_distill_topk_grad(x, t_ids, t_logits, d["stats"], gl), *fv.fv_linear_logprobs(a, w, None, lids, want_entropy=True).values()]
    first = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = calls()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(first, other))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = calls()
        graphs.append((g, outs))
    other_x, _ = rows_of(600, 20011, BF16, 32)
    keep = x.clone()
    x.copy_(other_x)
    for g, outs in graphs:
        g.replay()
    want = [t.clone() for t in calls()]
    for _, outs in graphs:
        assert all(torch.equal(p, q) for p, q in zip(want, outs))
    x.copy_(keep)
    for g, outs in graphs:
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, outs))


def test_two_calls_at_once():
    x, _ = rows_of(900, 30011, F32, 41)
    y, _ = rows_of(900, 30011, F32, 42)
    want = [fv.fv_token_logprobs(t, n_alt=33, want_entropy=True) for t in (x, y)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, t in zip(streams, (x, y)):
        with torch.cuda.stream(s):
            got.append([fv.fv_token_logprobs(t, n_alt=33, want_entropy=True) for _ in range(4)])
    torch.cuda.synchronize()
    for w, gs in zip(want, got):
        for r in gs:
            assert all(torch.equal(r[k], w[k]) for k in w)


def test_rows_beyond_32_bits():
    """Offsets past 2^32 bytes and 2^31 elements: a few rows far apart."""
    V, ld, rows = 1000, 1 << 29, 6
    buf = torch.empty(ld * (rows - 1) + V, dtype=BF16, device=DEV)
    x = buf.as_strided((rows, V), (ld, 1))
    x.copy_(torch.randn(rows, V, device=DEV))
    ids = torch.arange(rows, device=DEV, dtype=torch.int32)
    check_forward(x, ids, 1.0, 10)
    gl = torch.ones(rows, device=DEV)
    f = fv.fv_token_logprobs(x, ids)
    want = Ref(x, 1.0).grad(ids, gl, None)
    got = fv.fv_token_logprobs_grad(x, ids, f["stats"], gl, out=torch.empty(rows, V, dtype=BF16, device=DEV))
    near(got, want, 2.0 ** -8 * want.abs() + 1e-6)
    t_ids, t_logits = teacher_of(rows, V, 8, 1)
    want = Ref(x, 1.0).loss_grad(t_ids, t_logits, None)
    fv.fv_distill_topk(x, t_ids, t_logits, want_grad=True, out=x)
    near(x, want, 2.0 ** -8 * want.abs() + 2e-6)


# ------------------------------------------------------------------------------------------------- used together
def test_alternatives_of_one_head_teach_another():
    """Scores of a token map's own tokens, alternatives of the unpruned head as the teacher of a second one, a few steps down the gradient."""
    B, n, Cw, V = 2, 36, 256, 1024
    g = torch.Generator(device=DEV).manual_seed(1)
    y = torch.randn(B, n, Cw, device=DEV, generator=g)
    mod = torch.randn(B, 2, Cw, device=DEV, generator=g) * 0.1
    w = (torch.randn(V, Cw, device=DEV, generator=g) * 0.15).bfloat16()
    b = (torch.randn(V, device=DEV, generator=g) * 0.1).bfloat16()
    ids, logits = fv.fv_head_tokens(y, mod, w, b, want_logits=True)
    r, _ = check_forward(logits, ids.reshape(-1), 1.0, 16)
    assert torch.equal(r["alt_ids"][:, 0], ids.reshape(-1)) and torch.equal(r["alt_logprob"][:, 0], r["logprob"])
    a = fv.fv_gather_ln(y, None, mod[:, 0].contiguous(), mod[:, 1].contiguous(), Cw)
    lin = fv.fv_linear_logprobs(a.reshape(B * n, Cw), w, b, ids.reshape(-1), want_entropy=True)
    near(lin["logprob"], r["logprob"], 1e-5)        # the same product, summed in another order: 8 u sqrt(C) of logits of a few units
    near(lin["entropy"], r["entropy"], 1e-4)
    student = logits + 0.5 * torch.randn(B * n, V, device=DEV, generator=g)
    first = check_distill(student, r["alt_ids"], r["alt_logprob"], None, 1.0)[0]
    own = fv.fv_distill_topk(logits, r["alt_ids"], r["alt_logprob"])["loss"]
    # against itself the loss is -ln of the mass that the teacher's entries hold
    near(own, -r["alt_logprob"].double().exp().sum(1).log(), 1e-5)
    assert first["dlogits"].sum(1).abs().max() < 1e-4 and (first["loss"] > 0).all()
