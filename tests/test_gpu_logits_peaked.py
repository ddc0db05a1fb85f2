"""Entropies of rows whose head is nearly certain: one logit `gap` above the others, which lie within 0.25 of 0.

With u = 2^-24 and a gap of 24 or more, what one thread adds to the sum that holds the peak is below 4096 e^(0.5 - gap) = u / 60, so it may be lost there.  What is left: two powers of two next to
1 (4 u each), their product, the sums of the parts (5 steps in a warp, 5 over the parts, 3 in a thread), the logarithm and the difference that H is, u each: less than 32 u beside the
errors of the terms themselves, which the tests of ordinary rows bound by 200 u of H."""
import pytest
import torch

from paper_2503_23367_b200 import binding as fv
from test_gpu_logits import BF16, DEV, F32, U, Ref, near

pytestmark = pytest.mark.gpu
GAPS = [24.0, 27.0, 31.0, 36.0, 40.0, 42.5, 43.5]


def peaked(rows, V, dtype, at, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.rand(rows, V, device=DEV, generator=g) * 0.5 - 0.25
    gaps = torch.tensor(GAPS, device=DEV).repeat(rows // len(GAPS) + 1)[:rows]
    x[:, at] = gaps + torch.rand(rows, device=DEV, generator=g) * 0.5
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(1400, 900), (1400, 4096), (70, 4096), (70, 20011), (14, 131072)])     # a warp, a CTA, a cluster
@pytest.mark.parametrize("place", ["first", "early", "middle", "late", "last"])
def test_entropy_of_a_peak_anywhere_in_the_row(rows, V, dtype, place):
    at = {"first": 0, "early": V // 5, "middle": V // 2, "late": V - V // 9, "last": V - 1}[place]
    for tau in (1.0, 0.9):
        x = peaked(rows, V, dtype, at, V + at)
        ref = Ref(x, tau)
        assert 0 < float(ref.H.min()) and float(ref.H.max()) < 1e-3
        ids = torch.full((rows,), at, dtype=torch.int32, device=DEV)
        for n_alt in (0, 5, 30):
            r = fv.fv_token_logprobs(x, ids, tau=tau, n_alt=n_alt, want_entropy=True)
            near(r["entropy"], ref.H, 32 * U + 200 * U * ref.H)
            near(r["logprob"], ref.logprob(ids), 32 * U)


@pytest.mark.parametrize("dtype,far", [(F32, 300.0), (F32, -300.0), (F32, 40000.0), (BF16, 300.0), (BF16, -300.0)])
def test_entropy_of_a_peak_in_rows_away_from_zero(dtype, far):
    """The largest logit times log2 e rounds by up to 2^-24 of itself, which is put right."""
    x = peaked(70, 5000, F32, 4700, 3) + far
    x = x.to(dtype)
    ref = Ref(x, 1.0)
    r = fv.fv_token_logprobs(x, n_alt=0, want_entropy=True)
    near(r["entropy"], ref.H, 32 * U + 200 * U * ref.H)


@pytest.mark.parametrize("rows,V", [(40, 1000), (300, 1000), (600, 9504)])        # few rows, tiles of 128 columns, of 256
def test_entropy_of_a_peak_under_the_head(rows, V):
    """a and w are small, so that logits are the bias within 0.25 and exact to 2^-24 of that: H moves by less than u."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    a = (torch.rand(rows, 64, device=DEV, generator=g) * 0.1).bfloat16()
    w = ((torch.rand(V, 64, device=DEV, generator=g) - 0.5) * 0.02).bfloat16()
    for at in (0, V // 2, V - 1):
        for gap in GAPS:
            b = torch.zeros(V, device=DEV).bfloat16()
            b[at] = gap
            ref = Ref(a.double() @ w.double().t() + b.double(), 1.0)
            r = fv.fv_linear_logprobs(a, w, b, want_entropy=True)
            near(r["entropy"], ref.H, 33 * U + 200 * U * ref.H)
