"""fv_linear_logprobs where a CTA pair takes several tiles, a tile several segments of K and the ring wraps across tiles; and what the segments are for."""
import pytest
import torch

from paper_2503_23367_b200 import binding as fv
from test_gpu_logits import DEV, LN, U, Ref, near

pytestmark = pytest.mark.gpu


# 256 columns: 7 tiles per pair of 4 segments; 6 tiles of 3 segments, the last of 72; two to three tiles of one k-block, ragged.  128 columns: 160 tiles on 74 pairs,
# 3 segments, the last of 8; few rows that have too long a K for the other route; one row
@pytest.mark.parametrize("rows,Cw,V", [(8192, 2048, 4096), (3000, 1096, 8008), (4100, 64, 3000), (5000, 1032, 1000), (5000, 200, 1000), (7, 4096, 4096), (1, 2056, 9472), (48, 520, 20000)])
@pytest.mark.parametrize("bias,tau", [(True, 1.0), (False, 0.7)])
def test_tiles_and_segments_against_the_definition(rows, Cw, V, bias, tau):
    """Tolerances as for the other sizes: 8 u sqrt(C) of the sum of |a w| for a logit, twice that / tau for ln p."""
    g = torch.Generator(device=DEV).manual_seed(rows + V)
    a = torch.randn(rows, Cw, device=DEV, generator=g).bfloat16()
    w = (torch.randn(V, Cw, device=DEV, generator=g) * 2.5 / Cw ** 0.5).bfloat16()
    b = (torch.randn(V, device=DEV, generator=g) * 0.1).bfloat16() if bias else None
    ids = torch.randint(-1, V, (rows,), device=DEV, generator=g).to(torch.int32)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    first = fv.fv_linear_logprobs(a, w, b, ids, tau=tau, want_entropy=True, status=st)
    for _ in range(3):
        again = fv.fv_linear_logprobs(a, w, b, ids, tau=tau, want_entropy=True, status=st)
        assert all(torch.equal(first[k], again[k]) for k in first)
    assert int(st) == 0
    for r0 in range(0, rows, 2048):                                     # (bounds the memory of the definition)
        s = slice(r0, r0 + 2048)
        x = a[s].double() @ w.double().t() + (b.double() if bias else 0)
        ref = Ref(x, tau)
        size = float((a[s].double().abs() @ w.double().abs().t()).max())
        e = 8 * U * Cw ** 0.5 * max(1.0, size / Cw ** 0.5) / tau
        near(first["stats"][s, 0], ref.m, e * tau)
        near(first["stats"][s, 1], ref.L, 2 * e + LN)
        near(first["logprob"][s], ref.logprob(ids[s]), 2 * e + LN + 200 * U)
        near(first["entropy"][s], ref.H, 40 * e + 2 * LN + 200 * U * ref.H.abs())


@pytest.mark.parametrize("rows,Cw,V", [(1, 2048, 9472), (48, 2048, 9472), (20, 2048, 4096),          # few rows: K split
                                       (2048, 2048, 4096), (400, 2048, 4096), (600, 4096, 2048), (7, 4096, 4096), (5000, 2048, 1000)])
def test_products_of_one_sign_accumulate_in_pieces_of_at_most_512(rows, Cw, V):
    """The tensor core cuts a sum after every 16 products, by some share of its last place.  Of a sum that grows evenly in n cuts that comes to (n + 1) / 2 cuts of the whole: 64.5 in one piece of
    2048, 16.5 in pieces of 512 whatever their number, that is 0.26 of it (0.13 of 4096), and a step or two of rounding to nearest where pieces are joined.  The maximum of a row is the one logit that is returned; the
    library's own product in one piece (a 128-wide tile per CTA) is what it is held against."""
    g = torch.Generator(device=DEV).manual_seed(Cw)
    a = (torch.rand(rows, Cw, device=DEV, generator=g) + 0.5).bfloat16()
    w = (torch.rand(V, Cw, device=DEV, generator=g) + 0.5).bfloat16()
    m = fv.fv_linear_logprobs(a, w, None)["stats"][:, 0].double()
    ref = torch.cat([(a[i:i + 1024].double() @ w.double().t()).max(1).values for i in range(0, rows, 1024)])
    assert fv.lib().fv_gemm_force_path(4) == 0
    try:
        whole = fv.fv_gemm_bf16(a, w, None, 4, out=torch.empty(rows, V, device=DEV)).max(1).values.double()
    finally:
        assert fv.lib().fv_gemm_force_path(0) == 0
    mine, one_piece = (float(((v - ref) / ref).abs().mean()) / U for v in (m, whole))
    assert mine < 0.5 * one_piece, f"{mine:.1f} u in pieces, {one_piece:.1f} u in one"
