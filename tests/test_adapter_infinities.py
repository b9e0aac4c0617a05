"""GPU parity: infinities in the second matrix of a low-rank adapter.  u B^T has an infinity where u meets one (no number where u is 0 or two infinities
differ in sign), and every output whose row of B is finite keeps the bits that it has without them."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("rank", [8, 16, 24, 64, 128])
@pytest.mark.parametrize("T,n,runs", [(1, 3, 1), (6, 4, 2), (40, 3, 5), (300, 4, 2), (512, 20, 1), (650, 4, 2), (650, 20, 1), (1300, 3, 200), (700, 12, 30)])
@pytest.mark.parametrize("in_place", [False, True])
def test_infinities_in_b(dtype, rank, T, n, runs, in_place):
    K, N = 192, 136
    g = ref.seeded(71)
    x, y = ref.normal(g, (T, K), dtype), ref.normal(g, (T, N), dtype)
    a, b = ref.normal(g, (n, rank, K), dtype, K ** -0.5), ref.normal(g, (n, N, rank), dtype, rank ** -0.5)
    scales = torch.rand(n, generator=g, device="cuda") + 0.5
    scales[1::3] *= -1
    which = (torch.arange(T, device="cuda") // runs % (n + 1) - int(T > 1)).int()  # each adapter, and none
    which = torch.where(which < n, which, -1)
    clean = binding.linear_adapters(x, y, a, b, which, scales=scales)
    b[0, 5, 3], b[0, N - 1, rank - 1], b[0, 64, 0] = INF, -INF, INF
    b[1, 5, 3], b[1, 7, 0], b[1, 7, 1], b[1, 9, 2] = -INF, INF, -INF, NAN
    b[2, :, 2] = INF
    if n > 3:
        b[3, 0], b[3, 63, 4:6] = INF, INF
    y[T // 2, 64] = INF  # meets an infinity of adapter 0, or none
    first = binding.linear_adapters(x, y, a, b, which, scales=scales)
    out = binding.linear_adapters(x, y, a, b, which, scales=scales, out=y.clone()) if not in_place else y.clone()
    if in_place:
        binding.linear_adapters(x, out, a, b, which, scales=scales, out=out)
    assert torch.equal(torch.nan_to_num(out, nan=7.0), torch.nan_to_num(first, nan=7.0))
    binding.check_status()

    of = which.long().clamp_min(0)
    u = torch.einsum("tk,trk->tr", x.double(), a.double()[of]) * scales.double()[of, None]
    odd = ~torch.isfinite(b)[of] & (which >= 0)[:, None, None]             # [T, N, rank]
    y_odd = ~torch.isfinite(y)
    same = ~odd.any(2) & ~y_odd
    assert torch.equal(out[same], clean[same])
    # u is known to within 2^-10 of what its products come to, which is far below 2^-5: the sign of a larger one is certain
    sure = odd.any(2) & (~odd | (u.abs() > 2.0 ** -5)[:, None, :]).all(2)
    want = y.double() + torch.where(odd, u[:, None, :] * b.double()[of], 0.0).sum(2)
    assert sure.sum() >= (which >= 0).sum() // 8
    assert torch.equal(torch.isnan(out[sure]), torch.isnan(want[sure]))
    there = sure & ~torch.isnan(want)
    assert torch.equal(out[there].double(), want[there])
    assert (out[which < 0] == y[which < 0]).all()
    assert not torch.isfinite(out[y_odd]).any()


@pytest.mark.parametrize("T", [9, 700])
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
def test_sums_beyond_32_bits_are_infinite_as_they_were(dtype, T):
    """B finite, the sum not: a scale takes it there."""
    g = ref.seeded(72)
    x, y = ref.normal(g, (T, 64), dtype), ref.normal(g, (T, 72), dtype)
    a, b = ref.normal(g, (2, 8, 64), dtype, 30.0), ref.normal(g, (2, 72, 8), dtype, 200.0)
    scales = torch.tensor([2.0 ** 115, 1.0], device="cuda")
    which = (torch.arange(T, device="cuda") % 2).int()
    out = binding.linear_adapters(x, y, a, b, which, scales=scales)
    want = torch.einsum("tr,nr->tn", x.double() @ a[0].double().T * 2.0 ** 115, b[0].double())
    far = (which == 0)[:, None] & (want.abs() > 2.0 ** 130)
    assert far.sum() > 20
    # either an infinity of the sum's sign or, where infinities of both signs meet on the way, no number
    assert ((out[far].double() == want[far].sign() * INF) | torch.isnan(out[far])).all()
    assert torch.isfinite(out[which == 1]).all() if dtype == BF else True
