"""GPU parity: low-rank adapters of many requests beside a shared projection, against the definition in 64 bits with the bound that the
operator's roundings give."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
TYPES = pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])


def definition(x, y, a, b, which, scales):
    """(out in fp64, bound).  u = x A^T is summed in fp32 by instructions of 16 products: 2^-22 of the sum of magnitudes for each of them and the
    24 sums behind them (truncation allowed); its two 16-bit halves leave 2^-16 (bf16) or 2^-21 (fp16: 2^-11 of 2^-11, and 2^-39 of the token's
    largest) of it; the second product is summed likewise over twice the ranks; the sum with y is rounded to fp32, and once to the type."""
    K, r = x.shape[1], a.shape[1]
    split = 2.0 ** -16 if x.dtype == BF else 2.0 ** -21
    out, bound = y.double(), torch.zeros_like(y, dtype=torch.float64)
    for i in which.unique().tolist():
        if not 0 <= i < a.shape[0]:
            continue
        at = (which == i).nonzero().flatten()
        X, A, B, s = x[at].double(), a[i].double(), b[i].double(), float(scales[i]) if scales is not None else 1.0
        u, mag = X @ A.T * s, X.abs() @ A.abs().T * abs(s)
        e = mag * ((K / 16 + 24) * 2.0 ** -22) + u.abs() * (split + 2.0 ** -23) + u.abs().amax(1, keepdim=True) * 2.0 ** -38
        out[at] += u @ B.T
        bound[at] = e @ B.abs().T + u.abs() @ B.abs().T * ((2 * r / 16 + 8) * 2.0 ** -22)
    bound += out.abs() * (ref.HALF[x.dtype] * 1.01 + 2.0 ** -23) + 2.0 ** -25
    return out, bound


def make(seed, dtype, T, n, rank, K, N):
    g = ref.seeded(seed)
    x, y = ref.normal(g, (T, K), dtype), ref.normal(g, (T, N), dtype)
    a, b = ref.normal(g, (n, rank, K), dtype, K ** -0.5), ref.normal(g, (n, N, rank), dtype, rank ** -0.5)
    scales = torch.rand(n, generator=g, device="cuda") * 3 - 1
    return g, x, y, a, b, scales


def check(seed, dtype, T, n, rank, K, N, which=None, runs=1, with_scales=True):
    g, x, y, a, b, scales = make(seed, dtype, T, n, rank, K, N)
    if which is None:
        R = -(-T // runs)
        which = torch.randint(-1, n, (R,), generator=g, device="cuda").repeat_interleave(runs)[:T]
    which = which.int()
    scales = scales if with_scales else None
    out = binding.linear_adapters(x, y, a, b, which.contiguous(), scales=scales)
    want, bound = definition(x, y, a, b, which, scales)
    ref.assert_within(out, want, bound)
    assert torch.equal(out[which < 0], y[which < 0])
    assert torch.equal(out, binding.linear_adapters(x, y, a, b, which.contiguous(), scales=scales))
    return out


@TYPES
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("T,runs", [(1, 1), (3, 1), (40, 1), (150, 2), (333, 9), (1000, 1), (1300, 70)])
def test_ranks_and_tokens(dtype, rank, T, runs):
    check(1, dtype, T, 7, rank, 264, 200, runs=runs)


@TYPES
@pytest.mark.parametrize("K,N", [(8, 8), (64, 64), (72, 4096), (4096, 72), (768, 2304), (1000, 520), (14336, 136), (2048, 8192)])
@pytest.mark.parametrize("T,runs", [(5, 2), (400, 30), (700, 130)])
def test_widths(dtype, K, N, T, runs):
    check(2, dtype, T, 3, 16, K, N, runs=runs)


@TYPES
@pytest.mark.parametrize("T", [512, 513, 640, 2000, 2369, 4737, 9000])
def test_large_tiles(dtype, T):
    """Runs that begin and end anywhere in a tile, one of all its tokens, and tokens in turns."""
    check(3, dtype, T, 5, 64, 512, 256, runs=157)
    check(6, dtype, T, 40, 72, 192, 392, which=(torch.arange(T, device="cuda") // 900 * 7 + torch.arange(T, device="cuda") % 900 // 850 * torch.arange(T, device="cuda")) % 41 - 1)
    check(7, dtype, T, 6, 24, 64, 136, which=torch.where(torch.arange(T, device="cuda") < 512, -1, 3))
    check(4, dtype, T, 2, 8, 128, 64, which=torch.arange(T, device="cuda") % 3 - 1)
    check(5, dtype, T, 1, 128, 128, 128, which=torch.zeros(T, device="cuda"), with_scales=False)


def test_requests_say_whose_a_token_is():
    g, x, y, a, b, scales = make(6, BF, 90, 4, 16, 256, 320)
    adapters = torch.tensor([2, -1, 0, 3, 4, 9, -7], dtype=torch.int32, device="cuda")  # the last three name none
    requests = torch.randint(-2, 9, (90,), generator=g, device="cuda", dtype=torch.int32)
    out = binding.linear_adapters(x, y, a, b, adapters, requests=requests, scales=scales)
    inside = (requests >= 0) & (requests < 7)
    which = torch.where(inside, adapters[requests.clamp(0, 6).long()], -1)
    which = torch.where(which < 4, which, -1)
    want, bound = definition(x, y, a, b, which, scales)
    ref.assert_within(out, want, bound)


@TYPES
@pytest.mark.parametrize("T", [9, 500, 645])
def test_views_and_in_place(dtype, T):
    """The columns of a fused projection, in place; what lies beside them stays."""
    g, x, _, a, b, scales = make(7, dtype, T, 3, 32, 128, 64)
    wide_x, wide_y = ref.normal(g, (T, 400), dtype), ref.normal(g, (T, 200), dtype)
    xv, yv = wide_x[:, 16:144], wide_y[:, 72:136]
    which = (torch.arange(T, device="cuda") // 6 % 4 - 1).int()
    before = wide_y.clone()
    want, bound = definition(xv, yv.clone(), a, b, which, scales)
    other = torch.zeros((T, 96), dtype=dtype, device="cuda")
    binding.linear_adapters(xv, yv, a, b, which, scales=scales, out=other[:, 8:72])
    assert torch.equal(wide_y, before) and (other[:, :8] == 0).all() and (other[:, 72:] == 0).all()
    ref.assert_within(other[:, 8:72], want, bound)
    assert binding.linear_adapters(xv, yv, a, b, which, scales=scales, out=yv) is yv
    assert torch.equal(yv, other[:, 8:72])
    assert torch.equal(wide_y[:, :72], before[:, :72]) and torch.equal(wide_y[:, 136:], before[:, 136:])


@TYPES
@pytest.mark.parametrize("T", [6, 300, 650])
def test_what_is_no_number_stays_with_its_token_and_adapter(dtype, T):
    g, x, y, a, b, scales = make(8, dtype, T, 4, 16, 192, 128)
    which = (torch.arange(T, device="cuda") // 2 % 3).int()      # adapter 3 is nobody's
    clean = binding.linear_adapters(x, y, a, b, which, scales=scales)
    x[1, 5], x[4, 7] = float("nan"), float("inf")
    y[3, 9] = float("inf")
    a[3], b[3] = float("nan"), float("nan")
    scales[3] = float("nan")
    out = binding.linear_adapters(x, y, a, b, which, scales=scales)
    touched = torch.zeros(T, dtype=torch.bool, device="cuda")
    touched[[1, 3, 4]] = True
    assert torch.equal(out[~touched], clean[~touched])
    assert torch.isnan(out[1]).all() and not torch.isfinite(out[4]).any()
    assert out[3, 9] == float("inf") and torch.equal(out[3, :9], clean[3, :9]) and torch.equal(out[3, 10:], clean[3, 10:])
    a[2, 3, 3] = float("nan")
    out = binding.linear_adapters(x, y, a, b, which, scales=scales)
    assert torch.isnan(out[which == 2]).all() and torch.equal(out[(which < 2) & ~touched], clean[(which < 2) & ~touched])


def test_fp16_products_beyond_its_range():
    """x A^T may pass 65504 where B brings it back, and be far below 2^-24 where the scale does."""
    g, x, y, a, b, _ = make(9, HF, 20, 2, 16, 1024, 128)
    a *= 600
    x *= 60
    b *= 2.0 ** -11
    scales = torch.tensor([1.0, 2.0 ** -20], device="cuda")
    which = (torch.arange(20, device="cuda") % 2).int()
    out = binding.linear_adapters(x, y, a, b, which, scales=scales)
    assert (x.double() @ a[0].double().T).abs().max() > 65504
    want, bound = definition(x, y, a, b, which, scales)
    ref.assert_within(out, want, bound)
    zero = torch.zeros_like(y)
    scales = torch.tensor([0.0, 2.0 ** -12], device="cuda")
    out = binding.linear_adapters(x, zero, a, b, which, scales=scales)
    want, bound = definition(x, zero, a, b, which, scales)
    ref.assert_within(out, want, bound)
    assert (out[which == 0] == 0).all()


def test_a_workspace_may_hold_anything():
    g, x, y, a, b, scales = make(12, BF, 900, 12, 16, 256, 320)
    which = (torch.arange(900, device="cuda") // 70 % 13 - 1).int()
    which[256:384] = torch.arange(128, device="cuda").int() % 12  # a tile by groups of tokens
    want = binding.linear_adapters(x, y, a, b, which, scales=scales)
    need = binding.linear_adapters_workspace_bytes(900, 16)
    for fill in (0, 255, 127):
        buf = torch.full((need + 512,), fill, dtype=torch.uint8, device="cuda")
        out = binding.linear_adapters(x, y, a, b, which, scales=scales, workspace=buf[256: 256 + need], out=torch.empty_like(y))
        assert torch.equal(out, want)
        assert (buf[:256] == fill).all() and (buf[-256:] == fill).all()
    for short in (need - 1, 16):
        with pytest.raises(binding.ForgeError) as e:
            binding.linear_adapters(x, y, a, b, which, workspace=torch.zeros(short, dtype=torch.uint8, device="cuda"))
        assert e.value.status == binding.ERR_WORKSPACE


@TYPES
@pytest.mark.parametrize("T", [37, 700])
def test_beside_a_projection_in_a_graph(dtype, T):
    """linear_act, then the adapters in place, captured and replayed with other tokens and requests."""
    K, N, n, rank = 256, 512, 5, 16
    g, x, _, a, b, scales = make(10, dtype, T, n, rank, K, N)
    w = ref.normal(g, (K, N), dtype, K ** -0.5)
    y = torch.empty((T, N), dtype=dtype, device="cuda")
    requests, adapters = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")

    def step():
        binding.linear_act(x, w, act=binding.ACT_NONE, out=y)
        binding.linear_adapters(x, y, a, b, adapters, requests=requests, scales=scales, out=y)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        x.copy_(ref.normal(g, (T, K), dtype))
        requests.copy_(torch.randint(0, 6, (T,), generator=g, device="cuda").sort().values)
        adapters.copy_(torch.randint(-1, n, (6,), generator=g, device="cuda"))
        graph.replay()
        base = binding.linear_act(x, w, act=binding.ACT_NONE)
        want, bound = definition(x, base, a, b, adapters[requests.long()], scales)
        ref.assert_within(y, want, bound)


def test_on_a_stream_of_its_own():
    g, x, y, a, b, scales = make(11, BF, 64, 8, 16, 512, 512)
    which = (torch.arange(64, device="cuda") % 8).int()
    want = binding.linear_adapters(x, y, a, b, which, scales=scales)
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(binding.linear_adapters(x, y, a, b, which, scales=scales))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
