"""Low-rank adapters over views: rows that overlap, those of a broadcast row (stride 0) among them, are refused before anything is launched, by both
ways of marshalling."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

BF, HF = torch.bfloat16, torch.float16


class OnTheGpu:
    """What the binding looks at of a tensor, here without a GPU."""

    def __init__(self, t):
        self.t, self.is_cuda, self.dtype, self.shape = t, True, t.dtype, t.shape

    def dim(self):
        return self.t.dim()

    def stride(self, i):
        return self.t.stride(i)

    def data_ptr(self):
        return self.t.data_ptr()


def test_rows_that_overlap_have_no_stride():
    row = torch.zeros(1, 64, dtype=BF)
    wide = torch.zeros(40, 72, dtype=BF)
    for t in (row.expand(5, 64), wide.as_strided((5, 64), (8, 1)), wide.as_strided((2, 64), (56, 1))):
        with pytest.raises(ValueError):
            binding._rows(OnTheGpu(t), BF, "x", tuple(t.shape))
    for t, stride in ((wide[:, :64], 72), (wide, 72), (row, 0), (row.expand(1, 64), 0), (wide[:1], 0)):  # a row alone has no next one
        assert binding._rows(OnTheGpu(t), BF, "x", tuple(t.shape)) == (t.data_ptr(), stride)


def arguments(T, dtype, seed=1):
    g = ref.seeded(seed)
    x, y = ref.normal(g, (T, 128), dtype), ref.normal(g, (T, 64), dtype)
    a, b = ref.normal(g, (3, 16, 128), dtype, 128 ** -0.5), ref.normal(g, (3, 64, 16), dtype, 0.25)
    return x, y, a, b, (torch.arange(T, device="cuda") % 4 - 1).int()


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T", [2, 5, 300, 700])
def test_broadcast_rows_are_refused(monkeypatch, native, dtype, T):
    x, y, a, b, which = arguments(T, dtype)
    binding.load()
    assert binding._host_calls is not None
    if not native:
        monkeypatch.setattr(binding, "_host_calls", None)
    out = torch.full((T + 2, 64), 9.0, dtype=dtype, device="cuda")
    ws = torch.zeros(max(binding.linear_adapters_workspace_bytes(T, 16), 16), dtype=torch.uint8, device="cuda")
    for kw in (dict(x=x[:1].expand(T, 128)), dict(y=y[:1].expand(T, 64)), dict(y=y[0].expand(T, 64)), dict(o=out[1:2].expand(T, 64)),
               dict(x=x.view(-1).as_strided((T, 128), (64, 1))), dict(y=y.view(-1).as_strided((T, 64), (8, 1))),
               dict(y=out[1:2].expand(T, 64), o=out[1:2].expand(T, 64))):
        args = dict(x=x, y=y, o=out[1:-1]) | kw
        for workspace in (None, ws):
            with pytest.raises(ValueError):
                binding.linear_adapters(args["x"], args["y"], a, b, which, out=args["o"], workspace=workspace)
    assert (out == 9).all()
    binding.check_status()


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("T", [1, 5, 700])
def test_what_stands_for_them_is_taken(monkeypatch, native, T):
    """The rows written out; and a row alone, whatever its stride."""
    x, y, a, b, which = arguments(T, BF, seed=2)
    binding.load()
    if not native:
        monkeypatch.setattr(binding, "_host_calls", None)
    bias = y[:1]
    want = binding.linear_adapters(x, bias.repeat(T, 1), a, b, which)
    if T == 1:
        which = which + 1
        want = binding.linear_adapters(x, bias, a, b, which)
        assert torch.equal(binding.linear_adapters(x.expand(1, 128), bias.expand(1, 64), a, b, which, out=torch.empty_like(want).expand(1, 64)), want)
        assert not torch.equal(want, bias)
    else:
        assert torch.equal(want, binding.linear_adapters(x, bias.expand(T, 64).contiguous(), a, b, which, out=torch.empty_like(y)))
    binding.check_status()
