"""GPU parity: low-rank adapters of many tokens on several streams at once, beside one another and beside other operators, each with a workspace of its own."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def make(seed, dtype, T, n, rank, K, N, runs):
    g = ref.seeded(seed)
    x, y = ref.normal(g, (T, K), dtype), ref.normal(g, (T, N), dtype)
    a, b = ref.normal(g, (n, rank, K), dtype, K ** -0.5), ref.normal(g, (n, N, rank), dtype, rank ** -0.5)
    return x, y, a, b, (torch.arange(T, device="cuda") // runs % (n + 1) - 1).int()


@pytest.mark.parametrize("calls", [((700, 3, 16, 512, 512, 40), (650, 20, 16, 512, 1024, 1)), ((2000, 5, 128, 256, 512, 300), (900, 2, 64, 1024, 512, 90)),
                                   ((4000, 5, 32, 512, 2048, 500), (48, 40, 16, 1024, 1024, 1), (1300, 9, 24, 512, 520, 7))],
                         ids=["tiles-groups", "ranks", "three"])
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("captured", [False, True])
def test_calls_on_streams(dtype, calls, captured):
    sets = [make(31 + i, dtype, *c) for i, c in enumerate(calls)]
    want = [binding.linear_adapters(*s) for s in sets]
    spaces = [torch.empty(max(binding.linear_adapters_workspace_bytes(c[0], c[2]), 16), dtype=torch.uint8, device="cuda") for c in calls]
    outs = [[torch.zeros_like(w) for _ in range(4)] for w in want]
    streams = [torch.cuda.Stream() for _ in calls]
    g = ref.seeded(30)
    w, h = ref.normal(g, (512, 1024), dtype, 0.04), ref.normal(g, (300, 512), dtype)
    linear = binding.linear_act(h, w, act=binding.ACT_NONE)
    beside = [torch.zeros_like(linear) for _ in range(4)]
    torch.cuda.synchronize()
    graphs = []
    if captured:
        for i, s in enumerate(sets):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                for o in outs[i]:
                    binding.linear_adapters(*s, out=o, workspace=spaces[i])
        torch.cuda.synchronize()
    for turn in range(4):
        for i, s in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                if captured:
                    graphs[i].replay()
                else:
                    binding.linear_adapters(*s, out=outs[i][turn], workspace=spaces[i])
        binding.linear_act(h, w, act=binding.ACT_NONE, out=beside[turn])
    torch.cuda.synchronize()
    binding.check_status()
    for w_, os in zip(want, outs):
        assert all(torch.equal(o, w_) for o in os)
    assert all(torch.equal(o, linear) for o in beside)
