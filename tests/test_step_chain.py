"""GPU parity: steps of a server one behind the other, with no other kernel between them: room for a token of each request (the lengths in place), its row into
the cache in pages, attention of the query that the same call rotated.  Each step's output is that over caches in one block, bit for bit."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF, I8, E4 = torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn
STEPS = 30


@pytest.mark.parametrize("dtype,form", [(BF, BF), (HF, I8), (BF, E4)], ids=["bf16", "f16-int8", "bf16-e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (4, 4, 128), (22, 1, 128)])  # up to 8 query rows to a KV head, and more
@pytest.mark.parametrize("B", [1, 3, 40])
@pytest.mark.parametrize("captured", [False, True])
def test_steps_without_a_kernel_between(dtype, form, Hq, Hkv, D, B, captured):
    g = ref.seeded(81)
    P, max_pages = 16, 10
    fmt = binding._KV_TYPES.index(form)
    pages = binding.KVPages.empty(B * max_pages, Hkv, P, D, fmt)
    tables = binding.PageTables.empty(B, max_pages, B * max_pages, P)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    slots, positions = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    step_slots = binding.PageSlots(lens, None, slots, positions)  # the lengths grow in place
    rotary = binding.Rotary(binding.rotary_frequencies(D)[0].cuda())
    ws = torch.zeros(binding.attn_kv_workspace_bytes(B, Hq, Hkv, 1, D), dtype=torch.uint8, device="cuda")
    qkv = ref.normal(g, (STEPS, B, Hq + 2 * Hkv, D), dtype)
    q_out, out = (torch.zeros((STEPS, B, Hq, D), dtype=dtype, device="cuda") for _ in range(2))
    parts = [qkv[i].split([Hq, Hkv, Hkv], 1) for i in range(STEPS)]

    def run():
        for i, (q, k, v) in enumerate(parts):
            binding.assign_pages(tables, lens, step_slots)
            binding.kv_append_pages(pages, k, v, slots, positions=positions, rotary=rotary, q=q, q_out=q_out[i])
            binding.attn_decode_pages(q_out[i], pages, tables.table, lens, out=out[i], workspace=ws)

    # a first round fills what a call makes once; its rows stay behind, as a page's old rows do
    run()
    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
    start = torch.randint(0, 40, (B,), generator=g, device="cuda", dtype=torch.int32)
    fresh = binding.PageTables.empty(B, max_pages, B * max_pages, P)
    for have, want in ((tables.table, fresh.table), (tables.free_pages, fresh.free_pages), (tables.free_count, fresh.free_count)):
        have.copy_(want)
    # rows before the first step
    T0 = int(start.sum())
    lens.zero_()
    flat = binding.KVCache.empty(B, Hkv, P * max_pages, D, fmt)
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    if T0:
        first = binding.PageSlots.empty(B, T0)
        binding.assign_pages(tables, lens, first, counts=start)
        k0, v0 = (ref.normal(g, (B, Hkv, 40, D), dtype) for _ in range(2))
        at = (first.requests.long(), slice(None), first.positions.long())
        binding.kv_append_pages(pages, k0[at].contiguous(), v0[at].contiguous(), first.slots, positions=first.positions, rotary=rotary)
        binding.kv_append(flat, k0, v0, zero, counts=start, rotary=rotary)
    for turn in range(2):
        lens.copy_(start + turn * STEPS)
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay() if captured else run()
        torch.cuda.synchronize()
        assert torch.equal(lens, start + (turn + 1) * STEPS)
        n = start + turn * STEPS
        for i, (q, k, v) in enumerate(parts):
            turned = binding.kv_append(flat, k[:, :, None], v[:, :, None], n, rotary=rotary, q=q[:, :, None], q_out=torch.empty((B, Hq, 1, D), dtype=dtype, device="cuda"))
            n = n + 1
            assert torch.equal(q_out[i], turned[:, :, 0]), (turn, i)
            want = binding.attn_decode_kv(turned[:, :, 0].contiguous(), flat, n)
            assert torch.equal(out[i].view(torch.int16), want.view(torch.int16)), (turn, i)
    binding.check_status()
