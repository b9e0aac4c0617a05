"""Plain calls of a step of many requests are taken by the native marshalling: none of them is handed back to the general way."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF, I8, E4 = torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn
NAMES = ("assign_pages", "append_pages", "read_pages", "decode_pages", "tree_pages", "adapters")


class Counting:
    """The native module, with the answers of its calls kept."""

    def __init__(self, module):
        self.module, self.answers = module, {}

    def __getattr__(self, name):
        fn = getattr(self.module, name)

        def call(*a):
            st = fn(*a)
            self.answers.setdefault(name, []).append(st)
            return st
        return call


@pytest.mark.parametrize("dtype,form", [(BF, BF), (HF, HF), (HF, I8), (BF, E4)], ids=["bf16", "f16", "f16-int8", "bf16-e4m3"])
def test_plain_calls_are_taken(monkeypatch, dtype, form):
    binding.load()
    native = Counting(binding._host_calls)
    monkeypatch.setattr(binding, "_host_calls", native)
    g = ref.seeded(61)
    B, Hq, Hkv, D, P, T, num = 3, 6, 2, 64, 16, 9, 20
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    pages = binding.KVPages.empty(num, Hkv, P, D, binding._KV_TYPES.index(form))
    tables, step = binding.PageTables.empty(B, 5, num, P), binding.PageSlots.empty(B, T)
    rotary = binding.Rotary(binding.rotary_frequencies(D)[0].cuda())
    ws = torch.zeros(binding.attn_kv_workspace_bytes(B, Hq, Hkv, 8, D), dtype=torch.uint8, device="cuda")
    qkv = ref.normal(g, (T, Hq + 2 * Hkv, D), dtype)
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    n = i32([0, 4, 30])
    binding.assign_pages(tables, n, step, counts=i32([3, 4, 2]), free_left=i32([0]))
    binding.assign_pages(tables, n, step)
    binding.assign_pages(tables, step.lens, step)
    binding.kv_append_pages(pages, k, v, step.slots, positions=step.positions, rotary=rotary, q=q, q_out=torch.empty((T, Hq, D), dtype=dtype, device="cuda"))
    binding.kv_append_pages(pages, k, v, step.slots, positions=step.positions, rotary=rotary)
    binding.kv_append_pages(pages, k, v, step.slots)
    out = [torch.zeros((B, Hkv, 20, D), dtype=dtype, device="cuda") for _ in range(2)]
    binding.kv_read_pages(pages, tables.table, *out, first=i32([0, 1, 2]), counts=i32([3, 3, 3]))
    binding.kv_read_pages(pages, tables.table, *out)
    q1, qt = ref.normal(g, (B, Hq, D), dtype), ref.normal(g, (B, 8, Hq, D), dtype).transpose(1, 2)
    for scale in (None, 0.25):
        binding.attn_decode_pages(q1, pages, tables.table, step.lens, scale=scale, out=torch.empty_like(q1), workspace=ws)
        binding.attn_tree_pages(qt, pages, tables.table, n, scale=scale, out=torch.empty_like(qt), workspace=ws)
    bits = ref.tree_bits(ref.random_tree(g, B, 8))
    for tree in (bits, bits[:1].contiguous()):
        binding.attn_tree_pages(qt, pages, tables.table, n, tree, out=torch.empty_like(qt), workspace=ws)
    for tokens in (T, 600):
        wide = ref.normal(g, (tokens, 400), dtype)
        x, y = wide[:, :128], wide[:, 136:200]
        a, b = ref.normal(g, (4, 8, 128), dtype), ref.normal(g, (4, 64, 8), dtype)
        which, aws = torch.arange(tokens, device="cuda").int() % 5 - 1, torch.empty(binding.linear_adapters_workspace_bytes(600, 8), dtype=torch.uint8, device="cuda")
        o = torch.empty((tokens, 64), dtype=dtype, device="cuda")
        binding.linear_adapters(x, y, a, b, which, out=o, workspace=aws)
        binding.linear_adapters(x, y, a, b, which, scales=torch.ones(4, device="cuda"), out=o, workspace=aws)
        binding.linear_adapters(x, y, a, b, i32([0, 3, -1]), requests=torch.arange(tokens, device="cuda").int() % 3, out=y, workspace=aws)
    binding.linear_adapters(x[:1], y[:1], a, b, i32([2]), out=o[:1])
    binding.check_status()
    assert {name: native.answers.get(name) for name in NAMES} == {
        "assign_pages": [0] * 3, "append_pages": [0] * 3, "read_pages": [0] * 2, "decode_pages": [0] * 2, "tree_pages": [0] * 4, "adapters": [0] * 7}
