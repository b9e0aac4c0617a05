"""GPU parity: attention over a cache in pages with more than 8 query rows to a KV head and any number of KV heads, on both sides of where the rows are worked
on in parts, against the definition in 64 bits."""
import pytest
import torch

import kv_reference as ref
import test_parity_kv_pages as pages_tests
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF, I8, E4 = torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn


@pytest.mark.parametrize("dtype,form", [(BF, BF), (HF, HF), (HF, I8), (BF, E4)], ids=["bf16", "f16", "f16-int8", "bf16-e4m3"])
@pytest.mark.parametrize("B,Hkv", [(1, 1), (33, 1), (17, 4), (40, 8)])
@pytest.mark.parametrize("G,D", [(9, 128), (10, 64), (16, 128), (16, 80), (24, 128), (32, 128)])
def test_single_tokens(dtype, form, B, Hkv, G, D):
    lens = [(b * 37 + 5) % 331 if b % 7 else (0, 1, 330)[b % 3] for b in range(B)]
    pages_tests.check_decode(91, dtype, form, G * Hkv, Hkv, D, lens, 336, 16)


@pytest.mark.parametrize("dtype,form", [(BF, BF), (HF, I8)], ids=["bf16", "f16-int8"])
@pytest.mark.parametrize("B,Hkv", [(2, 2), (12, 4)])
@pytest.mark.parametrize("G,T", [(4, 4), (4, 3), (2, 7), (8, 4)])
def test_trees(dtype, form, B, Hkv, G, T):
    g = ref.seeded(92)
    Smax, D, P = 192, 128, 32
    cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding)
    paged, table = pages_tests.paged(g, cache, P)
    n = pages_tests.i32([(b * 41) % (Smax - T) for b in range(B)])
    q, sees = ref.normal(g, (B, G * Hkv, T, D), dtype), ref.random_tree(g, B, T)
    out = binding.attn_tree_pages(q, paged, table, n, ref.tree_bits(sees))
    binding.check_status()
    want, bound = ref.attention(q, cache, n, sees)
    ref.assert_within(out, want, bound)
