"""GPU parity: what a row of the cache may and may not do to the tokens of attn_decode_kv and attn_tree, whatever it holds; against the
definition in 64 bits with the bound that the roundings give."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF, I8, E4 = torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn
FORMS = [(BF, BF), (HF, HF), (BF, I8), (HF, I8), (BF, E4), (HF, E4)]
IDS = ["bf16", "f16", "bf16-int8", "f16-int8", "bf16-e4m3", "f16-e4m3"]


def lens_of(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def run_tree(q, cache, lens, tree=None, **kw):
    out = binding.attn_tree(q, cache, lens, tree, **kw)
    binding.check_status()
    return out


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("B,Hq,Hkv,T", [(60, 32, 8, 5), (45, 12, 12, 16)])
def test_not_a_number_in_every_item_of_a_long_run(dtype, form, B, Hq, Hkv, T):
    """Several items follow one another on each SM, and each has drafted rows of V that some of its tokens see and that are no
    numbers: every one of them reaches its tokens, and no other."""
    g = ref.seeded(61)
    lens = [(13 * b) % 40 for b in range(B)]
    cache = ref.make_cache(g, B, Hkv, 64, 64, form, binding)
    q, n = ref.normal(g, (B, Hq, T, 64), dtype), lens_of(lens)
    sees = torch.eye(T, dtype=torch.bool, device="cuda")
    sees[:, 0] = True
    bits = ref.tree_bits(sees)[None]
    before = run_tree(q, cache, n, bits)
    for b in range(B):  # the row of token 1 + b % (T - 1)
        (cache.v if cache.v_scale is None else cache.v_scale)[b, :, lens[b] + 1 + b % (T - 1)] = float("nan")
    hit = torch.zeros((B, T), dtype=torch.bool, device="cuda")
    for b in range(B):
        hit[b, 1 + b % (T - 1)] = True
    for _ in range(5):
        after = run_tree(q, cache, n, bits)
        assert torch.equal(after.isnan().all(-1), hit[:, None].expand(B, Hq, T))
        assert torch.equal(torch.where(hit[:, None, :, None], before, after), before)
