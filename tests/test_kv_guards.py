"""Nothing is written outside the outputs and the workspace of the operators around the KV cache: each lies between two
sentinel-filled guard regions, which have to be untouched; what is inside is compared with a call into ordinary buffers."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding
from util import Guarded

pytestmark = pytest.mark.gpu

BF, HF, I8, E4 = torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn
FORMS = [(BF, BF), (HF, HF), (BF, I8), (HF, E4)]
IDS = ["bf16", "f16", "bf16-int8", "f16-e4m3"]


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def workspace(B, Hq, Hkv, T, D):
    g = Guarded((binding.attn_kv_workspace_bytes(B, Hq, Hkv, T, D),), torch.uint8)
    binding.attn_kv_workspace_init(g.tensor)
    return g


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("B,Hq,Hkv,D,T,lens", [
    (3, 8, 2, 128, 1, [0, 1, 700]), (2, 12, 12, 64, 1, [333, 18]), (1, 8, 1, 80, 1, [9000]), (300, 4, 2, 16, 1, None),   # up to 8 rows
    (3, 8, 2, 128, 5, [0, 1, 700]), (2, 28, 4, 64, 16, [333, 18]), (1, 16, 1, 112, 1, [9000]), (1, 32, 8, 128, 64, [2000]), (90, 12, 2, 16, 7, None),
])
def test_attention_and_its_workspace_stay_inside(dtype, form, B, Hq, Hkv, D, T, lens):
    g = ref.seeded(81)
    lens = [(37 * b) % 200 for b in range(B)] if lens is None else lens
    cache = ref.make_cache(g, B, Hkv, max(lens) + T, D, form, binding)
    q, n = ref.normal(g, (B, Hq, T, D), dtype), ints(lens)
    out, ws = Guarded((B, Hq, T, D), dtype), workspace(B, Hq, Hkv, T, D)
    want = binding.attn_tree(q, cache, n)
    for _ in range(2):
        binding.attn_tree(q, cache, n, out=out.tensor, workspace=ws.tensor)
        binding.check_status()
        assert torch.equal(out.tensor, want)
        out.assert_intact()
        ws.assert_intact()
        out.tensor.fill_(float("nan"))
    if T == 1:
        want = binding.attn_decode_kv(q[:, :, 0].contiguous(), cache, n)
        binding.attn_decode_kv(q[:, :, 0].contiguous(), cache, n, out=out.tensor[:, :, 0], workspace=ws.tensor)
        binding.check_status()
        assert torch.equal(out.tensor[:, :, 0], want)
        out.assert_intact()
        ws.assert_intact()
    assert bool((ws.tensor[:262144] == 0).all())  # the counters, as the next call expects them


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("B,Hkv,S,D", [(1, 1, 1, 16), (3, 2, 77, 80), (2, 4, 130, 128), (1, 3, 1025, 64)])
def test_rows_read_back_stay_inside(dtype, form, B, Hkv, S, D):
    g = ref.seeded(82)
    cache = ref.make_cache(g, B, Hkv, S + 9, D, form, binding)
    outs = [Guarded((B, Hkv, S, D), dtype) for _ in range(2)]
    binding.kv_read(cache, *(o.tensor for o in outs), first=ints([9 - b for b in range(B)]))
    for o, codes, scale in zip(outs, (cache.k, cache.v), (cache.k_scale, cache.v_scale)):
        values = ref.decode_values(codes, scale)
        for b in range(B):
            want = values[b, :, 9 - b: 9 - b + S]
            assert ((o.tensor[b].double() - want).abs() <= want.abs() * (ref.HALF[dtype] + 2 * ref.F32) + 2.0 ** -25).all()
        o.assert_intact()


@pytest.mark.parametrize("dtype", [BF, HF, torch.float32])
@pytest.mark.parametrize("B,H,S,D,dims,layout", [(1, 1, 1, 8, 8, 0), (2, 3, 7, 80, 40, 0), (1, 5, 33, 256, 254, 1), (3, 40, 1, 128, 128, 0), (1, 2, 65, 96, 34, 0)])
def test_rotation_stays_inside(dtype, B, H, S, D, dims, layout):
    g = ref.seeded(83)
    f, _ = binding.rotary_frequencies(dims)
    r = binding.Rotary(f.cuda(), layout)
    x, out = ref.normal(g, (B, H, S, D), dtype), Guarded((B, H, S, D), dtype)
    binding.rotary_apply(x, r, out=out.tensor)
    assert torch.equal(out.tensor, binding.rotary_apply(x, r))
    out.assert_intact()


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("S,D,lens", [(1, 128, [0, 39]), (7, 80, [33, 36]), (130, 64, [0, 3])])
def test_appended_rows_and_rotated_queries_stay_inside(dtype, form, S, D, lens):
    """The cache is as full as it gets: its last rows are the last bytes of the buffers."""
    g = ref.seeded(84)
    B, Hq, Hkv, Smax = 2, 6, 2, max(lens) + S - 2 if S > 2 else 40
    kv = [Guarded((B, Hkv, Smax, D), form) for _ in range(2)]
    scales = [Guarded((B, Hkv, Smax), torch.float32) for _ in range(2)] if form in ref.TOP else []
    cache = binding.KVCache(*(x.tensor for x in kv + scales))
    f, _ = binding.rotary_frequencies(D)
    q, k, v = (ref.normal(g, (B, h, S, D), dtype) for h in (Hq, Hkv, Hkv))
    q_out = Guarded((B, Hq, S, D), dtype)
    binding.kv_append(cache, k, v, ints(lens), rotary=binding.Rotary(f.cuda()), q=q, q_out=q_out.tensor)
    want = binding.rotary_apply(q, binding.Rotary(f.cuda()), first=ints(lens))
    assert torch.equal(q_out.tensor, want)
    for x in (*kv, *scales, q_out):
        x.assert_intact()
