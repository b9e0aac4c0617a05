"""GPU parity: attention of single tokens and of trees of drafted tokens over caches of 16-bit and 8-bit rows, against the
definition in 64 bits with the bound that its roundings give (kv_reference.py)."""
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


def run_decode(q, cache, lens, **kw):
    out = binding.attn_decode_kv(q, cache, lens, **kw)
    binding.check_status()
    return out


def run_tree(q, cache, lens, tree=None, **kw):
    out = binding.attn_tree(q, cache, lens, tree, **kw)
    binding.check_status()
    return out


def check_decode(seed, dtype, form, Hq, Hkv, D, lens, Smax, scale=None, spread=1.0):
    g = ref.seeded(seed)
    B = len(lens)
    cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding, spread)
    q = ref.normal(g, (B, Hq, D), dtype)
    n = lens_of(lens)
    want, bound = ref.attention(q[:, :, None], cache, n, scale=scale)
    ref.assert_within(run_decode(q, cache, n, scale=scale), want[:, :, 0], bound[:, :, 0])


def check_tree(seed, dtype, form, Hq, Hkv, D, T, lens, Smax, scale=None, sees=None):
    g = ref.seeded(seed)
    B = len(lens)
    cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding)
    q = ref.normal(g, (B, Hq, T, D), dtype)
    n = lens_of(lens)
    sees = ref.random_tree(g, B, T) if sees is None else sees(g, B, T)
    want, bound = ref.attention(q, cache, n, sees, scale)
    ref.assert_within(run_tree(q, cache, n, ref.tree_bits(sees), scale=scale), want, bound)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (12, 12, 64), (14, 2, 128), (4, 4, 16), (6, 2, 80), (3, 1, 96)])
def test_decode_around_tile_borders(dtype, form, Hq, Hkv, D):
    check_decode(11, dtype, form, Hq, Hkv, D, [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300], 300)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("B,Hq,Hkv,D,Smax", [(1, 8, 8, 64, 40000), (1, 32, 8, 128, 33333), (2, 16, 1, 128, 9001), (1, 1, 1, 128, 1)])
def test_decode_of_few_long_sequences(dtype, form, B, Hq, Hkv, D, Smax):
    check_decode(12, dtype, form, Hq, Hkv, D, [Smax - 7 * b for b in range(B)], Smax)


@pytest.mark.parametrize("dtype,form", [FORMS[0], FORMS[2], FORMS[5]], ids=[IDS[0], IDS[2], IDS[5]])
@pytest.mark.parametrize("B", [32, 33, 64, 97, 300])
def test_decode_of_many_sequences(dtype, form, B):
    lens = [(37 * b * b + 11 * b) % 311 for b in range(B)]
    check_decode(13, dtype, form, 4, 2, 64, lens, 310)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,Hkv,T", [(32, 8, 5), (4, 4, 1), (12, 12, 16), (14, 2, 3), (8, 2, 17), (28, 4, 16), (8, 1, 33), (32, 8, 64)])
def test_trees(dtype, form, Hq, Hkv, T):
    check_tree(21, dtype, form, Hq, Hkv, 128, T, [0, 1, 100, 128 - T, 127, 128, 500, 600 - T], 600)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("D", [16, 64, 80, 112])
def test_trees_of_other_head_sizes(dtype, form, D):
    check_tree(22, dtype, form, 8, 2, D, 9, [3, 200, 130], 257)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_masks_with_any_bits(dtype, form):
    """Not only trees: any token may see any of the others, or none of them."""
    def sees(g, B, T):
        m = torch.rand((B, T, T), generator=g, device="cuda") < 0.3
        m[:, 2] = False
        m[0, T - 1] = True
        return m
    check_tree(23, dtype, form, 8, 2, 128, 40, [0, 0, 77, 128, 511], 560, sees=sees)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_rows_beyond_the_cache_are_not_there(dtype, form):
    """T tokens behind more rows than leave room for theirs; lengths outside the cache count as its ends."""
    check_tree(24, dtype, form, 8, 2, 64, 12, [150, 145, 1000, -5], 150)
    check_decode(25, dtype, form, 8, 2, 64, [150, 151, 100000, -1], 150)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_no_mask_is_a_chain_and_one_mask_serves_all(dtype, form):
    g = ref.seeded(26)
    B, Hq, Hkv, T, D, Smax = 3, 8, 2, 11, 128, 300
    cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding)
    q, n = ref.normal(g, (B, Hq, T, D), dtype), lens_of([5, 250, 120])
    chain = torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
    bits = ref.tree_bits(chain)
    a = run_tree(q, cache, n)
    want, bound = ref.attention(q, cache, n, chain.expand(B, T, T))
    ref.assert_within(a, want, bound)
    assert torch.equal(a, run_tree(q, cache, n, bits[None]))
    assert torch.equal(a, run_tree(q, cache, n, bits[None].expand(B, T).contiguous()))
    assert torch.equal(a, run_tree(q, cache, n, bits[None] | (-1 << T)))  # bits from T on say nothing


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_a_chain_is_one_token_after_the_other(dtype, form):
    """The t-th token of a chain sees what a single token with t + 1 more rows sees."""
    g = ref.seeded(27)
    cache = ref.make_cache(g, 2, 2, 400, 128, form, binding)
    q, n = ref.normal(g, (2, 8, 6, 128), dtype), lens_of([300, 126])
    out = run_tree(q, cache, n)
    for t in range(6):
        m = n + t + 1
        _, bound = ref.attention(q[:, :, t:t + 1].contiguous(), cache, m)
        one = run_decode(q[:, :, t].contiguous(), cache, m)
        assert ((out[:, :, t].double() - one.double()).abs() <= 2 * bound[:, :, 0]).all()


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-3, 3.0])
def test_scales(dtype, form, scale):
    check_decode(31, dtype, form, 8, 2, 128, [1, 200, 129], 200, scale=scale)
    check_tree(32, dtype, form, 8, 2, 64, 5, [0, 120, 33], 200, scale=scale)


@pytest.mark.parametrize("dtype,form", FORMS[2:], ids=IDS[2:])
def test_rows_of_very_different_sizes(dtype, form):
    check_decode(33, dtype, form, 8, 2, 128, [513, 200, 40], 520, scale=0.01, spread=100.0)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_large_and_small_queries(dtype, form):
    """Queries at the ends of their type's range: only their products with the scale are ordinary numbers."""
    g = ref.seeded(34)
    cache = ref.make_cache(g, 1, 2, 150, 64, form, binding)
    base = torch.randn((1, 4, 64), generator=g, device="cuda")
    for size in (2.0 ** 12, 2.0 ** -12) if dtype == HF else (2.0 ** 100, 2.0 ** -100):
        q = (base * size).to(dtype)
        scale = 0.125 / size
        want, bound = ref.attention(q[:, :, None], cache, lens_of([150]), scale=scale)
        ref.assert_within(run_decode(q, cache, lens_of([150]), scale=scale), want[:, :, 0], bound[:, :, 0] + abs(want[:, :, 0]) * 2 ** -9)


def poison(cache, b, rows):
    """NaN and infinities in some rows of sequence b."""
    for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        if s is None:
            t[b, :, rows] = float("nan")
            t[b, :, rows, ::3] = float("inf")
        else:
            s[b, :, rows] = float("nan")


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("D", [64, 128])
def test_rows_behind_the_last_may_hold_anything(dtype, form, D):
    g = ref.seeded(41)
    cache = ref.make_cache(g, 3, 2, 300, D, form, binding)
    q, n = ref.normal(g, (3, 8, D), dtype), lens_of([5, 129, 290])
    qt = ref.normal(g, (3, 8, 7, D), dtype)
    before, tree = run_decode(q, cache, n), run_tree(qt, cache, n - 3)
    sees = torch.ones((7, 7), dtype=torch.bool, device="cuda").tril()
    sees[:, 3:] = False  # row lens[b] and what follows: nobody sees them
    tree = run_tree(qt, cache, n - 3, ref.tree_bits(sees)[None])
    for b in range(3):
        poison(cache, b, slice(int(n[b]), 300))
    assert torch.equal(before, run_decode(q, cache, n))
    assert torch.equal(tree, run_tree(qt, cache, n - 3, ref.tree_bits(sees)[None]))


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,T", [(2, 6), (8, 40)])
def test_a_row_that_is_not_a_number_reaches_those_who_see_it_and_no_others(dtype, form, Hq, T):
    g = ref.seeded(42)
    for past in (40, 125):
        cache = ref.make_cache(g, 2, 2, 300, 128, form, binding)
        q, n = ref.normal(g, (2, Hq, T, 128), dtype), lens_of([past, past])
        sees = torch.eye(T, dtype=torch.bool, device="cuda")
        sees[:, 0] = True
        bits = ref.tree_bits(sees)[None]
        before = run_tree(q, cache, n, bits)
        poison(cache, 0, slice(past + 3, past + 4))
        after = run_tree(q, cache, n, bits)
        assert after[0, :, 3].isnan().all()
        after[0, :, 3] = before[0, :, 3]
        assert torch.equal(before, after)
        poison(cache, 1, slice(7, 8))
        after = run_tree(q, cache, n, bits)
        assert after[1].isnan().all() and torch.equal(after[0].isnan().any(-1).any(0), torch.arange(T, device="cuda") == 3)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_views(dtype, form):
    """Queries in a fused projection's output, outputs token by token as the output projection reads them; what lies between
    stays as it was."""
    g = ref.seeded(51)
    B, Hq, Hkv, T, D = 2, 8, 2, 13, 64
    cache = ref.make_cache(g, B, Hkv, 200, D, form, binding)
    qkv = ref.normal(g, (B, T, Hq + 2 * Hkv, D), dtype)
    out = torch.full((B, T, Hq + 1, D), 7.0, dtype=dtype, device="cuda")
    q, n = qkv[:, :, :Hq].permute(0, 2, 1, 3), lens_of([150, 30])
    got = run_tree(q, cache, n, out=out[:, :, :Hq].permute(0, 2, 1, 3))
    assert torch.equal(got, run_tree(q.contiguous(), cache, n))
    assert (out[:, :, Hq] == 7).all()


@pytest.mark.parametrize("dtype,form", [FORMS[0], FORMS[3]], ids=[IDS[0], IDS[3]])
def test_one_workspace_serves_calls_of_other_shapes_and_the_same_bits_come_again(dtype, form):
    g = ref.seeded(52)
    ws = torch.empty(binding.attn_kv_workspace_bytes(8, 32, 8, 64, 128), dtype=torch.uint8, device="cuda")
    binding.attn_kv_workspace_init(ws)
    cases = []
    for B, Hq, Hkv, T, D, Smax in [(8, 32, 8, 64, 128, 700), (1, 8, 8, 1, 64, 5000), (5, 8, 1, 20, 128, 900), (3, 4, 2, 1, 64, 17)]:
        cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding)
        q = ref.normal(g, (B, Hq, T, D), dtype)
        cases.append((q, cache, lens_of([Smax - T - b for b in range(B)])))
    first = [binding.attn_tree(*c, workspace=ws).clone() for c in cases]
    for _ in range(3):
        for c, f in zip(cases, first):
            assert torch.equal(f, binding.attn_tree(*c, workspace=ws))
    binding.check_status()
    for c, f in zip(cases, first):
        assert torch.equal(f, run_tree(*c))


def test_offsets_beyond_32_bits():
    """A cache of 2.2e9 elements: its last rows lie behind 2^31 of them."""
    B, Hkv, D, Smax = 2, 1, 128, 8_600_000
    g = ref.seeded(53)
    store = [torch.zeros((B, Hkv, Smax, D), dtype=I8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((B, Hkv, Smax), device="cuda") for _ in range(2)]
    tail = 300
    for t, s in zip(store, scales):
        c, sc = ref.quantise(torch.randn((B, Hkv, tail, D), generator=g, device="cuda"), I8)
        t[:, :, -tail:], s[:, :, -tail:] = c, sc
    q = ref.normal(g, (B, 4, D), BF)
    # the other rows have score 0 and value 0: each weighs exp(0)
    small = binding.KVCache(*(t[:, :, -tail:].contiguous() for t in store), *(s[:, :, -tail:].contiguous() for s in scales))
    s = torch.einsum("bhd,bjd->bhj", q.double(), ref.decode_values(small.k, small.k_scale)[:, 0]) * D ** -0.5 * 20
    w = s.exp()
    want = torch.einsum("bhj,bjd->bhd", w, ref.decode_values(small.v, small.v_scale)[:, 0]) / (w.sum(-1) + Smax - tail)[..., None]
    out = run_decode(q, binding.KVCache(*store, *scales), lens_of([Smax, Smax]), scale=D ** -0.5 * 20)
    # probabilities and outputs rounded as elsewhere; the zeros' sum is of 8.6e6 equal terms in fp32, spread over 148 * 32 partial sums
    bound = 2 ** -8 * want.abs() + (2 ** -11 + 2 ** -9) * torch.einsum("bhj,bjd->bhd", w, ref.decode_values(small.v, small.v_scale)[:, 0].abs()) / (w.sum(-1) + Smax - tail)[..., None] + 1e-9
    assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype,form", [FORMS[0], FORMS[4]], ids=[IDS[0], IDS[4]])
def test_captured_and_replayed_with_new_lengths(dtype, form):
    g = ref.seeded(54)
    cache = ref.make_cache(g, 4, 2, 900, 128, form, binding)
    q, n = ref.normal(g, (4, 8, 9, 128), dtype), lens_of([10, 20, 30, 40])
    ws = torch.zeros(binding.attn_kv_workspace_bytes(4, 8, 2, 9, 128), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    binding.attn_tree(q, cache, n, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.attn_tree(q, cache, n, out=out, workspace=ws)
    for lens in ([10, 20, 30, 40], [0, 891, 500, 127], [300, 1, 0, 890]):
        n.copy_(lens_of(lens))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, run_tree(q, cache, n))


def test_two_streams_with_a_workspace_each():
    g = ref.seeded(55)
    caches = [ref.make_cache(g, 4, 8, 2000, 128, I8, binding) for _ in range(2)]
    qs = [ref.normal(g, (4, 32, 128), BF) for _ in range(2)]
    n = lens_of([2000, 1500, 3, 777])
    want = [run_decode(q, c, n) for q, c in zip(qs, caches)]
    ws = [torch.zeros(binding.attn_kv_workspace_bytes(4, 32, 8), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.empty_like(q) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                binding.attn_decode_kv(qs[i], caches[i], n, out=outs[i], workspace=ws[i])
    torch.cuda.synchronize()
    binding.check_status()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("B,Hq,Hkv,D", [(5, 12, 4, 128), (40, 6, 3, 64), (37, 12, 1, 128), (49, 3, 3, 80)])
def test_sequences_of_nearly_the_same_length(dtype, form, B, Hq, Hkv, D):
    """No more (sequence, KV head) pairs than CTAs, and of lengths that are not worth sharing, with some without rows."""
    lens = [0 if b % 13 == 5 else 260 - (7 * b) % 60 for b in range(B)]
    check_decode(31, dtype, form, Hq, Hkv, D, lens, 270)
    check_tree(32, dtype, form, Hq, Hkv, D, 5, lens, 270)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,D,T", [(8, 128, 1), (4, 64, 2), (24, 64, 1), (16, 128, 3)])
def test_one_kv_head_over_a_long_cache(dtype, form, Hq, D, T):
    """One item shared by many CTAs: as many parts as a merge is worth, of any length."""
    for lens in ([19999 - T], [4097], [1, 12000]):
        check_tree(33, dtype, form, Hq, 1, D, T, lens, 20000)
