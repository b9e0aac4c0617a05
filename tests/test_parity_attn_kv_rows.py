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


# ------------------------------------------------------------------------------------------------------- as close as it is said to be
def definition(q, cache, past, sees=None, scale=None):
    """q [B,Hq,T,D], the rows as in kv_reference.attention -> (out in 64 bits, bound), both from the rows that a token sees alone.
    Weights (softmax, times the row's scale with 8-bit rows) are rounded to the operands' type, and what that leaves once more: off by half a
    step of half a step, 2^-11 squared for 8-bit rows; for 16-bit ones, whose weights are rounded towards zero first, by half a step of a
    whole one, twice 2^-8 or 2^-11 squared.  In fp16 also by half of 2^-24, where the token's largest has come to 2^5 or more: 2^-30 of it;
    with 16-bit rows by 2^-24, where it has come to 2^6: as much.  The output is rounded once.  Scores and sums as in kv_reference.attention."""
    B, Hq, T, D = q.shape
    k, v = ref.decode_values(cache.k, cache.k_scale), ref.decode_values(cache.v, cache.v_scale)
    Smax, Hkv = k.shape[2], k.shape[1]
    G, eight = Hq // Hkv, cache.k_scale is not None
    scale = D ** -0.5 if scale is None else scale
    past = past.clamp(0, Smax)
    smallest = 2.0 ** -25 if q.dtype == HF else 2.0 ** -134  # half of the type's smallest number
    operand = torch.float16 if eight else q.dtype
    u = ref.HALF[operand] ** 2 * (1 if eight else 2)
    top = cache.v_scale.double().abs() * ref.TOP[cache.v.dtype] if eight else v.abs().amax(-1)  # of a row's elements
    out, bound = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        for t in range(T):
            rows = torch.arange(Smax, device="cuda") < past[b]
            if sees is not None:
                at = int(past[b])
                n = min(T, Smax - at)
                rows[at:at + n] = sees[b, t, :n]
            if not bool(rows.any()):
                continue
            kb, vb, tb = k[b][:, rows], v[b][:, rows], top[b][:, rows]
            x = q[b, :, t].double().view(Hkv, G, D)
            s = torch.einsum("hgd,hjd->hgj", x, kb) * scale
            mag = (torch.einsum("hgd,hjd->hgj", x.abs(), kb.abs()) * abs(scale)).amax(-1)
            w = torch.softmax(s, -1)
            o = torch.einsum("hgj,hjd->hgd", w, vb)
            wv = torch.einsum("hgj,hjd->hgd", w, vb.abs())
            if operand == BF:
                lost = 0.0
            elif eight:  # of the largest weight times its row
                lost = w.shape[-1] * 2.0 ** -30 * (w * tb[:, None]).amax(-1)
            else:        # of the largest weight, times any row
                lost = w.shape[-1] * 2.0 ** -30 * w.amax(-1) * tb.amax(-1)[:, None]
            e = (u + 2 * mag * (D + 8) * 2.0 ** -22 + 2.0 ** -17)[..., None] * wv + ref.HALF[q.dtype] * o.abs() * 1.01 + smallest
            out[b, :, t], bound[b, :, t] = o.view(Hq, D), (e + (lost if operand == BF else lost[..., None])).view(Hq, D)
    return out, bound


def run_decode(q, cache, lens, **kw):
    out = binding.attn_decode_kv(q, cache, lens, **kw)
    binding.check_status()
    return out


def assert_close(q, cache, lens, sees=None, scale=None, what=""):
    """The call for these tokens (a single one, with no rows of its own: decode)."""
    want, bound = definition(q, cache, lens, sees, scale)
    if sees is None:
        got = run_decode(q[:, :, 0].contiguous(), cache, lens, scale=scale)[:, :, None]
    else:
        got = run_tree(q, cache, lens, ref.tree_bits(sees), scale=scale)
    ref.assert_within(got, want, bound, what)


def rows_cache(k, v, form):
    """A cache of the rows k, v (fp32, finite)."""
    (k, ks), (v, vs) = (ref.quantise(x, form) if form in ref.TOP else (x.to(form), None) for x in (k, v))
    return binding.KVCache(k, v, ks, vs)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,T", [(2, 6), (8, 40)])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 100, float("inf")])
def test_the_size_of_a_row_that_is_not_seen_changes_nothing(dtype, form, Hq, T, size):
    g = ref.seeded(62)
    if dtype == HF and form == HF:
        size = min(size, 60000.0)
    for past in (0, 40, 125):
        cache = ref.make_cache(g, 2, 2, 300, 128, form, binding)
        q, n = ref.normal(g, (2, Hq, T, 128), dtype), lens_of([past, past])
        sees = torch.eye(T, dtype=torch.bool, device="cuda")
        sees[:, 0] = True
        bits = ref.tree_bits(sees)[None]
        before = run_tree(q, cache, n, bits)
        at = past + 3  # token 3 alone sees it
        if cache.v_scale is None:
            cache.k[:, :, at], cache.v[:, :, at] = 0, size
        else:
            cache.v_scale[:, :, at] = size
        after = run_tree(q, cache, n, bits)
        after[:, :, 3] = before[:, :, 3]
        assert torch.equal(before, after)


@pytest.mark.parametrize("dtype,form", FORMS[2:], ids=IDS[2:])
@pytest.mark.parametrize("Hq,T", [(2, 1), (2, 3), (16, 5)])
@pytest.mark.parametrize("power", [16, 30, 45, 60, 100])
@pytest.mark.parametrize("at", [0, 70, 299])
def test_a_huge_row_with_next_to_no_weight(dtype, form, Hq, T, power, at):
    """A row of V 2^power times the others' size, whose weight makes less of it than of any of them: first, in the middle, last."""
    g = ref.seeded(63)
    B, Hkv, D, past = 2, 2, 64, 300
    k, v = (torch.randn((B, Hkv, 310, D), generator=g, device="cuda") for _ in range(2))
    q = ref.normal(g, (B, Hq, T, D), dtype)
    k[..., 0], q[..., 0] = 0, 8
    k[:, :, at] = 0
    k[:, :, at, 0] = -(power + 20.0)  # a score of -(power + 20) below zero: a weight of 2^(-1.44 (power + 20))
    v[:, :, at] *= 2.0 ** power
    cache = rows_cache(k, v, form)
    sees = None if T == 1 else torch.ones((B, T, T), dtype=torch.bool, device="cuda").tril()
    assert_close(q, cache, lens_of([past, past - at // 100]), sees, 0.125)


@pytest.mark.parametrize("dtype,form", FORMS[2:], ids=IDS[2:])
@pytest.mark.parametrize("Hq,T", [(2, 1), (2, 3), (16, 5)])
def test_sizes_and_scores_far_apart(dtype, form, Hq, T):
    """Rows of V between 2^-30 and 2^30 and scores of -60 to 60, apart from one another and the larger the smaller: what has the
    most of the output changes over the rows, upwards and downwards."""
    g = ref.seeded(64)
    B, Hkv, D, past = 6, 2, 64, 700
    k, v = (torch.randn((B, Hkv, 710, D), generator=g, device="cuda") for _ in range(2))
    x = torch.linspace(-60, 60, 710, device="cuda")
    x = torch.stack([x, -x, x.abs(), -x.abs(), 60 * torch.sin(x), x[torch.randperm(710, generator=g, device="cuda")]])[:, None, :]
    q = ref.normal(g, (B, Hq, T, D), dtype, 0.1)
    q[..., 0] = 8
    k[..., 0] = x
    v *= torch.exp2(-0.5 * x + 4 * torch.randn((B, Hkv, 710), generator=g, device="cuda"))[..., None]
    cache = rows_cache(k, v, form)
    sees = None if T == 1 else torch.ones((B, T, T), dtype=torch.bool, device="cuda").tril()
    assert_close(q, cache, lens_of([past - 50 * b for b in range(B)]), sees, 0.125)


@pytest.mark.parametrize("dtype,form", FORMS[2:], ids=IDS[2:])
@pytest.mark.parametrize("Hq,T", [(2, 1), (16, 5)])
def test_rows_of_the_smallest_and_largest_sizes(dtype, form, Hq, T):
    """The ends of what kv_append keeps of bf16 rows, one sequence each; outputs of fp16 tokens stay within their range."""
    g = ref.seeded(65)
    sizes = [2.0 ** -99, 2.0 ** -60, 2.0 ** 100] if dtype == BF else [2.0 ** -20, 1.0, 2.0 ** 10]
    k, v = (torch.randn((len(sizes), 2, 200, 64), generator=g, device="cuda") for _ in range(2))
    v *= torch.tensor(sizes, device="cuda")[:, None, None, None]
    cache = rows_cache(k, v, form)
    q = ref.normal(g, (len(sizes), Hq, T, 64), dtype)
    sees = None if T == 1 else torch.ones((len(sizes), T, T), dtype=torch.bool, device="cuda").tril()
    assert_close(q, cache, lens_of([190] * len(sizes)), sees)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,T", [(2, 1), (2, 3), (8, 6), (32, 1), (24, 17)])
def test_weights_keep_their_bits(dtype, form, Hq, T):
    """Few rows, of which half cancel the other half: what the rounding of the weights leaves shows in the output."""
    g = ref.seeded(66)
    B, Hkv, D = 24, 2, 64
    v = torch.randn((B, Hkv, 40, D), generator=g, device="cuda")
    v[:, :, 1::2] = -v[:, :, 0::2]
    k = torch.randn((B, Hkv, 40, D), generator=g, device="cuda")
    cache = rows_cache(k, v, form)
    q = ref.normal(g, (B, Hq, T, D), dtype)
    sees = None if T == 1 and Hq == 2 else torch.ones((B, T, T), dtype=torch.bool, device="cuda").tril()
    assert_close(q, cache, lens_of([2 + 2 * (b % 9) for b in range(B)]), sees, 0.02)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,T", [(2, 1), (8, 6)])
def test_scores_of_queries_of_one_sign(dtype, form, Hq, T):
    """Keys with one large element, where the query has none, and otherwise small ones of either sign: the score is no larger than
    its few small terms, however large the sum of the query's elements is."""
    g = ref.seeded(67)
    B, Hkv, D = 48, 2, 128
    k = torch.randint(-1, 2, (B, Hkv, 30, D), generator=g, device="cuda").float()
    k[..., 0] = 127
    v = torch.randn((B, Hkv, 30, D), generator=g, device="cuda")
    v[:, :, 1::2] = -v[:, :, 0::2]
    cache = rows_cache(k, v, form)
    q = (1 + 0.3 * torch.rand((B, Hq, T, D), generator=g, device="cuda")).to(dtype)
    q[..., 0] = 0
    sees = None if T == 1 else torch.ones((B, T, T), dtype=torch.bool, device="cuda").tril()
    assert_close(q, cache, lens_of([2 + 2 * (b % 8) for b in range(B)]), sees, 0.25)


@pytest.mark.parametrize("form", [I8, E4])
@pytest.mark.parametrize("Hq,T", [(4, 1), (32, 4)])
@pytest.mark.parametrize("power", [126, 120, -96, -110, -124])
def test_queries_at_the_ends_of_bf16(form, Hq, T, power):
    """Only their products with the scale are ordinary numbers."""
    g = ref.seeded(68)
    k, v = (torch.randn((2, 2, 150, 64), generator=g, device="cuda") for _ in range(2))
    cache = rows_cache(k / 16 if power > 0 else k, v, form)
    q = ((torch.rand((2, Hq, T, 64), generator=g, device="cuda") * 3.9 - 1.95) * 2.0 ** power).to(BF)
    sees = None if T == 1 else torch.ones((2, T, T), dtype=torch.bool, device="cuda").tril()
    assert_close(q, cache, lens_of([140, 77]), sees, (2.0 if power > 0 else 0.125) * 2.0 ** -power)


@pytest.mark.parametrize("form", [I8, E4])
@pytest.mark.parametrize("Hq,T", [(4, 1), (32, 4)])
@pytest.mark.parametrize("power", [110, 119, -90])
def test_keys_of_any_size(form, Hq, T, power):
    """Rows of K between the ends of what kv_append keeps; only their products with the scale are ordinary numbers."""
    g = ref.seeded(69)
    k, v = (torch.randn((2, 2, 150, 64), generator=g, device="cuda") for _ in range(2))
    cache = rows_cache(k * 2.0 ** power, v, form)
    q = ref.normal(g, (2, Hq, T, 64), BF)
    sees = None if T == 1 else torch.ones((2, T, T), dtype=torch.bool, device="cuda").tril()
    assert_close(q, cache, lens_of([140, 77]), sees, 0.125 * 2.0 ** -power)


@pytest.mark.parametrize("G,T", [(8, 1), (1, 9)])
def test_a_shape_of_many_items_shares_a_workspace(G, T):
    """More (sequence, KV head) pairs than 65536 in one call, few in the next, over the same workspace."""
    g = ref.seeded(70)
    B, Hkv, D, Smax = 2150, 32, 64, 160
    big = ref.make_cache(g, B, Hkv, Smax, D, I8, binding)
    qb, nb = ref.normal(g, (B, Hkv * G, T, D), BF), lens_of([90 + (7 * b) % (Smax - T - 89) for b in range(B)])
    small = ref.make_cache(g, 1, 1, 5000, D, I8, binding)
    qs, ns = ref.normal(g, (1, G, T, D), BF), lens_of([4900])
    ws = torch.empty(binding.attn_kv_workspace_bytes(B, Hkv * G, Hkv, T, D), dtype=torch.uint8, device="cuda")
    binding.attn_kv_workspace_init(ws)
    first = [run_tree(qb, big, nb, workspace=ws), run_tree(qs, small, ns, workspace=ws)]
    for _ in range(3):
        for c, f in (((qb, big, nb), first[0]), ((qs, small, ns), first[1])):
            out = torch.full_like(f, float("nan"))
            run_tree(*c, out=out, workspace=ws)
            assert torch.equal(out, f)
    fresh = run_tree(qb, big, nb)
    assert torch.equal(fresh, first[0])


def test_not_a_number_behind_more_rows_than_31_bits_count_twice():
    """2^30 rows of 16 bits; a drafted row behind them is no number, and another is infinite."""
    past, T, D = (1 << 30) + 5, 4, 8
    k, v = (torch.zeros((1, 1, past + 8, D), dtype=BF, device="cuda") for _ in range(2))
    v[0, 0, past + 1, 3] = float("nan")
    v[0, 0, past + 2, 7] = -float("inf")
    sees = torch.eye(T, dtype=torch.bool, device="cuda")
    sees[:, 0] = True
    out = run_tree(torch.zeros((1, 4, T, D), dtype=BF, device="cuda"), binding.KVCache(k, v), lens_of([past]), ref.tree_bits(sees)[None])
    want = torch.zeros((T, D), device="cuda")
    want[1, 3], want[2, 7] = float("nan"), -float("inf")
    torch.testing.assert_close(out[0].float(), want.expand(4, T, D), rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_the_same_bits_whatever_ran_before(dtype, form):
    """Two and three steps of keys, with a kernel in between whose code and data take the caches: however late some of the warps are, the
    outputs are those of the first call."""
    g = ref.seeded(72)
    cases = []
    for B, Hq, Hkv, T, Smax, lens in ((5, 12, 4, 5, 270, [260, 253, 246, 239, 232]), (5, 16, 2, 16, 140, [120, 70, 64, 1, 100]), (3, 32, 4, 5, 400, [380, 300, 390])):
        cache = ref.make_cache(g, B, Hkv, Smax, 128, form, binding)
        cases.append((ref.normal(g, (B, Hq, T, 128), dtype), cache, lens_of(lens)))
    first = []
    for q, cache, n in cases:
        out = run_tree(q, cache, n)
        T = q.shape[2]
        want, bound = ref.attention(q, cache, n, torch.ones((T, T), dtype=torch.bool, device="cuda").tril().expand(q.shape[0], T, T))
        ref.assert_within(out, want, bound)
        first.append(out)
    a = torch.randn((1024, 1024), generator=g, device="cuda")
    big = torch.empty(200 << 20, dtype=torch.uint8, device="cuda")
    for i in range(60):
        big.fill_(i)
        torch.sort(a[:64].flatten())
        for c, f in zip(cases, first):
            assert torch.equal(run_tree(*c), f)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("Hq,T", [(4, 1), (4, 3), (16, 5), (8, 16)])
@pytest.mark.parametrize("size", [0.0, 1.0])
def test_an_infinity_that_all_see_is_one_in_the_output(dtype, Hq, T, size):
    """Elements of V that are infinite, among the past rows: the output's element is infinite, the others are what they were.  With queries of
    zeros all weights are one power of two."""
    g = ref.seeded(71)
    B, Hkv, D, Smax = 3, 2, 64, 420
    cache = ref.make_cache(g, B, Hkv, Smax, D, dtype, binding)
    q, n = ref.normal(g, (B, Hq, T, D), dtype, size), lens_of([400, 256, 33])
    sees = None if T == 1 else torch.ones((B, T, T), dtype=torch.bool, device="cuda").tril()
    want, bound = definition(q, cache, n, sees, 0.125)
    cache.v[:, :, 5, 3], cache.v[:, :, 20, 7] = float("inf"), -float("inf")
    got = run_decode(q[:, :, 0].contiguous(), cache, n, scale=0.125)[:, :, None] if T == 1 else run_tree(q, cache, n, ref.tree_bits(sees), scale=0.125)
    assert (got[..., 3] == float("inf")).all() and (got[..., 7] == -float("inf")).all()
    got[..., 3], got[..., 7] = want[..., 3].to(dtype), want[..., 7].to(dtype)
    ref.assert_within(got, want, bound)
