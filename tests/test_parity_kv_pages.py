"""GPU parity: a KV cache in pages.  Tables, slots and free pages against their definition; rows written and read back, and attention, bit
for bit as over a cache in one block that holds the same rows (whose operators are compared with 64 bits elsewhere), and with 64 bits here too."""
import random

import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF, I8, E4 = torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn
FORMS = [(BF, BF), (HF, HF), (BF, I8), (HF, I8), (BF, E4), (HF, E4)]
IDS = ["bf16", "f16", "bf16-int8", "f16-int8", "bf16-e4m3", "f16-e4m3"]


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------------- tables
def assigned(table, lens, counts, free, room, P, T, num_pages):
    """The definition, request by request: (new_lens, starts, slots, positions, requests, table, pages left)."""
    table, cap = [list(r) for r in table], len(table[0]) * P
    new_lens, starts, slots, positions, requests = [], [0], [], [], []
    total, short, room = 0, False, min(max(room, 0), num_pages)
    for b, (n, more) in enumerate(zip(lens, counts)):
        n, more = min(max(n, 0), cap), max(more, 0)
        total += more
        starts.append(min(total, T))
        have, need = -(-n // P), -(-(n + more) // P)
        ok = need <= len(table[b]) and total <= T
        if ok and need > have:
            short = short or need - have > room
            ok = not short
        if ok:
            for i in range(have, need):
                room -= 1
                table[b][i] = free[room]
        new_lens.append(n + more if ok else n)
        for p in range(n, n + min(more, max(0, T - len(slots)))):
            page = table[b][p // P] if ok else -1
            slots.append(page * P + p % P if 0 <= page < num_pages else -1)
            positions.append(p)
            requests.append(b)
    pad = T - len(slots)
    return new_lens, starts, slots + [-1] * pad, positions + [0] * pad, requests + [-1] * pad, table, [room]


def check_assign(seed, B, P, max_pages, num_pages, T, lens, counts, room=None):
    r = random.Random(seed)
    order = list(range(num_pages))
    r.shuffle(order)
    table = [[-1] * max_pages for _ in range(B)]
    for b in range(B):
        for i in range(min(-(-max(lens[b], 0) // P), max_pages)):
            table[b][i] = order.pop() if order else 0
    free = order + [-5] * (num_pages - len(order))
    room = len(order) if room is None else room
    tables = binding.PageTables(i32(table), i32(free), i32([room]), P)
    out, left = binding.PageSlots.empty(B, T), i32([77])
    binding.assign_pages(tables, i32(lens), out, None if counts is None else i32(counts), left)
    want = assigned(table, lens, [1] * B if counts is None else counts, free, room, P, T, num_pages)
    for name, got, w in zip(("lens", "starts", "slots", "positions", "requests", "table", "left"),
                            (out.lens, out.starts, out.slots, out.positions, out.requests, tables.table, left), want):
        assert got.tolist() == w, name
    assert tables.free_pages.tolist() == free and tables.free_count.tolist() == [room]


@pytest.mark.parametrize("B,P,max_pages,T", [(1, 16, 1, 1), (1, 16, 9, 100), (5, 32, 4, 9), (64, 16, 20, 64), (1023, 16, 3, 1023), (1024, 16, 3, 1030),
                                             (1025, 64, 2, 1100), (3000, 16, 4, 2500), (7, 128, 33, 5000), (2100, 16, 40, 9000)])
def test_assign_random_requests(B, P, max_pages, T):
    for seed in range(3):
        r = random.Random(1000 * seed + B)
        lens = [r.randint(0, max_pages * P) if r.random() < 0.8 else 0 for _ in range(B)]
        many = max(1, 2 * T // B)
        counts = None if seed == 0 else [r.choice([0, 1, 1, r.randint(0, many)]) for _ in range(B)]
        need = sum(-(-n // P) for n in lens)
        for room in (None, 0, max(1, B // 3)):
            check_assign(seed, B, P, max_pages, need + B * max_pages // (1 + seed) + 1, T, lens, counts, room)


def test_assign_counts_and_lengths_out_of_range():
    check_assign(1, 6, 16, 3, 30, 40, [-4, 48, 100, 17, 0, 47], [5, 1, 1, -3, 2 ** 31 - 1, 1])
    check_assign(2, 4, 16, 3, 30, 10, [0, 0, 0, 0], [4, 7, 6, 0])   # the second has no room in T, nor has anything behind it
    check_assign(3, 4, 16, 3, 30, 10, [16, 15, 32, 47], [1, 1, 1, 1], room=-3)
    check_assign(4, 4, 16, 3, 30, 10, [16, 15, 32, 47], [1, 1, 1, 1], room=2 ** 31 - 1)  # as many as there are
    check_assign(5, 3, 16, 3, 30, 3000, [0, 0, 0], [2 ** 31 - 1, 2 ** 31 - 1, 5])
    check_assign(6, 2, 1 << 20, 1, 3, 4000, [1, 0], [1999, 2001])


def test_assign_in_place_and_without_the_extras():
    """lens may be the new lengths, free_count what is left; starts, positions and requests may be left out."""
    B, P, T = 3, 16, 5000
    for more in (1, 1500):  # one CTA, and a cluster (by T)
        tables = binding.PageTables.empty(B, 400, 1000, P)
        T = 8 if more == 1 else 5000
        lens, slots = i32([0, 0, 0]), torch.zeros(T, dtype=torch.int32, device="cuda")
        out = binding.PageSlots(lens, None, slots)
        for step in range(3):
            binding.assign_pages(tables, lens, out, i32([more] * B))
        assert lens.tolist() == [3 * more] * B
        used = B * -(-3 * more // P)
        assert tables.free_count.tolist() == [1000 - used]
        held = tables.table[tables.table >= 0].tolist()
        assert len(held) == used and len(set(held)) == used
        assert held and sorted(held + tables.free_pages[: 1000 - used].tolist()) == list(range(1000))


@pytest.mark.parametrize("B", [1, 5, 1024, 2500])
def test_release(B):
    r = random.Random(B)
    P, max_pages, num_pages = 16, 5, 6 * B + 9
    order = list(range(num_pages))
    r.shuffle(order)
    lens = [r.choice([0, -1, 1, 16, 17, r.randint(0, 80), 1000]) for _ in range(B)]
    done = [r.choice([0, 1, -1]) for _ in range(B)]
    table = [[order.pop() if r.random() < 0.9 else r.choice([-1, num_pages, 2 ** 31 - 1]) for _ in range(max_pages)] for _ in range(B)]
    back = [e for b in range(B) if done[b] for e in table[b][: -(-min(max(lens[b], 0), 80) // P)] if 0 <= e < num_pages]
    room = len(order)
    tables = binding.PageTables(i32(table), i32(order + [-7] * (num_pages - room)), i32([room]), P)
    left = i32([0])
    binding.release_pages(tables, i32(lens), i32(done), left)
    assert left.tolist() == [room + len(back)] and tables.free_count.tolist() == [room]
    assert tables.free_pages.tolist() == order + back + [-7] * (num_pages - room - len(back))
    assert tables.table.tolist() == table
    binding.release_pages(tables, i32(lens), i32([0] * B))
    assert tables.free_count.tolist() == [room]


# ------------------------------------------------------------------------------------------------------- a cache in pages
def paged(g, cache, P, max_pages=None, spare=3, poison=True):
    """The rows of a KVCache in pages anywhere, and their table; other pages hold NaN or codes with a NaN scale."""
    B, Hkv, Smax, D = cache.k.shape
    n = -(-Smax // P)
    max_pages = n if max_pages is None else max_pages
    num = B * n + spare
    order = torch.randperm(num, generator=g, device="cuda")[: B * n]
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    table[:, :n] = order.view(B, n).int()

    def scatter(x, fill):
        out = torch.full((num, Hkv, P, *x.shape[3:]), fill, device="cuda").to(x.dtype) if poison else torch.zeros((num, Hkv, P, *x.shape[3:]), dtype=x.dtype, device="cuda")
        for b in range(B):
            for i in range(n):
                rows = x[b, :, i * P: (i + 1) * P]
                out[order[b * n + i], :, : rows.shape[1]] = rows
        return out.contiguous()
    fill = float("nan") if cache.k_scale is None else 1.0
    k, v = scatter(cache.k, fill), scatter(cache.v, fill)
    scales = [] if cache.k_scale is None else [scatter(cache.k_scale, float("nan")), scatter(cache.v_scale, float("nan"))]
    return binding.KVPages(k, v, *scales), table


def same_bits(a, b):
    """Bit for bit, NaN included."""
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def one_kernel(Hq, Hkv, T=1):
    """Whether the operator does not split the query heads of a KV head where that of a cache in one block does not."""
    G = Hq // Hkv
    return G * T <= 8 or not any(G % p == 0 and G // p * T <= 8 for p in (2, 3, 4))


def check_decode(seed, dtype, form, Hq, Hkv, D, lens, Smax, P):
    g = ref.seeded(seed)
    cache = ref.make_cache(g, len(lens), Hkv, Smax, D, form, binding)
    pages, table = paged(g, cache, P)
    q, n = ref.normal(g, (len(lens), Hq, D), dtype), i32(lens)
    out = binding.attn_decode_pages(q, pages, table, n)
    binding.check_status()
    want, bound = ref.attention(q[:, :, None], cache, n)
    ref.assert_within(out, want[:, :, 0], bound[:, :, 0])
    if Smax % P == 0 and one_kernel(Hq, Hkv):
        assert same_bits(out, binding.attn_decode_kv(q, cache, n))


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("P", [16, 32, 64, 256])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (12, 12, 64), (6, 2, 80), (4, 4, 16), (16, 1, 128), (11, 1, 128), (18, 2, 64), (22, 2, 80), (32, 1, 64)])
def test_decode_around_borders(dtype, form, P, Hq, Hkv, D):
    """Up to 8 heads to a KV head, and more, which another kernel serves."""
    check_decode(11, dtype, form, Hq, Hkv, D, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 512], 512, P)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("B,Hq,Hkv,D,Smax,P", [(1, 8, 8, 64, 40000, 16), (1, 32, 8, 128, 33280, 64), (2, 16, 1, 128, 9008, 16), (1, 1, 1, 128, 1, 16),
                                               (300, 4, 2, 64, 320, 32), (33, 8, 1, 128, 700, 16)])
def test_decode_of_long_and_many(dtype, form, B, Hq, Hkv, D, Smax, P):
    check_decode(12, dtype, form, Hq, Hkv, D, [max(0, Smax - (37 * b * b + 11 * b) % Smax) for b in range(B)], Smax, P)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("P", [16, 32, 128])
@pytest.mark.parametrize("Hq,Hkv,D,T", [(32, 8, 128, 5), (16, 4, 64, 3), (12, 2, 128, 2), (4, 4, 64, 1), (4, 4, 128, 8), (28, 4, 128, 16), (8, 1, 64, 33), (16, 8, 80, 64)])
def test_trees(dtype, form, P, Hq, Hkv, D, T):
    g = ref.seeded(21)
    lens = [0, 1, 100, 128 - T, 127, 128, 500, 640 - T, 640, 700]
    cache = ref.make_cache(g, len(lens), Hkv, 640, D, form, binding)
    pages, table = paged(g, cache, P)
    q, n = ref.normal(g, (len(lens), Hq, T, D), dtype), i32(lens)
    sees = ref.random_tree(g, len(lens), T)
    bits = ref.tree_bits(sees)
    out = binding.attn_tree_pages(q, pages, table, n, bits)
    binding.check_status()
    want, bound = ref.attention(q, cache, n, sees)
    ref.assert_within(out, want, bound)
    chain = binding.attn_tree_pages(q, pages, table, n)
    want, bound = ref.attention(q, cache, n, torch.ones((T, T), dtype=torch.bool, device="cuda").tril().expand(len(lens), T, T))
    ref.assert_within(chain, want, bound)
    if one_kernel(Hq, Hkv, T):
        assert same_bits(out, binding.attn_tree(q, cache, n, bits))
        assert same_bits(chain, binding.attn_tree(q, cache, n))


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq", [4, 8, 32])
def test_infinities_in_rows_that_some_tokens_see(dtype, form, Hq):
    """Rows of drafted tokens may hold anything for the tokens that do not see them; those that do get it."""
    g = ref.seeded(22)
    B, Hkv, D, T, Smax = 3, 2, 64, 4 if Hq <= 8 else 9, 160
    cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding)
    n = i32([0, 61, 150])
    sees = ref.random_tree(g, B, T)
    for b, past in enumerate(n.tolist()):
        if form in (BF, HF):
            cache.v[b, :, past + 1, 3] = float("inf")
            cache.v[b, :, past + 2, 5] = float("nan")
        else:
            cache.v_scale[b, :, past + 2] = float("nan")
    q = ref.normal(g, (B, Hq, T, D), dtype)
    pages, table = paged(g, cache, 16)
    out = binding.attn_tree_pages(q, pages, table, n, ref.tree_bits(sees))
    binding.check_status()
    if one_kernel(Hq, Hkv, T):
        assert same_bits(out, binding.attn_tree(q, cache, n, ref.tree_bits(sees)))
    bad = torch.isfinite(out).all(-1).logical_not().any(1)   # [B, T]
    see = sees[:, :, 2] | (sees[:, :, 1] & (form in (BF, HF)))
    assert torch.equal(bad, see)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq", [8, 22])
def test_entries_that_name_no_page(dtype, form, Hq):
    """Behind the last row they do not matter; before it their rows are zeros, as written into a cache in one block."""
    g = ref.seeded(23)
    B, Hkv, D, Smax, P = 4, 2, 64, 192, 16
    cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding)
    pages, table = paged(g, cache, P)
    q, n = ref.normal(g, (B, Hq, D), dtype), i32([0, 33, 100, 192])
    want = binding.attn_decode_kv(q, cache, n)
    for junk in (-1, -2 ** 31, 2 ** 31 - 1, pages.num_pages):
        t = table.clone()
        for b, rows in enumerate(n.tolist()):
            t[b, -(-rows // P):] = junk
        assert same_bits(binding.attn_decode_pages(q, pages, t, n), want)
        t[2, 3] = t[3, 0] = t[3, 11] = t[1, 1] = junk
        holes = binding.KVCache(cache.k.clone(), cache.v.clone(), *([] if cache.k_scale is None else [cache.k_scale.clone(), cache.v_scale.clone()]))
        for b, i in ((2, 3), (3, 0), (3, 11), (1, 1)):
            for x in (holes.k, holes.v, holes.k_scale, holes.v_scale):
                if x is not None:
                    x[b, :, i * P: (i + 1) * P] = 0
        got = binding.attn_decode_pages(q, pages, t, n)
        binding.check_status()
        assert same_bits(got, binding.attn_decode_kv(q, holes, n))


def test_shared_pages_and_a_table_of_more_columns():
    """Requests may share a prefix; a table may have room for more rows than any request has."""
    g = ref.seeded(24)
    B, Hq, Hkv, D, P, Smax = 6, 8, 2, 128, 32, 320
    cache = ref.make_cache(g, B, Hkv, Smax, D, E4, binding)
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        x[:, :, :160] = x[:1, :, :160]
    pages, table = paged(g, cache, P, max_pages=4000)
    table[:, :5] = table[0, :5]
    q, n = ref.normal(g, (B, Hq, D), BF), i32([320, 200, 161, 160, 159, 64])
    out = binding.attn_decode_pages(q, pages, table, n)
    want, bound = ref.attention(q[:, :, None], cache, n)
    ref.assert_within(out, want[:, :, 0], bound[:, :, 0])


@pytest.mark.parametrize("form,Hq", [(I8, 8), (BF, 8), (E4, 11), (E4, 16)])
def test_a_cache_of_more_than_32_bits(form, Hq):
    """Pages whose elements lie beyond 2^32 from the start."""
    g = ref.seeded(25)
    Hkv, P, D, num = 1, 16, 128, (1 << 32) // (16 * 128) + 700
    cache = ref.make_cache(g, 2, Hkv, 512, D, form, binding)
    k, v = (torch.empty((num, Hkv, P, D), dtype=form, device="cuda") for _ in range(2))
    scales = [] if cache.k_scale is None else [torch.empty((num, Hkv, P), device="cuda") for _ in range(2)]
    table = (num - 1 - torch.arange(64, device="cuda").view(2, 32)).int()
    for x, y in zip((k, v, *scales), (cache.k, cache.v, cache.k_scale, cache.v_scale)):
        x[table.long()] = y.view(2, 1, 32, P, *y.shape[3:]).transpose(1, 2)
    pages = binding.KVPages(k, v, *scales)
    q, n = ref.normal(g, (2, Hq, D), BF), i32([512, 100])
    got = binding.attn_decode_pages(q, pages, table, n)
    want, bound = ref.attention(q[:, :, None], cache, n)
    ref.assert_within(got, want[:, :, 0], bound[:, :, 0])
    if one_kernel(Hq, Hkv):
        assert same_bits(got, binding.attn_decode_kv(q, cache, n))
    # rows there: written by slot, read back
    new = ref.normal(g, (3, Hkv, D), BF)
    slots = i32([int(table[0, 31]) * P + 15, int(table[1, 0]) * P, int(table[0, 0]) * P + 3])
    binding.kv_append_pages(pages, new, new, slots)
    out = [torch.zeros((2, Hkv, 512, D), dtype=BF, device="cuda") for _ in range(2)]
    binding.kv_read_pages(pages, table, *out)
    small = binding.KVCache.empty(3, Hkv, 1, D, pages.format)
    binding.kv_append(small, new[:, :, None], new[:, :, None], i32([0, 0, 0]))
    back = [torch.zeros((3, Hkv, 1, D), dtype=BF, device="cuda") for _ in range(2)]
    binding.kv_read(small, *back)
    for o, w in zip(out, back):
        assert same_bits(torch.stack([o[0, :, 511], o[1, :, 0], o[0, :, 3]]), w[:, :, 0])


# ------------------------------------------------------------------------------------------------------- rows in and out
@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("D,dims,layout", [(64, 64, 0), (128, 96, 1), (80, 40, 0), (128, 0, 0), (96, 44, 0)])
def test_append_is_that_of_a_cache_in_one_block(dtype, form, D, dims, layout):
    g = ref.seeded(31)
    B, Hq, Hkv, S, P, Smax = 4, 6, 2, 37, 16, 112
    if form in (I8, E4) and D % 16:
        pytest.skip("8-bit rows are multiples of 16")
    counts, lens = [37, 0, 1, 20], [3, 50, 111, 16]
    fmt = binding._KV_TYPES.index(form)
    flat = binding.KVCache.empty(B, Hkv, Smax, D, fmt)
    pages, table = paged(g, flat, P, poison=False)
    qkv = ref.normal(g, (B, S, Hq + 2 * Hkv, D), dtype)
    q, k, v = (x.permute(0, 2, 1, 3) for x in qkv.split([Hq, Hkv, Hkv], 2))
    rotary = binding.Rotary(binding.rotary_frequencies(dims)[0].cuda(), layout, 0.75) if dims else None
    q_want = torch.zeros_like(q)
    kw = dict(rotary=rotary, q=q, q_out=q_want) if dims else {}
    binding.kv_append(flat, k, v, i32(lens), counts=i32(counts), **kw)
    # the same tokens, packed, between tokens without a slot
    token = [(b, i) for b in range(B) for i in range(counts[b])]
    T = len(token) + 3
    packed = torch.full((T, Hq + 2 * Hkv, D), float("nan"), device="cuda").to(dtype)
    slots, positions = [-1] * T, [0] * T
    for t, (b, i) in enumerate(token):
        packed[t + 1] = qkv[b, i]
        positions[t + 1] = lens[b] + i
        slots[t + 1] = int(table[b, (lens[b] + i) // P]) * P + (lens[b] + i) % P
    slots[0], slots[-1], slots[-2] = -5, pages.num_pages * P, 2 ** 31 - 1
    pq, pk, pv = packed.split([Hq, Hkv, Hkv], 1)
    q_out = torch.full((T, Hq, D), 7.0, device="cuda").to(dtype)
    kw = dict(rotary=rotary, positions=i32(positions), q=pq, q_out=q_out) if dims else {}
    binding.kv_append_pages(pages, pk, pv, i32(slots), **kw)
    gather = lambda x: x[table.long()].transpose(1, 2).reshape(B, Hkv, Smax, *x.shape[3:])
    for got, want in ((pages.k, flat.k), (pages.v, flat.v), (pages.k_scale, flat.k_scale), (pages.v_scale, flat.v_scale)):
        if want is not None:
            assert torch.equal(gather(got).float(), want.float())
            free = torch.ones(pages.num_pages, dtype=torch.bool, device="cuda")
            free[table.long()] = False
            assert (got[free].float() == 0).all()
    if dims:
        for t, (b, i) in enumerate(token):
            assert same_bits(q_out[t + 1], q_want[b, :, i].contiguous())
        assert (q_out[[0, -1, -2]].float() == 7).all()
    # and back
    outs = [torch.full((B, 60, Hkv, D), 3.0, device="cuda").to(dtype).transpose(1, 2) for _ in range(4)]
    first, n = i32([3, 60, -2, 100]), i32([60, 11, 70, 70])
    binding.kv_read(flat, *outs[:2], first=first, counts=n)
    binding.kv_read_pages(pages, table, *outs[2:], first=first, counts=n)
    for a, b in zip(outs[:2], outs[2:]):
        assert same_bits(a.contiguous(), b.contiguous())


def test_read_leaves_rows_of_no_page():
    g = ref.seeded(32)
    cache = ref.make_cache(g, 2, 3, 64, 64, BF, binding)
    pages, table = paged(g, cache, 16)
    table[0, 1], table[1, 3] = -1, pages.num_pages
    out = [torch.full((2, 3, 80, 64), 5.0, device="cuda").to(BF) for _ in range(2)]
    binding.kv_read_pages(pages, table, *out)
    for o, x in zip(out, (cache.k, cache.v)):
        want = torch.full_like(o, 5.0)
        want[:, :, :64] = x
        want[0, :, 16:32] = want[1, :, 48:64] = 5.0
        assert same_bits(o, want)


def test_rows_against_64_bits():
    """K rotated at far positions and kept in 8 bits."""
    g = ref.seeded(33)
    T, Hkv, D, P = 50, 3, 128, 32
    inv = binding.rotary_frequencies(D)[0].cuda()
    for form in (I8, E4, BF):
        pages = binding.KVPages.empty(4, Hkv, P, D, binding._KV_TYPES.index(form))
        k, v = ref.normal(g, (T, Hkv, D), BF), ref.normal(g, (T, Hkv, D), BF)
        slots = torch.randperm(4 * P, generator=g, device="cuda")[:T].int()
        pos = torch.randint(0, 1 << 20, (T,), generator=g, device="cuda", dtype=torch.int32)
        binding.kv_append_pages(pages, k, v, slots, positions=pos, rotary=binding.Rotary(inv))
        turned, err = ref.rotate(k.permute(1, 0, 2)[None], pos[None], inv)
        s = slots.long()
        at = lambda x: None if x is None else x[s // P, :, s % P]
        ref.assert_rows_kept(at(pages.k), at(pages.k_scale), turned[0].transpose(0, 1), err[0].transpose(0, 1), "k")
        ref.assert_rows_kept(at(pages.v), at(pages.v_scale), v.double(), torch.zeros_like(v, dtype=torch.float64), "v")


# ------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,form", [(BF, BF), (HF, I8), (BF, E4)], ids=["bf16", "f16-int8", "bf16-e4m3"])
@pytest.mark.parametrize("captured", [False, True])
def test_requests_come_and_go(dtype, form, captured):
    """Steps of a server: tokens packed, pages handed out and given back, rows appended, attention.  Each step's outputs are those
    over caches in one block per request.  Captured: the step is one graph, replayed."""
    g = ref.seeded(41)
    r = random.Random(5)
    B, Hq, Hkv, D, P, max_pages, num_pages = 5, 8, 2, 64, 16, 8, 9
    T, Smax = 40, P * max_pages
    fmt = binding._KV_TYPES.index(form)
    pages = binding.KVPages.empty(num_pages, Hkv, P, D, fmt)
    flat = binding.KVCache.empty(B, Hkv, Smax, D, fmt)
    tables = binding.PageTables.empty(B, max_pages, num_pages, P)
    out = binding.PageSlots.empty(B, T)
    rotary = binding.Rotary(binding.rotary_frequencies(D)[0].cuda())
    ws = torch.zeros(binding.attn_kv_workspace_bytes(B, Hq, Hkv, 1, D), dtype=torch.uint8, device="cuda")
    lens, counts, done = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    qkv, q1 = torch.zeros((T, Hq + 2 * Hkv, D), dtype=dtype, device="cuda"), torch.zeros((B, Hq, D), dtype=dtype, device="cuda")
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    q_out, o = torch.zeros((T, Hq, D), dtype=dtype, device="cuda"), torch.zeros_like(q1)

    def step():
        binding.release_pages(tables, lens, done)
        lens.mul_(1 - done)
        binding.assign_pages(tables, lens, out, counts)
        binding.kv_append_pages(pages, k, v, out.slots, positions=out.positions, rotary=rotary, q=q, q_out=q_out)
        binding.attn_decode_pages(q1, pages, tables.table, out.lens, out=o, workspace=ws)

    if captured:
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    refused = 0
    for turn in range(25):
        ends = [1 if r.random() < 0.15 else 0 for _ in range(B)]
        more = [r.choice([0, 1, 1, 1, r.randint(1, 17)]) for _ in range(B)]
        while sum(more) > T:
            more[r.randrange(B)] = 0
        done.copy_(i32(ends))
        counts.copy_(i32(more))
        qkv.copy_(ref.normal(g, qkv.shape, dtype))
        q1.copy_(ref.normal(g, q1.shape, dtype))
        before = lens.clone() * (1 - done)
        graph.replay() if captured else step()
        binding.check_status()
        got = (out.lens - before).tolist()
        refused += sum(a != b for a, b in zip(got, more))
        assert all(a in (0, b) for a, b in zip(got, more))
        starts = out.starts.tolist()
        for b in range(B):  # the same into the request's own cache
            if got[b]:
                one = binding.KVCache(*(x[b: b + 1] for x in (flat.k, flat.v)), *([] if flat.k_scale is None else [x[b: b + 1] for x in (flat.k_scale, flat.v_scale)]))
                rows = lambda x: x[starts[b]: starts[b] + got[b]].transpose(0, 1)[None]
                binding.kv_append(one, rows(k), rows(v), before[b: b + 1].contiguous(), rotary=rotary)
        assert same_bits(o, binding.attn_decode_kv(q1, flat, out.lens))
        held = [e for b in range(B) for e in tables.table[b, : -(-int(out.lens[b]) // P)].tolist()]
        left = int(tables.free_count)
        assert sorted(held + tables.free_pages[:left].tolist()) == list(range(num_pages))
        lens.copy_(out.lens)
    assert refused > 0  # pages did run short


def test_calls_on_two_streams():
    g = ref.seeded(42)
    cache = ref.make_cache(g, 4, 2, 512, 128, I8, binding)
    pages, table = paged(g, cache, 32)
    q, n = ref.normal(g, (4, 8, 128), BF), i32([512, 3, 77, 300])
    want = binding.attn_decode_kv(q, cache, n)
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(binding.attn_decode_pages(q, pages, table, n))
    torch.cuda.synchronize()
    assert all(same_bits(o, want) for o in outs)


def test_native_and_general_marshalling_do_the_same(monkeypatch):
    """Each call by the native way and by Python's, with and without its optional arguments."""
    g = ref.seeded(43)
    B, Hq, Hkv, D, P, T = 3, 6, 2, 64, 16, 9
    cache = ref.make_cache(g, B, Hkv, 96, D, I8, binding)
    q, n = ref.normal(g, (B, Hq, D), HF), i32([90, 4, 40])
    qt = ref.normal(g, (B, T, Hq, D), HF).transpose(1, 2)
    bits = ref.tree_bits(ref.random_tree(g, B, T))
    k, v, qa = ref.normal(g, (T, Hkv, D), HF), ref.normal(g, (T, Hkv, D), HF), ref.normal(g, (T, Hq, D), HF)
    rotary = binding.Rotary(binding.rotary_frequencies(D)[0].cuda())
    x, y = ref.normal(g, (T, 128), HF), ref.normal(g, (T, 64), HF)
    a, b = ref.normal(g, (4, 8, 128), HF), ref.normal(g, (4, 64, 8), HF)
    which = i32([0, 1, -1, 3, 3, 2, 0, 1, 1])
    scales = torch.rand(4, generator=g, device="cuda")

    def everything():
        out = []
        pages, table = paged(ref.seeded(44), cache, P)
        tables = binding.PageTables(table.clone(), torch.arange(pages.num_pages, dtype=torch.int32, device="cuda"), i32([5]), P)
        step, left = binding.PageSlots.empty(B, T), i32([0])
        out.append(binding.assign_pages(tables, n, step, counts=i32([3, 4, 2]), free_left=left).slots.clone())
        out += [step.lens.clone(), step.starts.clone(), step.positions.clone(), step.requests.clone(), tables.table.clone(), left]
        binding.assign_pages(tables, n, step)
        out += [step.slots.clone(), tables.free_count.clone()]
        slots = torch.arange(T, dtype=torch.int32, device="cuda") * 5
        out.append(binding.kv_append_pages(pages, k, v, slots, positions=slots, rotary=rotary, q=qa, q_out=torch.zeros_like(qa)))
        assert binding.kv_append_pages(pages, v, k, slots + 1) is None
        out += [pages.k.clone(), pages.v_scale.clone().nan_to_num()]
        ko, vo = (torch.zeros((B, Hkv, 20, D), dtype=HF, device="cuda") for _ in range(2))
        out += list(binding.kv_read_pages(pages, table, ko, vo, first=i32([3, 0, 30]), counts=i32([20, 4, 9])))
        ws = torch.zeros(1 << 25, dtype=torch.uint8, device="cuda")
        out.append(binding.attn_decode_pages(q, pages, table, n, out=torch.empty_like(q), workspace=ws))
        out.append(binding.attn_tree_pages(qt, pages, table, n - 2, bits, scale=0.3, out=torch.empty_like(qt), workspace=ws))
        out.append(binding.attn_tree_pages(qt, pages, table, n - 2, out=torch.empty_like(qt), workspace=ws))
        out.append(binding.linear_adapters(x, y, a, b, which, scales=scales, out=torch.empty_like(y)))
        out.append(binding.linear_adapters(x, y, a, b, which[:4].contiguous(), requests=which, out=torch.empty_like(y)))
        binding.check_status()
        return out

    native = everything()
    monkeypatch.setattr(binding, "_host_calls", None)
    for i, (one, other) in enumerate(zip(native, everything())):
        assert torch.equal(one.float(), other.float()), i


def test_nothing_beside_the_outputs_is_written():
    """Slots, tables and rows lie between guards."""
    P, num, Hkv, D = 16, 8, 2, 64
    guard = 64
    for T, more in ((40, [3, 20]), (3000, [3, 90])):
        buf = {n: torch.full((m + 2 * guard,), 77, dtype=torch.int32, device="cuda")
               for n, m in (("lens", 2), ("starts", 3), ("slots", T), ("positions", T), ("requests", T), ("left", 1), ("table", 2 * 6))}
        mid = {n: x[guard:-guard] for n, x in buf.items()}
        mid["table"].fill_(-1)
        tables = binding.PageTables(mid["table"].view(2, 6), torch.arange(num, dtype=torch.int32, device="cuda"), i32([num]), P)
        binding.assign_pages(tables, i32([0, 0]), binding.PageSlots(*(mid[n] for n in ("lens", "starts", "slots", "positions", "requests"))),
                             counts=i32(more), free_left=mid["left"])
        assert mid["lens"].tolist() == more and mid["left"].tolist() == [num - sum(-(-m // P) for m in more)]
        for x in buf.values():
            assert (x[:guard] == 77).all() and (x[-guard:] == 77).all()
    big = torch.full((num + 2, Hkv, P, D), 9.0, dtype=BF, device="cuda")
    other = big.clone()
    pages = binding.KVPages(big[1:-1], other[1:-1])
    k = torch.ones((4, Hkv, D), dtype=BF, device="cuda")
    binding.kv_append_pages(pages, k, k, i32([0, num * P - 1, num * P, -1]))
    for x in (big, other):
        assert (x[0] == 9).all() and (x[-1] == 9).all() and (x == 1).sum() == 2 * Hkv * D
        assert (x[1, :, 0] == 1).all() and (x[-2, :, -1] == 1).all()
    q = torch.ones((3, 4, D), dtype=BF, device="cuda")
    out = torch.full((5, 4, D), 9.0, dtype=BF, device="cuda")
    binding.attn_decode_pages(q, pages, i32([[0, 1]] * 3), i32([32, 0, 7]), out=out[1:4])
    assert (out[0] == 9).all() and (out[4] == 9).all() and (out[2] == 0).all()
