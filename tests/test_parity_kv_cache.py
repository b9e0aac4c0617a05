"""GPU parity: rotary positions, appending rows to a KV cache and reading them back, against the definition in 64 bits with the
bounds that the roundings give (kv_reference.py)."""
import pytest
import torch

import kv_reference as ref
from paper_2604_16498_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF, F32, I8, E4 = torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.float8_e4m3fn
LAYOUTS = {"half": binding.ROTARY_HALF, "interleaved": binding.ROTARY_INTERLEAVED}
FORMAT = {BF: binding.KV_BF16, HF: binding.KV_F16, I8: binding.KV_INT8, E4: binding.KV_E4M3}


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def rotary_of(dims, layout="half", amplitude=1.0, base=10000.0):
    f, _ = binding.rotary_frequencies(dims, base)
    return binding.Rotary(f.cuda(), LAYOUTS[layout], amplitude)


def assert_rotated(got, x, positions, rotary, layout, amplitude=1.0, inverse=False):
    want, err = ref.rotate(x, positions, rotary.inv_freq, layout, amplitude, inverse)
    ref.assert_within(got, want, err + ref.HALF[x.dtype] * want.abs() * 1.01 + 2.0 ** -25)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,dims", [(128, 128), (64, 64), (256, 256), (128, 96), (80, 80), (80, 40), (128, 2), (128, 20), (8, 8), (8, 2),
                                    (64, 34), (200, 126), (96, 96), (16, 6)])
def test_rotary(dtype, layout, D, dims):
    g = ref.seeded(1)
    B, H, S = 2, 5, 7
    x = ref.normal(g, (B, H, S, D), dtype)
    pos = torch.randint(0, 5000, (B, S), generator=g, device="cuda", dtype=torch.int32)
    r = rotary_of(dims, layout)
    assert_rotated(binding.rotary_apply(x, r, positions=pos), x, pos, r, layout)
    assert_rotated(binding.rotary_apply(x, r, positions=pos, inverse=True), x, pos, r, layout, inverse=True)


@pytest.mark.parametrize("S,B,H", [(1, 1, 1), (1, 16, 40), (1, 300, 3), (777, 3, 12), (2048, 1, 33), (5, 1, 64)])
def test_rotary_sizes_and_where_positions_come_from(S, B, H):
    g = ref.seeded(2)
    x = ref.normal(g, (B, H, S, 128), BF)
    r = rotary_of(128)
    s = torch.arange(S, device="cuda", dtype=torch.int32)
    first = torch.randint(0, 9000, (B,), generator=g, device="cuda", dtype=torch.int32)
    assert_rotated(binding.rotary_apply(x, r), x, s.expand(B, S), r, "half")
    assert_rotated(binding.rotary_apply(x, r, first=first), x, first[:, None] + s, r, "half")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("far,more", [(1 << 20, 0.0), (-1000, 0.0), (2**31 - 2, 3e-6), (-2**31, 3e-6)])
def test_far_and_negative_positions(layout, far, more):
    """Beyond 2^20 the frequency's 2^-53 counts: 2^31 x 2^-53 turns and the reference's own angle (2^31 in fp64, 2^-22 of it off)."""
    g = ref.seeded(3)
    x = ref.normal(g, (1, 2, 2, 128), F32)
    pos = ints([[far, far + 1]])
    r = rotary_of(128, layout)
    want, err = ref.rotate(x, pos, r.inv_freq, layout)
    got = binding.rotary_apply(x, r, positions=pos)
    ref.assert_within(got, want, err + ref.F32 * want.abs() + more * x.abs().max())


def test_rotary_in_place_on_a_projection_and_back():
    """Query and key heads of a fused projection in one call; the value heads beside them stay as they are."""
    g = ref.seeded(4)
    B, S, Hq, Hkv, D = 2, 33, 6, 2, 64
    for dims, layout in ((64, "half"), (64, "interleaved"), (20, "half"), (48, "half")):
        qkv = ref.normal(g, (B, S, Hq + 2 * Hkv, D), F32)
        was = qkv.clone()
        qk = qkv[:, :, :Hq + Hkv].permute(0, 2, 1, 3)
        r = rotary_of(dims, layout)
        first = ints([0, 500])
        binding.rotary_apply(qk, r, first=first, out=qk)
        pos = first[:, None] + torch.arange(S, device="cuda", dtype=torch.int32)
        assert_rotated(qk, was[:, :, :Hq + Hkv].permute(0, 2, 1, 3), pos, r, layout)
        assert torch.equal(qkv[:, :, Hq + Hkv:], was[:, :, Hq + Hkv:])
        binding.rotary_apply(qk, r, first=first, inverse=True, out=qk)
        assert (qkv - was).abs().max() < 1e-5


def test_the_inverse_is_the_gradient():
    """d/dx <w, rotate(x)> = rotate back(w), the amplitude included; against differences of the fp32 operator."""
    g = ref.seeded(5)
    x, w = ref.normal(g, (1, 2, 3, 32), F32), ref.normal(g, (1, 2, 3, 32), F32)
    r = rotary_of(24, "half", amplitude=1.3)
    grad = binding.rotary_apply(w, r, inverse=True)
    for at in ((0, 0, 0, 0), (0, 1, 2, 5), (0, 0, 1, 12), (0, 1, 1, 23), (0, 0, 2, 24), (0, 1, 0, 31)):
        step = torch.zeros_like(x)
        step[at] = 0.5  # linear: the step's size does not matter
        diff = ((binding.rotary_apply(x + step, r).double() - binding.rotary_apply(x - step, r).double()) * w.double()).sum()
        assert abs(diff - grad[at].double()) < 1e-4
    want, err = ref.rotate(w, torch.arange(3, device="cuda")[None], r.inv_freq, "half", 1.3, True)
    ref.assert_within(grad, want, err + ref.F32 * want.abs())


def test_zero_angle_and_amplitude():
    g = ref.seeded(6)
    x = ref.normal(g, (1, 3, 1, 128), BF)
    assert torch.equal(binding.rotary_apply(x, rotary_of(128)), x)  # position 0
    y = binding.rotary_apply(x, rotary_of(64, amplitude=2.0))
    assert torch.equal(y[..., :64], 2 * x[..., :64]) and torch.equal(y[..., 64:], x[..., 64:])


# ------------------------------------------------------------------------------------------------------------- append
def snapshot(cache):
    return [None if t is None else t.clone().view(torch.uint8) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]


def assert_only_rows_changed(cache, before, changed):
    """changed [B, Smax] bool."""
    for t, was in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), before):
        if t is not None:
            same = t.view(torch.uint8).view(was.shape) == was
            if t.dim() == 3:
                same = same.view(*t.shape, 4)
            same = same.flatten(3).all(-1)  # [B, Hkv, Smax]
            assert bool((same | changed[:, None]).all()), "a row that was not appended has changed"


def check_append(seed, dtype, form, B, Hq, Hkv, S, Smax, D, lens, dims=None, layout="half", counts=None, positions=None, with_q=True):
    g = ref.seeded(seed)
    cache = binding.KVCache.empty(B, Hkv, Smax, D, FORMAT[form])
    for t in (cache.k, cache.v):
        t.view(torch.uint8).fill_(0x2a)
    before = snapshot(cache)
    qkv = ref.normal(g, (B, S, Hq + 2 * Hkv, D), dtype)
    q, k, v = (x.permute(0, 2, 1, 3) for x in qkv.split([Hq, Hkv, Hkv], 2))
    n = ints(lens)
    cnt = None if counts is None else ints(counts)
    r = None if dims == 0 else rotary_of(dims or D, layout)
    q_out = torch.full((B, S, Hq, D), 9.0, dtype=dtype, device="cuda").permute(0, 2, 1, 3) if with_q and r else None
    binding.kv_append(cache, k, v, n, counts=cnt, positions=positions, rotary=r, q=q if q_out is not None else None, q_out=q_out)
    binding.check_status()
    start = n.clamp(0, Smax)
    pos = start[:, None] + torch.arange(S, device="cuda", dtype=torch.int32) if positions is None else positions
    if r is None:
        want_k, err_k = k.double(), torch.zeros_like(k, dtype=torch.float64)
    else:
        want_k, err_k = ref.rotate(k, pos, r.inv_freq, layout)
    changed = torch.zeros((B, Smax), dtype=torch.bool, device="cuda")
    for b in range(B):
        c = S if counts is None else min(max(counts[b], 0), S)
        at, m = int(start[b]), min(c, Smax - int(start[b]))
        changed[b, at:at + m] = True
        if m > 0:
            sl = lambda t: None if t is None else t[b, :, at:at + m]  # noqa: E731
            ref.assert_rows_kept(sl(cache.k), sl(cache.k_scale), want_k[b, :, :m], err_k[b, :, :m], "k")
            ref.assert_rows_kept(sl(cache.v), sl(cache.v_scale), v[b, :, :m].double(), torch.zeros_like(v[b, :, :m], dtype=torch.float64), "v")
        if q_out is not None:
            want, err = ref.rotate(q[b:b + 1, :, :c], pos[b:b + 1, :c], r.inv_freq, layout)
            if c:
                ref.assert_within(q_out[b:b + 1, :, :c], want, err + ref.HALF[dtype] * want.abs() * 1.01 + 2.0 ** -25)
            assert (q_out[b, :, c:] == 9).all()
    assert_only_rows_changed(cache, before, changed)
    return cache, changed


FORMS = [(BF, BF), (HF, HF), (BF, I8), (HF, I8), (BF, E4), (HF, E4)]
IDS = ["bf16", "f16", "bf16-int8", "f16-int8", "bf16-e4m3", "f16-e4m3"]


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,Hkv,D,dims,layout", [(32, 8, 128, 128, "half"), (12, 12, 64, 64, "interleaved"), (7, 1, 128, 96, "half"),
                                                  (3, 3, 80, 80, "half"), (4, 2, 16, 6, "half"), (5, 5, 96, 36, "half"), (2, 1, 112, 0, "half")])
def test_append(dtype, form, Hq, Hkv, D, dims, layout):
    check_append(11, dtype, form, 3, Hq, Hkv, 5, 40, D, [0, 17, 35], dims, layout)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_append_one_token_and_long_prompts(dtype, form):
    check_append(12, dtype, form, 16, 8, 2, 1, 64, 128, list(range(16)))
    check_append(13, dtype, form, 2, 8, 2, 1031, 1500, 128, [0, 469])


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_append_ragged_full_and_out_of_range(dtype, form):
    """Counts of nothing, of too much; lengths behind which there is no room, or which lie outside the cache."""
    check_append(14, dtype, form, 8, 4, 2, 9, 33, 64, [0, 24, 25, 30, 33, 40, -3, 5], counts=[9, 9, 9, 100, 5, 4, 3, -1])
    check_append(15, dtype, form, 3, 4, 2, 6, 33, 64, [0, 3, 30], counts=[0, 1, 6], with_q=False)


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_append_positions_of_a_tree(dtype, form):
    check_append(16, dtype, form, 2, 4, 2, 6, 50, 64, [10, 40], positions=ints([[10, 11, 11, 12, 12, 13], [40, 41, 42, 41, 42, 41]]))


@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
def test_accepted_rows_are_appended_once_more(dtype, form):
    g = ref.seeded(17)
    B, Hkv, T, D, Smax = 3, 2, 7, 64, 40
    k, v = (ref.normal(g, (B, Hkv, T, D), dtype) for _ in range(2))
    r = rotary_of(D)
    rows, counts, n = ints([[0, 2, 5, 6], [0, 0, 1, 9], [-1, 3, 0, 0]]), ints([4, 4, 2]), ints([0, 30, 38])
    depth = ints([[0, 1, 1, 2, 2, 2, 3]] * 3)
    a, b = (binding.KVCache.empty(B, Hkv, Smax, D, FORMAT[form]) for _ in range(2))
    binding.kv_append(a, k, v, n, counts=counts, rows=rows, rotary=r)
    binding.kv_append(b, k, v, n, counts=counts, rows=rows, rotary=r, positions=n[:, None] + depth)
    # the same by picking the tokens first: what is out of range is left out
    for i in range(B):
        for j in range(int(counts[i])):
            t, at = int(rows[i, j]), int(n[i]) + j
            for cache, pos in ((a, at), (b, int(n[i]) + int(depth[i, t]) if 0 <= t < T else 0)):
                if not 0 <= t < T:
                    assert (cache.k[i, :, at].view(torch.uint8) == 0).all()
                    continue
                one = binding.KVCache.empty(1, Hkv, Smax, D, FORMAT[form])
                binding.kv_append(one, k[i:i + 1, :, t:t + 1].contiguous(), v[i:i + 1, :, t:t + 1].contiguous(), ints([at]),
                                  positions=ints([[pos]]), rotary=r)
                for x, y in ((cache.k, one.k), (cache.v, one.v)):
                    assert torch.equal(x[i, :, at].view(torch.uint8), y[0, :, at].view(torch.uint8))


@pytest.mark.parametrize("dtype,form", FORMS[2:], ids=IDS[2:])
def test_rows_of_zeros_tiny_ones_infinities_and_nan(dtype, form):
    x = torch.zeros((1, 1, 6, 32), dtype=dtype, device="cuda")
    x[0, 0, 1, 3] = 2.0 ** -110 if dtype == BF else 2.0 ** -24
    x[0, 0, 2, 31] = float("inf")
    x[0, 0, 3, 0] = float("nan")
    x[0, 0, 4] = torch.finfo(dtype).max
    x[0, 0, 5, :16] = -1
    cache = binding.KVCache.empty(1, 1, 6, 32, FORMAT[form])
    binding.kv_append(cache, x, x, ints([0]))
    top = ref.TOP[form]
    for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        c = t.float()[0, 0]
        assert (c[0] == 0).all() and s[0, 0, 0] == 0
        if dtype == BF:
            assert (c[1] == 0).all() and s[0, 0, 1] == 0
        else:
            assert c[1, 3] == top and s[0, 0, 1] > 0
        assert (c[2:4] == 0).all() and s[0, 0, 2:4].isnan().all()
        assert (c[4] == top).all() and torch.isfinite(s[0, 0, 4])
        assert (c[5, :16] == -top).all() and (c[5, 16:] == 0).all()
    out = torch.empty_like(x)
    binding.kv_read(cache, out, torch.empty_like(x))
    assert out[0, 0, 2:4].isnan().all() and (out[0, 0, 4] - x[0, 0, 4]).abs().max() <= 2 ** -7 * x[0, 0, 4, 0]
    assert torch.equal(out[0, 0, 5], x[0, 0, 5])


# --------------------------------------------------------------------------------------------------------------- read
@pytest.mark.parametrize("dtype,form", FORMS, ids=IDS)
@pytest.mark.parametrize("D", [16, 64, 80, 128])
def test_read(dtype, form, D):
    g = ref.seeded(21)
    B, Hkv, Smax, S = 4, 3, 301, 130
    cache = ref.make_cache(g, B, Hkv, Smax, D, form, binding)
    for first, counts in ((None, None), ([0, 100, 200, 300], [130, 7, 130, 130]), ([-3, 5, 0, 400], [0, -1, 500, 9])):
        outs = [torch.full((B, S, Hkv, D), 5.0, dtype=dtype, device="cuda").permute(0, 2, 1, 3) for _ in range(2)]
        binding.kv_read(cache, *outs, first=None if first is None else ints(first), counts=None if counts is None else ints(counts))
        binding.check_status()
        for out, codes, scale in ((outs[0], cache.k, cache.k_scale), (outs[1], cache.v, cache.v_scale)):
            want = torch.full((B, Hkv, S, D), 5.0, dtype=torch.float64, device="cuda")
            values = ref.decode_values(codes, scale)
            for b in range(B):
                f, c = (first or [0] * B)[b], min(max((counts or [S] * B)[b], 0), S)
                for i in range(c):
                    if 0 <= f + i < Smax:
                        want[b, :, i] = values[b, :, f + i]
            # the product with the scale in fp32, then one rounding
            assert ((out.double() - want).abs() <= want.abs() * (ref.HALF[dtype] + 2 * ref.F32) + 2.0 ** -25).all()


@pytest.mark.parametrize("form", [I8, E4])
def test_every_code(form):
    """All 256 bytes (but e4m3's NaN) come back as the numbers they are."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(form).view(1, 1, 2, 128)
    one = torch.ones((1, 1, 2), device="cuda")
    for dtype in (BF, HF):
        k, v = (torch.empty((1, 1, 2, 128), dtype=dtype, device="cuda") for _ in range(2))
        binding.kv_read(binding.KVCache(codes, codes, one, one), k, v)
        fine = ~codes.float().isnan()
        assert torch.equal(k[fine].float(), codes.float()[fine]) and torch.equal(k.view(torch.int16), v.view(torch.int16))


# -------------------------------------------------------------------------------------------------- the step as it is used
@pytest.mark.parametrize("form", [BF, I8, E4], ids=["bf16", "int8", "e4m3"])
def test_a_serving_loop(form):
    """Projection -> append -> attention, as a model does it: a prompt in two chunks, single tokens, a tree of drafted tokens of which a path is
    accepted, single tokens again; each step against attention in 64 bits over what the cache holds, and the cache against the
    projections' rows.  One captured graph does the single tokens."""
    g = ref.seeded(31)
    B, Hq, Hkv, D, Smax, W = 2, 8, 2, 64, 160, 256
    w = ref.normal(g, (W, (Hq + 2 * Hkv) * D), BF, W ** -0.5)
    cache = binding.KVCache.empty(B, Hkv, Smax, D, FORMAT[form])
    r = rotary_of(D)
    ws = torch.empty(binding.attn_kv_workspace_bytes(B, Hq, Hkv, 64, D), dtype=torch.uint8, device="cuda")
    binding.attn_kv_workspace_init(ws)
    lens = ints([0, 0])

    def project(T):
        x = ref.normal(g, (B * T, W), BF)
        qkv = binding.linear_act(x, w, act=binding.ACT_NONE).view(B, T, Hq + 2 * Hkv, D)
        return (t.permute(0, 2, 1, 3) for t in qkv.split([Hq, Hkv, Hkv], 2))

    def step(T, positions=None, counts=None, sees=None):
        q, k, v = project(T)
        q2 = binding.kv_append(cache, k, v, lens, counts=counts, positions=positions, rotary=r, q=q)
        out = binding.attn_tree(q2, cache, lens, None if sees is None else ref.tree_bits(sees), workspace=ws)
        binding.check_status()
        mask = torch.ones((T, T), dtype=torch.bool, device="cuda").tril().expand(B, T, T) if sees is None else sees
        want, bound = ref.attention(q2, cache, lens, mask)
        if counts is None:
            ref.assert_within(out, want, bound)
        else:
            for b in range(B):
                ref.assert_within(out[b, :, :int(counts[b])], want[b, :, :int(counts[b])], bound[b, :, :int(counts[b])])
        return k, v

    step(40)
    lens += 40
    step(33, counts=ints([33, 20]))  # the second prompt is shorter
    lens += ints([33, 20])
    # a cached prefix read back feeds the prefill attention
    n = int(lens.max())
    kd, vd = (torch.zeros((B, Hkv, n, D), dtype=BF, device="cuda") for _ in range(2))
    binding.kv_read(cache, kd, vd, counts=lens)
    q = ref.normal(g, (B, Hq, 5, D), BF)
    out = binding.attn_fused(q, kd, vd, binding.MASK_PADDING, lens)
    # the rows are rounded once more, and P to bf16
    want, bound = ref.attention(q, cache, lens, rows_off=0.0 if form == BF else 2 ** -8, half_p=2 ** -8)
    ref.assert_within(out, want, bound)
    # single tokens, captured
    qkv = torch.zeros((B, 1, Hq + 2 * Hkv, D), dtype=BF, device="cuda")
    q1, k1, v1 = (t.permute(0, 2, 1, 3) for t in qkv.split([Hq, Hkv, Hkv], 2))
    q2, out = torch.zeros((B, Hq, 1, D), dtype=BF, device="cuda"), torch.zeros((B, Hq, 1, D), dtype=BF, device="cuda")
    before = lens.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.kv_append(cache, k1, v1, lens, rotary=r, q=q1, q_out=q2)
        binding.attn_tree(q2, cache, lens, out=out, workspace=ws)
        lens += 1
    for _ in range(3):
        qkv.copy_(ref.normal(g, qkv.shape, BF))
        graph.replay()
        torch.cuda.synchronize()
        want, bound = ref.attention(q2, cache, lens)
        ref.assert_within(out, want, bound)
        assert torch.equal(binding.attn_decode_kv(q2[:, :, 0].contiguous(), cache, lens), out[:, :, 0])
    assert torch.equal(lens, before + 3)
    # a tree, and the path of it that is accepted
    T = 9
    sees = ref.random_tree(g, B, T)
    depth = sees.sum(-1, dtype=torch.int32) - 1
    k, v = step(T, positions=lens[:, None] + depth, sees=sees)
    paths = [[u for u in range(T) if sees[b, T - 1, u]] for b in range(B)]
    m = max(map(len, paths))
    rows = ints([p + [0] * (m - len(p)) for p in paths])
    binding.kv_append(cache, k, v, lens, counts=ints([len(p) for p in paths]), rows=rows, rotary=r)
    for b, path in enumerate(paths):
        at = int(lens[b])
        pos = torch.arange(at, at + len(path), device="cuda")[None]
        want, err = ref.rotate(k[b:b + 1, :, path], pos, r.inv_freq)
        sl = lambda t: None if t is None else t[b, :, at:at + len(path)]  # noqa: E731
        ref.assert_rows_kept(sl(cache.k), sl(cache.k_scale), want[0], err[0], "k")
        ref.assert_rows_kept(sl(cache.v), sl(cache.v_scale), v[b, :, path].double(), torch.zeros_like(want[0]), "v")
    lens += ints([len(p) for p in paths])
    step(1)
