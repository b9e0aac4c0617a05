"""Host-only checks of the operators of a step of many requests (pages, adapters): the refusals, which come before any launch."""
import ctypes

import pytest
import torch

from paper_2604_16498_b200 import binding, build

P = 0x10000  # a fake, aligned pointer: validation must reject the call before touching it
I64x2, I64x3 = ctypes.c_int64 * 2, ctypes.c_int64 * 3
BAD, UNS, WS = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def pages(**kw):
    a = dict(k=P, v=P, k_scale=P, v_scale=P, num_pages=9, Hkv=2, page_size=16, D=64, format=binding.KV_INT8)
    a.update(kw)
    return binding.KVPagesDesc(**a)


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 4), dict(k_scale=None), dict(v_scale=None), dict(k_scale=P + 4), dict(num_pages=0),
             dict(num_pages=-1), dict(Hkv=0), dict(page_size=0), dict(page_size=-16), dict(D=0), dict(format=4), dict(format=-1)]
UNSUPPORTED_PAGES = [dict(page_size=8), dict(page_size=24), dict(page_size=48), dict(page_size=1 << 21), dict(D=136), dict(D=72), dict(Hkv=70000),
                     dict(num_pages=1 << 26), dict(num_pages=1 << 30, page_size=1 << 20)]


def tables(**kw):
    a = dict(table=P, free_pages=P, free_count=P, B=3, max_pages=4, page_size=16, num_pages=9)
    a.update(kw)
    return binding.PageTablesDesc(**a)


def test_assign_and_release_refusals(lib):
    def assign(t=tables(), lens=P, counts=None, T=8, new_lens=P, starts=None, slots=P, positions=None, requests=None, left=None):
        out = binding.PageSlotsDesc(new_lens, starts, slots, positions, requests, T)
        return lib.forge_kv_assign_pages(None if t is None else ctypes.byref(t), lens, counts, ctypes.byref(out), left, None)

    def release(t=tables(), lens=P, done=P, left=None):
        return lib.forge_kv_release_pages(None if t is None else ctypes.byref(t), lens, done, left, None)

    bad = [dict(t=None), dict(lens=None), dict(lens=P + 2), dict(left=P + 1)]
    bad += [dict(t=tables(**kw)) for kw in (dict(table=None), dict(table=P + 2), dict(free_pages=None), dict(free_pages=P + 1), dict(free_count=None),
                                            dict(free_count=P + 2), dict(B=0), dict(B=-1), dict(max_pages=0), dict(page_size=0), dict(num_pages=0))]
    unsupported = [dict(t=tables(**kw)) for kw in (dict(page_size=8), dict(page_size=17), dict(page_size=1 << 21), dict(B=65536),
                                                   dict(max_pages=(1 << 26) + 1), dict(num_pages=1 << 27))]
    for kw in bad:
        assert assign(**kw) == BAD and release(**kw) == BAD, kw
    for kw in unsupported:
        assert assign(**kw) == UNS and release(**kw) == UNS, kw
    for kw in (dict(T=0), dict(T=-1), dict(new_lens=None), dict(slots=None), dict(counts=P + 2), dict(new_lens=P + 1), dict(starts=P + 2),
               dict(slots=P + 3), dict(positions=P + 2), dict(requests=P + 1)):
        assert assign(**kw) == BAD, kw
    assert assign(T=(1 << 30) + 1) == UNS
    assert lib.forge_kv_assign_pages(ctypes.byref(tables()), P, None, None, None, None) == BAD
    assert release(done=None) == BAD and release(done=P + 2) == BAD


def test_append_refusals(lib):
    rot = binding.RotaryDesc(inv_freq=P, dims=64, layout=0, amplitude=1.0)

    def call(c=pages(), rotary=rot, **kw):
        a = dict(k=P, v=P, q=P, q_out=P, slots=P, positions=P, dtype=0, Hq=4, T=5)
        strides = {x: kw.pop(x) for x in ("k_strides", "v_strides", "q_strides", "q_out_strides") if x in kw}
        a.update(kw)
        d = binding.KVAppendPagesDesc(**a)
        for name, x in strides.items():
            setattr(d, name, x)
        if rotary is not None:
            d.rotary = ctypes.pointer(rotary)
        return lib.forge_kv_append_pages(None if c is None else ctypes.byref(c), ctypes.byref(d), None)

    assert lib.forge_kv_append_pages(ctypes.byref(pages()), None, None) == BAD
    assert call(c=None) == BAD
    for kw in BAD_PAGES:
        assert call(c=pages(**kw)) == BAD, kw
    for kw in UNSUPPORTED_PAGES:
        assert call(c=pages(**kw)) == UNS, kw
    for kw in (dict(k=None), dict(v=None), dict(k=P + 8), dict(slots=None), dict(slots=P + 2), dict(positions=P + 2), dict(positions=None), dict(T=0),
               dict(dtype=3), dict(q_out=None), dict(q=None), dict(Hq=0), dict(q=P + 8), dict(rotary=None), dict(k_strides=I64x2(0, 64)),
               dict(q_strides=I64x2(256, -64)), dict(q_out_strides=I64x2(512, 64)),
               dict(rotary=binding.RotaryDesc(inv_freq=P, dims=66, layout=0, amplitude=1.0))):
        assert call(**kw) == BAD, kw
    for kw in (dict(dtype=2), dict(v_strides=I64x2(130, 64)), dict(Hq=70000)):
        assert call(**kw) == UNS, kw
    assert call(c=pages(format=binding.KV_F16)) == BAD  # a 16-bit cache has the activations' type


def test_read_refusals(lib):
    def call(c=pages(), table=P, B=3, max_pages=4, k=P, v=P, dtype=0, S=7, ks=None, vs=None, first=None, counts=None):
        return lib.forge_kv_read_pages(None if c is None else ctypes.byref(c), table, B, max_pages, k, v, dtype, S, ks, vs, first, counts, None)

    for kw in BAD_PAGES:
        assert call(c=pages(**kw)) == BAD, kw
    for kw in UNSUPPORTED_PAGES:
        assert call(c=pages(**kw)) == UNS, kw
    for kw in (dict(c=None), dict(table=None), dict(table=P + 2), dict(B=0), dict(max_pages=0), dict(k=None), dict(v=P + 8), dict(S=0), dict(dtype=5),
               dict(first=P + 2), dict(counts=P + 1), dict(ks=I64x3(8, 0, 8))):
        assert call(**kw) == BAD, kw
    for kw in (dict(B=65536), dict(max_pages=(1 << 26) + 1), dict(dtype=2), dict(vs=I64x3(8, 8, 12))):
        assert call(**kw) == UNS, kw


def test_attention_refusals(lib):
    def decode(c=pages(), table=P, B=3, max_pages=4, q=P, out=P, dtype=0, Hq=4, lens=P, scale=0.1, ws=P, n=1 << 30):
        return lib.forge_attn_decode_pages(None if c is None else ctypes.byref(c), table, B, max_pages, q, out, dtype, Hq, lens, scale, ws, n, None)

    def tree(c=pages(), table=P, B=3, max_pages=4, q=P, out=P, dtype=0, Hq=4, lens=P, scale=0.1, ws=P, n=1 << 30, T=5, qs=None, os=None, tree=P,
             tree_B=None):
        return lib.forge_attn_tree_pages(None if c is None else ctypes.byref(c), table, B, max_pages, q, out, dtype, Hq, T, qs, os, lens, tree, B if tree_B is None else tree_B,
                                         scale, ws, n, None)

    for f in (decode, tree):
        for kw in BAD_PAGES:
            assert f(c=pages(**kw)) == BAD, kw
        for kw in UNSUPPORTED_PAGES:
            assert f(c=pages(**kw)) == UNS, kw
        for kw in (dict(c=None), dict(table=None), dict(table=P + 2), dict(B=0), dict(max_pages=-1), dict(q=None), dict(out=None), dict(q=P + 8),
                   dict(lens=None), dict(lens=P + 2), dict(Hq=3), dict(Hq=0), dict(ws=None), dict(ws=P + 8), dict(dtype=3)):
            assert f(**kw) == BAD, kw
        for kw in (dict(dtype=2), dict(Hq=70000), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(B=65536),
                   dict(max_pages=(1 << 26) + 1), dict(B=60000, max_pages=1 << 20)):
            assert f(**kw) == UNS, kw
        assert f(n=1000) == WS
    for kw in (dict(T=0), dict(tree=P + 4), dict(tree_B=2), dict(qs=I64x3(0, 8, 8))):
        assert tree(**kw) == BAD, kw
    for kw in (dict(T=65), dict(os=I64x3(8, 8, 4))):
        assert tree(**kw) == UNS, kw


def test_adapters_refusals(lib):
    def call(s="given", x=P, y=P + 4096, out=P + 8192, T=3, xs=0, ys=0, os=0, requests=P, adapters=P, R=2, ws=None, nws=0, **kw):
        a = dict(a=P, b=P, scales=P, n=2, rank=16, K=64, N=64, dtype=0)
        a.update(kw)
        d = binding.AdaptersDesc(**a)
        return lib.forge_linear_adapters(None if s is None else ctypes.byref(d), x, y, out, T, xs, ys, os, requests, adapters, R, ws, nws, None)

    for kw in (dict(s=None), dict(a=None), dict(b=None), dict(a=P + 8), dict(b=P + 2), dict(scales=P + 2), dict(n=0), dict(rank=0), dict(K=0), dict(N=-8),
               dict(dtype=3), dict(dtype=-1), dict(x=None), dict(y=None), dict(out=None), dict(x=P + 8), dict(y=P + 8), dict(out=P + 4), dict(T=0),
               dict(R=0), dict(adapters=None), dict(adapters=P + 2), dict(requests=P + 2), dict(requests=None), dict(xs=56), dict(ys=32), dict(os=63),
               dict(xs=-64), dict(y=P, out=P, ys=128, os=64)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dtype=2), dict(rank=12), dict(rank=136), dict(K=60), dict(N=68), dict(xs=68), dict(ys=70), dict(os=66),
               dict(n=1 << 26), dict(n=1 << 28, N=8), dict(T=(1 << 30) + 1, ws=P, nws=1 << 60)):
        assert call(**kw) == UNS, kw
    # many tokens need a workspace
    need = lib.forge_linear_adapters_workspace_bytes(600, 16)
    assert need >= 600 * (16 * 4 + 8) and lib.forge_linear_adapters_workspace_bytes(512, 16) == 0
    assert lib.forge_linear_adapters_workspace_bytes(600, 130) == 0 and lib.forge_linear_adapters_workspace_bytes(-5, 16) == 0
    assert call(T=600) == BAD and call(T=600, ws=P + 8, nws=need) == BAD and call(T=600, ws=P, nws=need - 1) == WS


def test_the_binding_checks_shapes_and_places():
    i32 = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.KVPages(x[None], x[None])  # not on the GPU
    with pytest.raises(ValueError):
        binding.KVPages(x[None].to(torch.int8), x[None].to(torch.int8))  # 8-bit rows without scales
    with pytest.raises(ValueError):
        binding.KVPages(x, x)
    with pytest.raises(ValueError):
        binding.PageTables(i32[None], i32, i32, 16)
    with pytest.raises(ValueError):
        binding.PageSlots(i32, None, i32)
    with pytest.raises(ValueError):
        binding.linear_adapters(x[:, 0], x[:, 0], x, x, i32)
    with pytest.raises(ValueError):
        binding.linear_adapters(x[:, 0].float(), x[:, 0], x, x, i32)
    with pytest.raises(ValueError):
        binding.linear_adapters(x, x, x, x, i32)


# ------------------------------------------------------------------------------------------------------- native marshalling
def test_what_is_not_plain_goes_the_general_way():
    binding.load()
    c = binding._host_calls
    assert c is not None
    for bad in ((), (1,) * 6, (1,) * 8, (0,) * 7, ("x",) * 7):
        with pytest.raises((TypeError, ValueError)):
            c.bind_pages(*bad)
    x, i, t = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 3, dtype=torch.int32)
    ws = torch.zeros(64, dtype=torch.uint8)
    for desc in (pages(), tables()):
        at = ctypes.addressof(desc)
        for dev in (0, None, "0", 1 << 40):
            assert c.assign_pages(at, dev, i, None, at, dev, 3, None) == -1
            assert c.append_pages(at, dev, x, x, i, None, None, None, None, None) == -1
            assert c.read_pages(at, dev, t, x[None], x[None], None, None) == -1
            assert c.decode_pages(at, dev, x, t, i, None, x, ws) == -1
            assert c.tree_pages(at, dev, x[None], t, i, None, None, x[None], ws) == -1
    assert c.adapters(x[:, 0], x[:, 0], x, x, i, None, None, x[:, 0], None) == -1
    for fn in (c.assign_pages, c.append_pages, c.read_pages, c.decode_pages, c.tree_pages, c.adapters):
        for bad in ((), (None,), (None,) * 7, (None,) * 8, (None,) * 9, (None,) * 10, (x,) * 8, (0,) * 10):
            assert fn(*bad) == -1
