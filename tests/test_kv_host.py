"""Host-only checks of the operators around the KV cache: the rotary frequencies against their formulas, and the refusals, which come
before any launch."""
import ctypes
import math

import pytest
import torch

from paper_2604_16498_b200 import binding, build

P = 0x10000  # a fake, aligned pointer: validation must reject the call before touching it
I64 = ctypes.c_int64 * 3


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


# ------------------------------------------------------------------------------------------------------- frequencies
def scaling(kind, factor=4.0, fast=32.0, slow=1.0, original_len=4096):
    return binding.RotaryScaling(kind, factor, fast, slow, original_len)


def assert_frequencies(got, want):
    want = torch.tensor(want, dtype=torch.float64)
    # rounded once to fp32; pow and log are a few 2^-53 off in either library
    assert ((got.double() - want).abs() <= want * (2.0 ** -24 + 2.0 ** -40)).all()


@pytest.mark.parametrize("dims,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (96, 1e6), (256, 10000.0)])
def test_plain_frequencies(dims, base):
    f, amplitude = binding.rotary_frequencies(dims, base)
    assert f.shape == (dims // 2,) and amplitude == 1.0
    assert_frequencies(f, [base ** (-2 * i / dims) for i in range(dims // 2)])
    g, _ = binding.rotary_frequencies(dims, base, scaling(binding.ROTARY_SCALE_NONE))
    assert torch.equal(f, g)


def test_scaled_frequencies():
    dims, base, n = 128, 10000.0, 64
    plain = [base ** (-2 * i / dims) for i in range(n)]
    f, a = binding.rotary_frequencies(dims, base, scaling(binding.ROTARY_SCALE_LINEAR))
    assert a == 1.0
    assert_frequencies(f, [x / 4 for x in plain])
    f, a = binding.rotary_frequencies(dims, base, scaling(binding.ROTARY_SCALE_BASE))
    b2 = base * 4 ** (dims / (dims - 2))
    assert a == 1.0 and abs(float(f[-1]) * 4 - plain[-1]) < 1e-6 * plain[-1]  # the slowest pair is slowed by the factor
    assert_frequencies(f, [b2 ** (-2 * i / dims) for i in range(n)])
    # ramp over indices: bounds of the indices that make 32 and 1 turns over 4096 positions
    lo = math.floor(dims * math.log(4096 / (32 * 2 * math.pi)) / (2 * math.log(base)))
    hi = math.ceil(dims * math.log(4096 / (1 * 2 * math.pi)) / (2 * math.log(base)))
    assert 0 < lo < hi < n
    f, a = binding.rotary_frequencies(dims, base, scaling(binding.ROTARY_SCALE_RAMP_ROTATIONS))
    ramp = [min(max((i - lo) / (hi - lo), 0), 1) for i in range(n)]
    assert_frequencies(f, [x * (1 - r) + x / 4 * r for x, r in zip(plain, ramp)])
    assert abs(a - (0.1 * math.log(4) + 1)) < 1e-7
    # ramp over wavelengths
    f, a = binding.rotary_frequencies(dims, base, scaling(binding.ROTARY_SCALE_RAMP_WAVELENGTH, 8.0, 4.0, 1.0, 8192))
    want = []
    for x in plain:
        wavelength = 2 * math.pi / x
        if wavelength < 8192 / 4:
            want.append(x)
        elif wavelength > 8192:
            want.append(x / 8)
        else:
            s = (8192 / wavelength - 1) / 3
            want.append((1 - s) * x / 8 + s * x)
    assert a == 1.0 and want[0] == plain[0] and want[-1] == plain[-1] / 8
    assert_frequencies(f, want)


@pytest.mark.parametrize("kind", range(5))
def test_factor_one_changes_nothing(kind):
    f, a = binding.rotary_frequencies(64, 10000.0, scaling(kind, 1.0))
    assert_frequencies(f, [10000.0 ** (-2 * i / 64) for i in range(32)])
    assert a == 1.0


def test_frequencies_refusals():
    for dims, base, s in [(0, 1e4, None), (3, 1e4, None), (64, 1.0, None), (64, float("nan"), None), (64, float("inf"), None),
                          (64, 1e4, scaling(5)), (64, 1e4, scaling(-1)), (64, 1e4, scaling(1, 0.5)), (64, 1e4, scaling(1, float("nan"))),
                          (2, 1e4, scaling(2)), (64, 1e4, scaling(3, 4.0, 1.0, 1.0)), (64, 1e4, scaling(4, 4.0, 4.0, 0.0)),
                          (64, 1e4, scaling(3, 4.0, 32.0, 1.0, 0))]:
        with pytest.raises(binding.ForgeError) as e:
            binding.rotary_frequencies(dims, base, s)
        assert e.value.status == binding.ERR_INVALID_ARG


# ---------------------------------------------------------------------------------------------------------- refusals
def rotary(dims=64, layout=0, ptr=P):
    return binding.RotaryDesc(inv_freq=ptr, dims=dims, layout=layout, amplitude=1.0)


def cache(**kw):
    a = dict(k=P, v=P, k_scale=P, v_scale=P, B=2, Hkv=2, Smax=100, D=64, format=binding.KV_INT8)
    a.update(kw)
    return binding.KVCacheDesc(**a)


def test_rotary_refusals(lib):
    ok = dict(x=P, y=P + 1024, dtype=0, B=2, H=3, S=4, D=64, xs=None, ys=None, pos=None, first=None, r=rotary(), inverse=0)

    def call(**kw):
        a = {**ok, **kw}
        r = a["r"]
        return lib.forge_rotary_apply(a["x"], a["y"], a["dtype"], a["B"], a["H"], a["S"], a["D"], a["xs"], a["ys"], a["pos"], a["first"],
                                      None if r is None else ctypes.byref(r), a["inverse"], None)

    bad, uns = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    for kw in (dict(x=None), dict(y=None), dict(x=P + 8), dict(y=P + 2), dict(dtype=3), dict(dtype=-1), dict(B=0), dict(H=0), dict(S=-1), dict(D=0),
               dict(pos=P + 2), dict(first=P + 1), dict(r=None), dict(r=rotary(ptr=None)), dict(r=rotary(ptr=P + 2)), dict(r=rotary(0)),
               dict(r=rotary(63)), dict(r=rotary(66)), dict(r=rotary(layout=2)), dict(xs=I64(0, 64, 64)), dict(ys=I64(768, -256, 64)),
               dict(y=P, ys=I64(768, 64, 192))):
        assert call(**kw) == bad, kw
    for kw in (dict(D=60, r=rotary(60)), dict(D=264), dict(xs=I64(768, 256, 68)), dict(H=70000)):
        assert call(**kw) == uns, kw


def append_desc(**kw):
    a = dict(k=P, v=P, q=None, q_out=None, lens=P, counts=None, positions=None, rows=None, dtype=0, Hq=0, S=3, S_src=3)
    strides = {n: kw.pop(n) for n in list(kw) if n.endswith("_strides")}
    r = kw.pop("rotary", None)
    a.update(kw)
    d = binding.KVAppendDesc(**a)
    for n, s in strides.items():
        setattr(d, n, s)
    if r is not None:
        d.rotary = ctypes.pointer(r)
    return d


def test_append_refusals(lib):
    def call(c=None, **kw):
        return lib.forge_kv_append(cache() if c is None else c, append_desc(**kw), None)

    bad, uns = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    assert lib.forge_kv_append(None, append_desc(), None) == bad and lib.forge_kv_append(cache(), None, None) == bad
    for c in (cache(k=None), cache(v=P + 8), cache(k_scale=None), cache(v_scale=P + 4), cache(B=0), cache(Hkv=-1), cache(Smax=0), cache(D=0),
              cache(format=4), cache(format=-1), cache(format=binding.KV_F16)):  # the last: bf16 rows for an fp16 cache
        assert call(c) == bad
    for c in (cache(D=72), cache(D=256), cache(D=12, format=binding.KV_BF16), cache(B=70000), cache(B=60000, Hkv=60000)):
        assert call(c) == uns
    assert call(dtype=2) == uns and call(dtype=7) == bad
    q = dict(q=P, q_out=P, Hq=4, rotary=rotary())
    for kw in (dict(k=None), dict(v=P + 4), dict(lens=None), dict(lens=P + 2), dict(counts=P + 1), dict(positions=P + 3), dict(rows=P + 2),
               dict(S=0), dict(rows=P, S_src=0), dict(rotary=rotary(66)), dict(k_strides=I64(0, 8, 8)), dict(q_out=P),
               {**q, "q_out": None}, {**q, "rotary": None}, {**q, "Hq": 0}, {**q, "q": P + 8}, {**q, "rows": P},
               {**q, "q_strides": I64(768, 192, 64), "q_out_strides": I64(768, 64, 256)}):
        assert call(**kw) == bad, kw
    for kw in (dict(v_strides=I64(768, 192, 12)), {**q, "Hq": 70000}):
        assert call(**kw) == uns, kw


def test_read_refusals(lib):
    def call(c=None, k=P, v=P, dtype=0, S=5, ks=None, vs=None, first=None, counts=None):
        return lib.forge_kv_read(cache() if c is None else c, k, v, dtype, S, ks, vs, first, counts, None)

    bad, uns = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    for kw in (dict(c=cache(k=None)), dict(k=None), dict(v=P + 8), dict(dtype=9), dict(S=0), dict(ks=I64(8, 8, 0)), dict(first=P + 2), dict(counts=P + 1),
               dict(c=cache(format=binding.KV_BF16), dtype=1)):
        assert call(**kw) == bad, kw
    for kw in (dict(dtype=2), dict(vs=I64(8, 8, 4)), dict(S=2**31 - 1)):
        assert call(**kw) == uns, kw


def test_attention_refusals(lib):
    need = lib.forge_attn_kv_workspace_bytes(2, 8, 2, 5, 64)
    assert need == 65536 * 4 + 160 * 2 * (128 * 68 * 4)
    assert lib.forge_attn_kv_workspace_bytes(2, 8, 2, 1, 128) == 65536 * 4 + 160 * 2 * (8 * 132 * 4)
    assert lib.forge_attn_kv_workspace_bytes(1000, 128, 128, 64, 64) == 128000 * 4 + 160 * 2 * (128 * 68 * 4)
    for args in ((0, 8, 2, 5, 64), (2, 8, 3, 5, 64), (2, 8, 2, 0, 64), (2, 8, 2, 5, 0), (2, 0, 2, 5, 64)):
        assert lib.forge_attn_kv_workspace_bytes(*args) == 0

    def tree(c=None, q=P, out=P, dtype=0, Hq=8, T=5, qs=None, os_=None, lens=P, mask=None, mask_B=1, scale=1.0, ws=P, wsb=None):
        return lib.forge_attn_tree(cache() if c is None else c, q, out, dtype, Hq, T, qs, os_, lens, mask, mask_B, scale, ws,
                                   need if wsb is None else wsb, None)

    def decode(c=None, q=P, out=P, dtype=0, Hq=8, lens=P, scale=1.0, ws=P, wsb=1 << 30):
        return lib.forge_attn_decode_kv(cache() if c is None else c, q, out, dtype, Hq, lens, scale, ws, wsb, None)

    bad, uns, small = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
    for f in (tree, decode):
        for kw in (dict(c=cache(v=None)), dict(q=None), dict(out=P + 8), dict(lens=None), dict(lens=P + 2), dict(Hq=0), dict(Hq=7), dict(ws=None),
                   dict(ws=P + 8), dict(c=cache(format=binding.KV_BF16), dtype=1), dict(dtype=5)):
            assert f(**kw) == bad, kw
        for kw in (dict(c=cache(D=72)), dict(c=cache(D=136)), dict(dtype=2), dict(scale=float("nan")), dict(scale=float("inf"))):
            assert f(**kw) == uns, kw
        assert f(wsb=1000) == small
    for kw in (dict(T=0), dict(mask=P + 4), dict(mask=P, mask_B=3), dict(mask=P, mask_B=0), dict(qs=I64(0, 8, 8))):
        assert tree(**kw) == bad, kw
    for kw in (dict(T=65), dict(os_=I64(8, 8, 4)), dict(c=cache(B=2000, Hkv=2000, Smax=500000))):
        assert tree(**kw) == uns, kw
    assert tree(wsb=need - 1) == small


# -------------------------------------------------------------------------------------------------------- the binding
def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    bf = torch.bfloat16
    x, lens = torch.zeros((2, 3, 4, 64), dtype=bf), torch.zeros((2,), dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.Rotary(torch.zeros(32))
    with pytest.raises(ValueError):
        binding.KVCache(x, x)
    with pytest.raises(ValueError):
        binding.KVCache(x, x[:1])
    with pytest.raises(ValueError):
        binding.KVCache(x.float(), x.float())
    with pytest.raises(ValueError):
        binding.KVCache(x, x, torch.zeros((2, 3, 4)), torch.zeros((2, 3, 4)))
    with pytest.raises(ValueError):
        binding.KVCache(x.to(torch.int8), x.to(torch.int8))
    # stand-ins for handles whose tensors are on a GPU
    c = binding.KVCache.__new__(binding.KVCache)
    c.B, c.Hkv, c.Smax, c.D, c.k, c.desc = 2, 3, 4, 64, x, cache(Hkv=3, Smax=4, format=0)
    c.address, c.device = ctypes.addressof(c.desc), 0
    r = binding.Rotary.__new__(binding.Rotary)
    r.inv_freq, r.desc = torch.zeros(32), rotary()
    r.address, r.device = ctypes.addressof(r.desc), 0
    for call in (lambda: binding.rotary_apply(x, r), lambda: binding.rotary_apply(x.to(torch.int8), r), lambda: binding.kv_append(c, x, x, lens),
                 lambda: binding.kv_append(c, x[:, :2], x, lens), lambda: binding.kv_append(c, x.float(), x.float(), lens),
                 lambda: binding.kv_append(c, x, x, lens, rows=lens), lambda: binding.kv_read(c, x, x), lambda: binding.kv_read(c, x[0], x),
                 lambda: binding.attn_decode_kv(x[:, :, 0], c, lens), lambda: binding.attn_decode_kv(x[:1, :, 0], c, lens),
                 lambda: binding.attn_tree(x, c, lens), lambda: binding.attn_tree(x, c, lens, torch.zeros((3, 4), dtype=torch.int64)),
                 lambda: binding.attn_tree(x.float(), c, lens), lambda: binding.attn_kv_workspace_init(lens)):
        with pytest.raises(ValueError):
            call()


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The library launches on the current device, whatever device the tensors are on."""
    class On:
        def __init__(self, index):
            self.device = torch.device("cuda", index)
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    binding._on_current(On(1), None, On(1))
    with pytest.raises(ValueError, match="cuda:0"):
        binding._on_current(On(1), None, On(0))


def test_scales_that_the_exponentials_base_takes_out_of_range_are_refused(lib):
    """Scores are kept in powers of two: scale * log2(e) has to be a finite fp32 number."""
    for scale in (2.4e38, -3e38, 3.4028234e38):
        assert lib.forge_attn_decode_kv(cache(), P, P, 0, 8, P, scale, P, 1 << 30, None) == binding.ERR_UNSUPPORTED
        assert lib.forge_attn_tree(cache(), P, P, 0, 8, 5, None, None, P, None, 1, scale, P, 1 << 30, None) == binding.ERR_UNSUPPORTED
