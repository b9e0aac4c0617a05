"""The native marshalling of the calls around the KV cache: what it takes it does as the general Python way does, and what is not plain
it leaves to that way, which has the checks and the errors."""
import ctypes

import pytest
import torch

from paper_2604_16498_b200 import binding

NOT_PLAIN = -1
FORMATS = {torch.bfloat16: (binding.KV_BF16, binding.KV_INT8, binding.KV_E4M3), torch.float16: (binding.KV_F16, binding.KV_INT8, binding.KV_E4M3)}


class _Sub(torch.Tensor):
    pass


def _calls():
    binding.load()
    assert binding._host_calls is not None
    return binding._host_calls


def test_bind_kv_wants_five_addresses():
    c = _calls()
    for bad in ((), (1,) * 4, (1,) * 6, (0,) * 5, ("x",) * 5):
        with pytest.raises((TypeError, ValueError)):
            c.bind_kv(*bad)


def test_anything_else_goes_the_general_way():
    c = _calls()
    x = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    ws = torch.zeros(64, dtype=torch.uint8)
    handle = binding.KVCacheDesc(B=1, Hkv=2, Smax=8, D=64)  # stands for either kind of handle
    desc = ctypes.addressof(handle)
    for dev in (0, None, "0", 1 << 40):
        assert c.rotary(x, desc, dev, None, None, 0, x) == NOT_PLAIN
        assert c.append(desc, dev, x, x, i, None, None, None, None, None, None, None) == NOT_PLAIN
        assert c.read(desc, dev, x, x, None, None) == NOT_PLAIN
        assert c.decode_kv(desc, dev, x[:, :, 0], i, None, x[:, :, 0], ws) == NOT_PLAIN
        assert c.tree(desc, dev, x, i, None, None, x, ws) == NOT_PLAIN
    for fn in (c.rotary, c.append, c.read, c.decode_kv, c.tree):
        for bad in ((), (None,), (None,) * 6, (None,) * 7, (None,) * 8, (None,) * 12, (x,) * 7, (0,) * 12):
            assert fn(*bad) == NOT_PLAIN


class _Step:
    """A cache with some rows, and the tensors of one step."""

    def __init__(self, dtype, fmt, B=3, Hq=6, Hkv=2, S=5, Smax=70, D=64):
        g = torch.Generator(device="cuda").manual_seed(11)
        r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
        i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
        self.cache = binding.KVCache.empty(B, Hkv, Smax, D, fmt)
        self.rotary = binding.Rotary(binding.rotary_frequencies(D, 10000.0)[0].cuda())
        self.k, self.v, self.q = r(B, Hkv, S, D), r(B, Hkv, S, D), r(B, S, Hq, D).transpose(1, 2)
        self.lens, self.counts = i32(40, 0, 65), i32(5, 2, 0)
        self.positions, self.rows = i32(*range(7, 7 + B * S)).view(B, S), i32(*([4, 0, 2] * B)).view(B, 3)
        self.ws = torch.empty(binding.attn_kv_workspace_bytes(B, Hq, Hkv, S, D), dtype=torch.uint8, device="cuda")
        binding.attn_kv_workspace_init(self.ws)
        binding.kv_append(self.cache, r(B, Hkv, Smax, D), r(B, Hkv, Smax, D), i32(0, 0, 0))

    def tensors(self):
        c = self.cache
        return [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]

    def restore(self, kept):
        c = self.cache
        for t, k in zip([t for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None], kept):
            t.copy_(k)


def _same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt", [(t, f) for t in FORMATS for f in FORMATS[t]])
def test_the_step_equals_the_general_way(monkeypatch, dtype, fmt):
    c, s = _calls(), _Step(dtype, fmt)

    def general(fn, *a, **kw):
        with monkeypatch.context() as m:
            m.setattr(binding, "_host_calls", None)
            return fn(*a, **kw)

    cache, rot = s.cache, s.rotary
    for pos, first, inverse in ((None, None, 0), (s.positions, None, 1), (None, s.lens, 0)):
        out = torch.empty_like(s.q)
        assert c.rotary(s.q, rot.address, rot.device, pos, first, inverse, out) == binding.OK
        assert torch.equal(out, general(binding.rotary_apply, s.q, rot, pos, first, inverse))
    kept = s.tensors()
    for counts, pos, rows, r, with_q in ((None, None, None, None, False), (s.counts, s.positions, None, rot, True), (s.counts, s.positions, s.rows, rot, False)):
        q, out = (s.q, torch.zeros_like(s.q)) if with_q else (None, None)  # rows behind counts stay
        s.restore(kept)
        assert c.append(cache.address, cache.device, s.k, s.v, s.lens, counts, pos, rows, None if r is None else r.address,
                        None if r is None else r.device, q, out) == binding.OK
        got = s.tensors()
        s.restore(kept)
        want = None if q is None else torch.zeros_like(q)
        general(binding.kv_append, cache, s.k, s.v, s.lens, counts, pos, rows, r, q, want)
        assert _same(got, s.tensors()) and (q is None or torch.equal(out, want))
    for first, counts in ((None, None), (s.lens, s.counts)):
        k, v, k2, v2 = (torch.zeros_like(s.k) for _ in range(4))
        assert c.read(cache.address, cache.device, k, v, first, counts) == binding.OK
        general(binding.kv_read, cache, k2, v2, first, counts)
        assert torch.equal(k, k2) and torch.equal(v, v2)
    out, q1 = torch.empty_like(s.q), s.q[:, :, 0].contiguous()
    tree = torch.tensor([[1, 3, 5, 11, 21]], dtype=torch.int64, device="cuda")
    for scale in (None, 0.25):
        for t in (None, tree, tree.repeat(3, 1)):
            assert c.tree(cache.address, cache.device, s.q, s.lens, t, scale, out, s.ws) == binding.OK
            assert torch.equal(out, general(binding.attn_tree, s.q, cache, s.lens, t, scale, workspace=s.ws))
        o1 = torch.empty_like(q1)
        assert c.decode_kv(cache.address, cache.device, q1, s.lens, scale, o1, s.ws) == binding.OK
        assert torch.equal(o1, general(binding.attn_decode_kv, q1, cache, s.lens, scale, workspace=s.ws))
    binding.check_status()


@pytest.mark.gpu
def test_whatever_is_not_plain_is_left_to_the_general_way():
    c, s = _calls(), _Step(torch.bfloat16, binding.KV_INT8)
    a, d = s.cache.address, s.cache.device
    ra, rd = s.rotary.address, s.rotary.device
    out, turned = torch.empty_like(s.q), s.q.transpose(2, 3)
    sub, q1 = s.q.as_subclass(_Sub), s.q[:, :, 0].contiguous()
    o1 = torch.empty_like(q1)
    before = s.tensors()
    for bad in ((sub, ra, rd, None, None, 0, out), (s.q, ra, rd + 1, None, None, 0, out), (s.q, 0, rd, None, None, 0, out), (s.q, ra, rd, None, None, 0, None),
                (s.q, ra, rd, None, None, 0, out[:, :5]), (turned, ra, rd, None, None, 0, turned), (s.q, ra, rd, s.positions[:, :4], None, 0, out),
                (s.q, ra, rd, s.positions.long(), None, 0, out), (s.q, ra, rd, None, s.lens[:2], 0, out), (s.q, ra, rd, None, None, True, out),
                (s.q.double(), ra, rd, None, None, 0, out), (s.q[0], ra, rd, None, None, 0, out)):
        assert c.rotary(*bad) == NOT_PLAIN
    ok = (a, d, s.k, s.v, s.lens, None, None, None, None, None, None, None)
    for at, bad in ((1, d + 1), (2, s.k[:2]), (2, s.k.float()), (2, s.k.half()), (3, s.v[:, :, :4]), (4, s.lens[:2]), (4, s.lens.long()), (4, None),
                    (5, s.counts[:2]), (6, s.positions[:, :4]), (7, s.rows[:2]), (8, 0), (8, "x"), (10, s.q), (11, s.q)):
        assert c.append(*ok[:at], bad, *ok[at + 1:]) == NOT_PLAIN
    assert c.append(*ok[:10], s.q[:, :, :3], s.q) == NOT_PLAIN
    for bad in ((a, d + 1, s.k, s.v, None, None), (a, d, s.k[:2], s.v[:2], None, None), (a, d, s.k, s.v.half(), None, None), (a, d, s.k, s.v, s.lens[:1], None),
                (a, d, s.k, s.v, None, s.counts.long()), (a, d, s.k.float(), s.v.float(), None, None)):
        assert c.read(*bad) == NOT_PLAIN
    for bad in ((a, d + 1, q1, s.lens, None, o1, s.ws), (a, d, q1[:2], s.lens, None, o1, s.ws), (a, d, q1, s.lens, 1, o1, s.ws), (a, d, q1, s.lens, None, o1[:2], s.ws),
                (a, d, q1, s.lens, None, o1, None), (a, d, q1, s.lens, None, None, s.ws), (a, d, q1.as_subclass(_Sub), s.lens, None, o1, s.ws),
                (a, d, q1, s.lens, None, o1, s.ws.view(torch.int32))):
        assert c.decode_kv(*bad) == NOT_PLAIN
    tree = torch.ones((1, 5), dtype=torch.int64, device="cuda")
    for bad in ((a, d, s.q[:2], s.lens, None, None, out, s.ws), (a, d, s.q, s.lens, tree.int(), None, out, s.ws), (a, d, s.q, s.lens, tree[:, :4], None, out, s.ws),
                (a, d, s.q, s.lens, tree.repeat(2, 1), None, out, s.ws), (a, d, s.q, s.lens, None, None, None, s.ws), (a, d, s.q, s.lens, None, None, out, None),
                (a, d, sub, s.lens, None, None, out, s.ws)):
        assert c.tree(*bad) == NOT_PLAIN
    assert _same(before, s.tensors())
    # refused by the library: its status
    assert c.decode_kv(a, d, q1, s.lens, None, o1, s.ws[:16]) == binding.ERR_WORKSPACE
    with pytest.raises(binding.ForgeError):
        binding.attn_decode_kv(q1, s.cache, s.lens, out=o1, workspace=s.ws[:16])
