"""The serving step around the KV cache, as cases that can be timed and compared: rotary positions, writing a cache of 8-bit
(or 16-bit) rows, reading rows back, one token per sequence over such a cache, and a tree of drafted tokens over it.

``run`` computes a case in plain torch operations (``own`` false) or through the public entry points of
``paper_2604_16498_b200.binding`` (``own`` true).  Head counts and sizes are those of the library's workloads: a
GPT-2-small-shaped model (12 heads of 64), a 1B-class one (32 query and 8 KV heads of 64), an 8B-class one (32 / 8 of 128) and
one with 7 query heads per KV head (28 / 4 of 128).  Activations are unit-variance normals.

The inputs of rotary and append are views of a fused QKV projection's output [B, S, (Hq + 2 Hkv) D].  Caches are
[B, Hkv, Smax, D]; 8-bit ones have an fp32 scale per row.  What a cache holds is returned as the values it stands for.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_LARGEST = {"int8": 127.0, "e4m3": 448.0}
_SMALLEST_ROW = 2.0 ** -100  # a row whose largest magnitude is below this counts as zeros
_WORKSPACE = 32 << 20        # what the serving program gives the attention for its partial results, cleared once


# ---------------------------------------------------------------------------------------------------------- cases
def _rotary(dtype, B, H, S, D, dims, layout, far, inverse=False):
    """dims: how many of a head's D elements are rotated; far: the largest first position of a sequence."""
    return dict(kind="rotary", dtype=dtype, B=B, H=H, S=S, D=D, dims=dims, layout=layout, far=far, inverse=inverse)


def _append(dtype, form, B, Hq, Hkv, S, Smax, D, dims, layout, ragged=False):
    """S new tokens for each sequence (ragged: 0 .. S of them), behind 0 .. Smax - S rows."""
    return dict(kind="append", dtype=dtype, form=form, B=B, Hq=Hq, Hkv=Hkv, S=S, Smax=Smax, D=D, dims=dims, layout=layout,
                ragged=ragged)


def _read(dtype, form, B, Hkv, rows, Smax, D, min_len):
    """The first min_len .. rows rows of every sequence."""
    return dict(kind="read", dtype=dtype, form=form, B=B, Hkv=Hkv, rows=rows, Smax=Smax, D=D, min_len=min_len)


def _decode(dtype, form, B, Hq, Hkv, Smax, D, min_len):
    return dict(kind="decode", dtype=dtype, form=form, B=B, Hq=Hq, Hkv=Hkv, Smax=Smax, D=D, min_len=min_len)


def _tree(dtype, form, B, Hq, Hkv, T, Smax, D, min_len, chain=False):
    """T drafted tokens (chain: one behind the other) whose rows lie behind the min_len .. Smax - T rows of the sequence."""
    return dict(kind="tree", dtype=dtype, form=form, B=B, Hq=Hq, Hkv=Hkv, T=T, Smax=Smax, D=D, min_len=min_len, chain=chain)


def listed():
    return [
        # One token for each of 16 conversations of an 8B-class model: query and key heads together (latency).
        dict(_rotary("bf16", 16, 40, 1, 128, 128, "half", 4096), name="rotary_step_b16"),
        # Three prompts of odd length far into long documents; interleaved pairs, three quarters of the head.
        dict(_rotary("f16", 3, 32, 1777, 128, 96, "interleaved", 131072), name="rotary_prompt_far"),
        # A token for each of 16 conversations: rotary positions, 8-bit rows, cache (latency).
        dict(_append("bf16", "int8", 16, 32, 8, 1, 4096, 128, 128, "half"), name="append_step_int8_b16"),
        # Prompts of an 8B-class model.
        dict(_append("bf16", "e4m3", 4, 32, 8, 2048, 4096, 128, 128, "half"), name="append_prompt_e4m3"),
        # A cached prefix of uneven lengths, read back for a chunk of its prompt.
        dict(_read("f16", "int8", 3, 4, 1801, 2400, 128, 1024), name="read_prefix_int8"),
        # All of a batch's cache.
        dict(_read("bf16", "e4m3", 16, 8, 4096, 4096, 128, 1024), name="read_batch_e4m3"),
        # Token generation for a batch of 16 conversations of an 8B-class model.
        dict(_decode("bf16", "int8", 16, 32, 8, 4096, 128, 1024), name="decode_int8_b16"),
        # Token generation at the end of one long document.
        dict(_decode("f16", "e4m3", 1, 32, 8, 32768, 128, 32768), name="decode_e4m3_b1_32768"),
        # Many short conversations of a GPT-2-small-shaped model.
        dict(_decode("bf16", "int8", 40, 12, 12, 1000, 64, 37), name="decode_int8_d64_b40"),
        # The smallest: 5 drafted tokens behind a short chat.
        dict(_tree("bf16", "bf16", 1, 32, 8, 5, 777, 128, 600), name="tree_t5_b1"),
        # 16 drafted tokens for each of 8 conversations, 7 query heads per KV head, 8-bit rows.
        dict(_tree("f16", "int8", 8, 28, 4, 16, 2417, 128, 600), name="tree_t16_int8_b8"),
        # The largest trees: 64 drafted tokens.
        dict(_tree("bf16", "bf16", 4, 32, 8, 64, 4160, 128, 1024), name="tree_t64_b4"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8), (32, 8), (28, 4), (12, 12)]


def _draw_rotary(rng):
    Hq, Hkv = rng.choice(_HEADS)
    D = rng.choice([64, 80, 96, 128, 128, 128, 256])
    dims = rng.choice([D, D, D // 2, D // 4 * 3, D - 2 * rng.randint(1, 20)])
    S = _log_int(rng, 1, 4096)
    B = max(1, min(_log_int(rng, 1, 64), 16384 // S))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while B * S * (Hq + Hkv) * D > (40 << 20) // (2 if dtype == "f32" else 1):
        B, S = max(1, B // 2), (S + 1) // 2
    return _rotary(dtype, B, Hq + Hkv, S, D, dims, rng.choice(["half", "interleaved"]),
                   _log_int(rng, 16, 1 << 20), rng.random() < 0.3)


def _draw_append(rng):
    Hq, Hkv = rng.choice(_HEADS)
    D = 64 if Hq == 12 else rng.choice([64, 80, 128, 128])
    S = rng.choice([1, _log_int(rng, 1, 2048)])
    B = max(1, min(_log_int(rng, 1, 64), 7000 // S))
    dtype = rng.choice(["bf16", "f16"])
    return _append(dtype, rng.choice(["int8", "e4m3", dtype]), B, Hq, Hkv, S, S + _log_int(rng, 1, 2048), D,
                   rng.choice([D, D, D // 2, D // 4 * 3]), rng.choice(["half", "interleaved"]), ragged=rng.random() < 0.4)


def _draw_read(rng):
    Hkv = rng.choice([4, 8, 12])
    D = rng.choice([64, 80, 128, 128])
    rows = _log_int(rng, 1, 8192)
    B = max(1, min(_log_int(rng, 1, 64), (13 << 15) // (rows * Hkv)))
    dtype = rng.choice(["bf16", "f16"])
    return _read(dtype, rng.choice(["int8", "e4m3"]), B, Hkv, rows, rows + rng.randint(0, 99), D, max(1, rows // 2))


def _draw_decode(rng):
    B = _log_int(rng, 1, 64)
    Hq, Hkv = rng.choice(_HEADS + [(16, 1)])
    D = 64 if Hq == 12 else rng.choice([64, 96, 128, 128])
    dtype = rng.choice(["bf16", "f16"])
    form = rng.choice(["int8", "e4m3", "int8", "e4m3", dtype])
    Smax = min(_log_int(rng, 64, 32768), (1 << (20 if form in _LARGEST else 19)) // (B * Hkv))
    return _decode(dtype, form, B, Hq, Hkv, Smax, D, max(1, Smax // 4))


def _draw_tree(rng):
    B = _log_int(rng, 1, 32)
    Hq, Hkv = rng.choice(_HEADS)
    D = 64 if Hq == 12 else rng.choice([64, 96, 128, 128])
    T = _log_int(rng, 2, 64)
    Smax = T + min(_log_int(rng, 64, 8192), (1 << 17) // (B * Hkv), (30 << 20) // (B * Hq * T))
    dtype = rng.choice(["bf16", "f16"])
    return _tree(dtype, rng.choice(["int8", "e4m3", dtype, dtype]), B, Hq, Hkv, T, Smax, D, (Smax - T) // 4,
                 chain=rng.random() < 0.2)


def draw(rng):
    kind = rng.choice([_draw_rotary, _draw_append, _draw_read, _draw_decode, _draw_decode, _draw_tree, _draw_tree])
    return kind(rng)


# ---------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _frequencies(dims):
    return (10000.0 ** (-torch.arange(0, dims, 2, dtype=torch.float64) / dims)).to(torch.float32).cuda()


def _ints(g, shape, lo, hi):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _codes(x, form):
    """8-bit rows of a normal tensor with their scales, as a cache holds them."""
    top = _LARGEST[form]
    m = x.abs().amax(-1, keepdim=True)
    y = x * (top / m)
    codes = y.round().to(torch.int8) if form == "int8" else y.to(torch.float8_e4m3fn)
    return codes, (m / top).squeeze(-1).contiguous()


def _cache(g, form, B, Hkv, Smax, D):
    """A cache full of rows, with the row norms' spread of a few in a thousand that unit normals of that length have."""
    out = {}
    for name in ("k", "v"):
        x = torch.randn((B, Hkv, Smax, D), generator=g, device="cuda")
        if form in _LARGEST:
            out[name], out[name + "_scale"] = _codes(x, form)
        else:
            out[name], out[name + "_scale"] = x.to(_TYPES[form]), None
    return out


def _empty_cache(form, B, Hkv, Smax, D):
    t = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}.get(form) or _TYPES[form]
    out = {}
    for name in ("k", "v"):
        out[name] = torch.zeros((B, Hkv, Smax, D), dtype=t, device="cuda")
        out[name + "_scale"] = torch.zeros((B, Hkv, Smax), device="cuda") if form in _LARGEST else None
    return out


def _trees(g, B, T, chain):
    """Which drafted tokens each one sees, as bits: itself, its parent (an earlier one), its parent's parent, and so on."""
    parents = torch.rand((B, T), generator=g, device="cuda").cpu().tolist()
    rows = []
    for b in range(B):
        bits = []
        for t in range(T):
            mask = 1 << t
            if t:
                mask |= bits[t - 1 if chain else int(parents[b][t] * t)]
            bits.append(mask)
        rows.append([m - (1 << 64) if m >= 1 << 63 else m for m in bits])
    return torch.tensor(rows, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    kind, B, D = case["kind"], case["B"], case["D"]
    t = _TYPES[case["dtype"]]
    if kind == "rotary":
        H, S = case["H"], case["S"]
        s["x"] = torch.randn((B, S, H, D), generator=g, device="cuda").to(t).permute(0, 2, 1, 3)
        s["out"] = torch.empty((B, S, H, D), dtype=t, device="cuda").permute(0, 2, 1, 3)
        s["positions"] = _ints(g, (B, 1), 0, case["far"]) + torch.arange(S, device="cuda", dtype=torch.int32)
        s["inv_freq"] = _frequencies(case["dims"])
    elif kind == "append":
        Hq, Hkv, S, Smax = case["Hq"], case["Hkv"], case["S"], case["Smax"]
        qkv = torch.randn((B, S, Hq + 2 * Hkv, D), generator=g, device="cuda").to(t)
        s["q"], s["new_k"], s["new_v"] = (x.permute(0, 2, 1, 3) for x in qkv.split([Hq, Hkv, Hkv], dim=2))
        s["q_out"] = torch.zeros((B, S, Hq, D), dtype=t, device="cuda").permute(0, 2, 1, 3)
        s["lens"] = _ints(g, (B,), 0, Smax - S)
        s["counts"] = _ints(g, (B,), 0, S) if case["ragged"] else None
        s["inv_freq"] = _frequencies(case["dims"])
        s["store"] = _empty_cache(case["form"], B, Hkv, Smax, D)
        s["k_out"], s["v_out"] = (torch.zeros((B, Hkv, S, D), dtype=t, device="cuda") for _ in range(2))
    elif kind == "read":
        s["store"] = _cache(g, case["form"], B, case["Hkv"], case["Smax"], D)
        s["lens"] = _ints(g, (B,), case["min_len"], case["rows"])
        s["k_out"], s["v_out"] = (torch.zeros((B, case["Hkv"], case["rows"], D), dtype=t, device="cuda") for _ in range(2))
    else:
        Hq, Smax, T = case["Hq"], case["Smax"], case.get("T", 1)
        s["store"] = _cache(g, case["form"], B, case["Hkv"], Smax, D)
        s["q"] = torch.randn((B, Hq, T, D) if kind == "tree" else (B, Hq, D), generator=g, device="cuda").to(t)
        s["out"] = torch.empty_like(s["q"])
        s["lens"] = _ints(g, (B,), case["min_len"], Smax - T if kind == "tree" else Smax)
        s["workspace"] = torch.zeros(_WORKSPACE, dtype=torch.uint8, device="cuda")
        if kind == "tree":
            s["tree"] = _trees(g, B, T, case["chain"])
    return s


# ---------------------------------------------------------------------------------------------------------- the plain form
def _turned(x, positions, inv_freq, layout, inverse=False):
    """x [B, H, S, D] in 32 bits, rotated by positions [B, S]; angles in 64 bits, since far ones lose their fraction in 32."""
    n = 2 * inv_freq.numel()
    angle = positions.double()[:, None, :, None] * inv_freq.double()
    cos, sin = angle.cos().float(), angle.sin().float()
    if inverse:
        sin = -sin
    y = x.clone()
    if layout == "half":
        a, b = x[..., : n // 2], x[..., n // 2: n]
        y[..., : n // 2], y[..., n // 2: n] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y[..., 0:n:2], y[..., 1:n:2] = a * cos - b * sin, b * cos + a * sin
    return y


def _kept(x, form):
    """What a cache of `form` keeps of the rows x (32 bits)."""
    if form not in _LARGEST:
        return x.to(_TYPES[form]).float()
    top = _LARGEST[form]
    m = x.abs().amax(-1, keepdim=True)
    y = torch.where(m >= _SMALLEST_ROW, x * (top / m), 0.0)
    y = y.round() if form == "int8" else y.to(torch.float8_e4m3fn).float()
    return y * torch.where(m >= _SMALLEST_ROW, m / top, 0.0)


def _values(store, name):
    x = store[name].float()
    return x if store[name + "_scale"] is None else x * store[name + "_scale"][..., None]


def _attend(q, store, visible):
    """q [B, Hq, T, D], visible [B, T, Smax] -> [B, Hq, T, D] in 32 bits."""
    B, Hq, T, D = q.shape
    k, v = _values(store, "k"), _values(store, "v")
    Hkv = k.shape[1]
    scores = (q.float() * D ** -0.5).reshape(B, Hkv, Hq // Hkv * T, D) @ k.transpose(2, 3)
    scores = scores.view(B, Hkv, Hq // Hkv, T, -1).masked_fill(~visible[:, None, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = (scores - torch.where(m == -math.inf, 0.0, m)).exp()
    o = (p.view(B, Hkv, Hq // Hkv * T, -1) @ v) / p.sum(-1).view(B, Hkv, -1, 1).clamp_min(1e-37)
    return o.view(B, Hq, T, D)


def _visible(lens, T, tree, Smax):
    j = torch.arange(Smax, device="cuda") - lens[:, None]          # [B, Smax], >= 0: a drafted token's row
    bit = (tree[:, :, None] >> j.clamp(0, T - 1)[:, None]) & 1      # [B, T, Smax]
    return (j < 0)[:, None] | ((j >= 0) & (j < T))[:, None] & (bit == 1)


def _plain(s):
    c = s["case"]
    kind, t = c["kind"], _TYPES[c["dtype"]]
    if kind == "rotary":
        return _turned(s["x"].float(), s["positions"], s["inv_freq"], c["layout"], c["inverse"]).to(t)
    if kind == "append":
        i = torch.arange(c["S"], device="cuda")
        new = i < (s["lens"].new_full((c["B"],), c["S"]) if s["counts"] is None else s["counts"])[:, None]
        new = new[:, None, :, None]
        positions = s["lens"][:, None] + i
        q, k = (_turned(s[x].float(), positions, s["inv_freq"], c["layout"]) for x in ("q", "new_k"))
        out = q, _kept(k, c["form"]), _kept(s["new_v"].float(), c["form"])
        return tuple(torch.where(new, x, 0.0).to(t) for x in out)
    if kind == "read":
        there = (torch.arange(c["rows"], device="cuda") < s["lens"][:, None])[:, None, :, None]
        return tuple(torch.where(there, _values(s["store"], x)[:, :, : c["rows"]], 0.0).to(t) for x in ("k", "v"))
    if kind == "decode":
        there = torch.arange(c["Smax"], device="cuda") < s["lens"][:, None]
        return _attend(s["q"][:, :, None], s["store"], there[:, None])[:, :, 0].to(t)
    return _attend(s["q"], s["store"], _visible(s["lens"], c["T"], s["tree"], c["Smax"])).to(t)


# ---------------------------------------------------------------------------------------------------------- the library's calls
def _handles(s, forge):
    """The cache's and the frequencies' handles, which a program makes once."""
    if "handles" not in s:
        h = s["handles"] = {}
        if "inv_freq" in s:
            h["rotary"] = forge.Rotary(s["inv_freq"], forge.ROTARY_HALF if s["case"]["layout"] == "half" else forge.ROTARY_INTERLEAVED)
        if "store" in s:
            h["cache"] = forge.KVCache(s["store"]["k"], s["store"]["v"], s["store"]["k_scale"], s["store"]["v_scale"])
    return s["handles"]


def _library(s):
    from paper_2604_16498_b200 import binding as forge
    c, h = s["case"], _handles(s, forge)
    kind = c["kind"]
    if kind == "rotary":
        return forge.rotary_apply(s["x"], h["rotary"], positions=s["positions"], inverse=c["inverse"], out=s["out"])
    if kind == "append":
        forge.kv_append(h["cache"], s["new_k"], s["new_v"], s["lens"], counts=s["counts"], rotary=h["rotary"], q=s["q"],
                        q_out=s["q_out"])
        forge.kv_read(h["cache"], s["k_out"], s["v_out"], first=s["lens"], counts=s["counts"])
        return s["q_out"], s["k_out"], s["v_out"]
    if kind == "read":
        forge.kv_read(h["cache"], s["k_out"], s["v_out"], counts=s["lens"])
        return s["k_out"], s["v_out"]
    if kind == "decode":
        return forge.attn_decode_kv(s["q"], h["cache"], s["lens"], out=s["out"], workspace=s["workspace"])
    return forge.attn_tree(s["q"], h["cache"], s["lens"], s["tree"], out=s["out"], workspace=s["workspace"])


def run(s):
    return _library(s) if own else _plain(s)


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_turn(x, positions, inv_freq, layout, inverse=False):
    n = inv_freq.numel()
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                    positions.double()[:, None, :, None] * inv_freq.double() * (-1.0 if inverse else 1.0))
    x = x.double()
    head, tail = x[..., : 2 * n], x[..., 2 * n:]
    pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if layout == "half" else head.unflatten(-1, (n, 2))
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
    return torch.cat([(y.transpose(-1, -2) if layout == "half" else y).flatten(-2), tail], -1)


def _exact_kept(x, form):
    if form not in _LARGEST:
        return x.to(_TYPES[form]).double()
    step = x.abs().max(-1, keepdim=True).values / _LARGEST[form]
    y = torch.nan_to_num(x / step)
    return step * (y.round() if form == "int8" else y.float().to(torch.float8_e4m3fn).double())


def _exact_values(store, name, b, rows):
    x = store[name][b, :, :rows].double()
    return x if store[name + "_scale"] is None else x * store[name + "_scale"][b, :, :rows, None].double()


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    if kind == "rotary":
        return _exact_turn(s["x"], s["positions"], s["inv_freq"], c["layout"], c["inverse"])
    if kind == "append":
        positions = s["lens"].long()[:, None] + torch.arange(c["S"], device="cuda")
        q, k = (_exact_turn(s[x], positions, s["inv_freq"], c["layout"]) for x in ("q", "new_k"))
        out = [q, _exact_kept(k, c["form"]), _exact_kept(s["new_v"].double(), c["form"])]
        if s["counts"] is not None:
            for b, n in enumerate(s["counts"].tolist()):
                for x in out:
                    x[b, :, n:] = 0
        return tuple(out)
    lens = s["lens"].tolist()
    if kind == "read":
        out = [torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        for b, n in enumerate(lens):
            for x, name in zip(out, ("k", "v")):
                x[b, :, :n] = _exact_values(s["store"], name, b, n)
        return tuple(out)
    T, Hkv, D = c.get("T", 1), c["Hkv"], c["D"]
    q = s["q"].double().view(c["B"], Hkv, -1, T, D)
    out = torch.zeros_like(q)
    for b, n in enumerate(lens):
        rows = n if kind == "decode" else n + T
        k, v = (_exact_values(s["store"], x, b, rows) for x in ("k", "v"))
        w = torch.einsum("hgtd,hjd->hgtj", q[b], k) / math.sqrt(D)
        if kind == "tree":
            sees = torch.tensor([[m >> u & 1 for u in range(T)] for m in s["tree"][b].tolist()], device="cuda").bool()
            w[..., n:] = torch.where(sees, w[..., n:], -math.inf)
        out[b] = torch.einsum("hgtj,hjd->hgtd", torch.softmax(w, -1), v)
    return out.view(s["q"].shape)


# ---------------------------------------------------------------------------------------------------------- work
def work(case):
    """Lengths and counts drawn from the seed count with their mean."""
    c, kind, B, D = case, case["kind"], case["B"], case["D"]
    es = 4 if c["dtype"] == "f32" else 2
    if kind == "rotary":
        n = B * c["H"] * c["S"]
        return {"bytes": 2 * es * n * D + 4 * B * c["S"] + 2 * c["dims"], "flops": 3 * n * c["dims"]}
    row = D + 4 if c["form"] in _LARGEST else 2 * D  # of a cache, for one token and KV head
    if kind == "append":
        n = B * c["S"] / (2 if c["ragged"] else 1)
        moved = 2 * c["Hq"] * es * D + 2 * c["Hkv"] * (2 * es * D + 2 * row)  # q in and out; K and V in, kept, and back
        return {"bytes": n * moved + 4 * B, "flops": 3 * n * c["dims"] * (c["Hq"] + c["Hkv"]) + 4 * n * D * c["Hkv"]}
    if kind == "read":
        n = 2 * c["Hkv"] * B * (c["min_len"] + c["rows"]) // 2
        return {"bytes": n * (row + es * D), "flops": n * D}
    T = c.get("T", 1)
    rows = B * ((c["min_len"] + c["Smax"] - T) // 2 + T) if kind == "tree" else B * (c["min_len"] + c["Smax"]) // 2
    return {"bytes": 2 * c["Hkv"] * row * rows + 2 * es * B * c["Hq"] * T * D + 4 * B + (8 * B * T if kind == "tree" else 0),
            "flops": 4 * D * c["Hq"] * T * rows}
