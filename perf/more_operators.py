"""A batch of many requests in one serving step, as cases that can be timed and compared: the step's page tables and slots, rows
into a KV cache kept in pages, attention over such a cache, and low-rank adapters of the requests beside a shared projection.

``run`` computes a case in plain torch operations (``own`` false) or through the public entry points of
``paper_2604_16498_b200.binding`` (``own`` true).  Head counts and sizes are those of the library's workloads: a
GPT-2-small-shaped model (768 wide, 12 heads of 64), a 1B-class one (2048, 32 query and 8 KV heads of 64), an 8B-class one (4096,
32 / 8 of 128, MLP 14336), one with 7 query heads per KV head (28 / 4 of 128) and one with a single KV head (16 / 1).

The step's tokens are packed, request after request: activations are [T, ...], and the heads of a token are views of a fused QKV
projection's output [T, (Hq + 2 Hkv) D].  A cache is [pages, Hkv, page size, D] with an fp32 scale per row in the 8-bit formats; the
pages of a request are anywhere in it, in the order that the request's row of the table says.  What a cache holds is returned as the
values it stands for.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_LARGEST = {"int8": 127.0, "e4m3": 448.0}
_SMALLEST_ROW = 2.0 ** -100  # a row whose largest magnitude is below this counts as zeros
_WORKSPACE = 32 << 20        # what the serving program gives the attention for its partial results, cleared once


# ---------------------------------------------------------------------------------------------------------- cases
def _assign(B, T, P, longest, prompts, scarce=False):
    """B requests with up to `longest` rows in the cache and T tokens in all: one each, or (prompts) some with many and some with
    none.  scarce: fewer free pages than the last of them need."""
    return dict(kind="assign", B=B, T=T, P=P, longest=longest, prompts=prompts, scarce=scarce)


def _append(dtype, form, B, S, Hq, Hkv, D, P, dims, layout, longest):
    """Up to S new tokens (S > 1: S / 2 at least) for each of B requests, behind 0 .. longest rows."""
    return dict(kind="append", dtype=dtype, form=form, B=B, S=S, Hq=Hq, Hkv=Hkv, D=D, P=P, dims=dims, layout=layout, longest=longest)


def _decode(dtype, form, B, Hq, Hkv, D, P, lo, hi):
    return dict(kind="decode", dtype=dtype, form=form, B=B, Hq=Hq, Hkv=Hkv, D=D, P=P, lo=lo, hi=hi)


def _tree(dtype, form, B, Hq, Hkv, D, P, lo, hi, T):
    """T drafted tokens whose rows lie behind the lo .. hi rows of the request; a token sees a path of earlier ones."""
    return dict(kind="tree", dtype=dtype, form=form, B=B, Hq=Hq, Hkv=Hkv, D=D, P=P, lo=lo, hi=hi, T=T)


def _adapters(dtype, T, R, n, rank, K, N):
    """T tokens of R requests, which use n adapters (every eighth request none)."""
    return dict(kind="adapters", dtype=dtype, T=T, R=R, n=n, rank=rank, K=K, N=N)


def listed():
    return [
        # A token for each of 64 conversations (latency).
        dict(_assign(64, 64, 16, 4096, False), name="assign_step_b64"),
        # Chunks of prompts between conversations, when pages run short.
        dict(_assign(300, 8192, 32, 3000, True, scarce=True), name="assign_mixed_t8192"),
        # A token for each of 64 conversations of an 8B-class model: rotary positions, 8-bit rows, pages (latency).
        dict(_append("bf16", "e4m3", 64, 1, 32, 8, 128, 16, 128, "half", 4096), name="append_step_e4m3_b64"),
        # Prompts of uneven lengths; interleaved pairs, three quarters of the head.
        dict(_append("f16", "int8", 5, 1500, 28, 4, 128, 64, 96, "interleaved", 700), name="append_prompts_int8"),
        # The smallest: one short chat of a 1B-class model.
        dict(_decode("bf16", "bf16", 1, 32, 8, 64, 16, 333, 333), name="decode_bf16_b1"),
        # Token generation for 16 conversations of an 8B-class model.
        dict(_decode("bf16", "bf16", 16, 32, 8, 128, 16, 1024, 4096), name="decode_bf16_b16"),
        # Many conversations of uneven lengths, 8-bit rows.
        dict(_decode("f16", "int8", 61, 28, 4, 128, 32, 100, 3000), name="decode_int8_b61"),
        # Token generation at the end of one long document; a single KV head.
        dict(_decode("bf16", "e4m3", 2, 16, 1, 128, 64, 60000, 65536), name="decode_e4m3_one_head"),
        # 16 drafted tokens for each of 8 conversations.
        dict(_tree("bf16", "bf16", 8, 32, 8, 128, 32, 600, 2400, 16), name="tree_t16_b8"),
        # A token for each of 48 requests, most with an adapter of its own (bound by reading the adapters).
        dict(_adapters("bf16", 48, 48, 40, 16, 4096, 4096), name="adapters_step_b48"),
        # A few requests of a GPT-2-small-shaped model (latency).
        dict(_adapters("f16", 13, 3, 2, 8, 768, 2304), name="adapters_small"),
        # Prompts beside the MLP's first projection.
        dict(_adapters("bf16", 4000, 9, 5, 64, 4096, 14336), name="adapters_prompts"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8, 128), (32, 8, 128), (28, 4, 128), (32, 8, 64), (12, 12, 64), (16, 1, 128), (8, 2, 96)]


def _draw_assign(rng):
    B = _log_int(rng, 1, 512)
    prompts = rng.random() < 0.6
    T = _log_int(rng, max(B, 16), 8192) if prompts else B + rng.choice([0, 0, rng.randint(0, 40)])
    return _assign(B, T, rng.choice([16, 32, 64, 128]), _log_int(rng, 1, 8192), prompts, rng.random() < 0.3)


def _draw_append(rng):
    Hq, Hkv, D = rng.choice(_HEADS)
    S = rng.choice([1, _log_int(rng, 2, 2000)])
    B = max(1, min(_log_int(rng, 1, 256), 7500 // S))
    dtype = rng.choice(["bf16", "f16"])
    return _append(dtype, rng.choice(["int8", "e4m3", dtype]), B, S, Hq, Hkv, D, rng.choice([16, 32, 64, 256]),
                   rng.choice([D, D, D // 2, D // 4 * 3]), rng.choice(["half", "interleaved"]), _log_int(rng, 1, 4096))


def _draw_decode(rng):
    Hq, Hkv, D = rng.choice(_HEADS)
    B = _log_int(rng, 1, 128)
    dtype = rng.choice(["bf16", "f16"])
    form = rng.choice(["int8", "e4m3", dtype, dtype])
    hi = min(_log_int(rng, 16, 65536), (1 << (20 if form in _LARGEST else 19)) // (B * Hkv))
    return _decode(dtype, form, B, Hq, Hkv, D, rng.choice([16, 16, 32, 64, 128]), rng.choice([0, hi // 4, hi // 2, hi]), hi)


def _draw_tree(rng):
    Hq, Hkv, D = rng.choice(_HEADS)
    B, T = _log_int(rng, 1, 24), _log_int(rng, 2, 64)
    hi = min(_log_int(rng, 16, 8192), (1 << 17) // (B * Hkv), (30 << 20) // (B * Hq * T))
    dtype = rng.choice(["bf16", "f16"])
    return _tree(dtype, rng.choice(["int8", "e4m3", dtype, dtype]), B, Hq, Hkv, D, rng.choice([16, 32, 64, 128]), hi // 4, hi, T)


def _draw_adapters(rng):
    K, N = rng.choice([(768, 2304), (2048, 2048), (2048, 8192), (4096, 4096), (4096, 6144), (14336, 4096), (1000, 520)])
    T = min(_log_int(rng, 1, 4096), (1 << 26) // max(K, N))
    R = rng.choice([T, _log_int(rng, 1, T)])
    return _adapters(rng.choice(["bf16", "f16"]), T, R, min(R, _log_int(rng, 1, 40)), rng.choice([8, 16, 16, 32, 64, 128]), K, N)


def draw(rng):
    return rng.choice([_draw_assign, _draw_append, _draw_decode, _draw_decode, _draw_tree, _draw_adapters, _draw_adapters])(rng)


# ---------------------------------------------------------------------------------------------------------- inputs
def _ints(g, shape, lo, hi):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _cut(g, total, parts):
    """Where `parts` pieces of 0 .. total, one at least each, end."""
    inner = torch.randperm(total - 1, generator=g, device="cuda")[: parts - 1] + 1 if parts > 1 else torch.empty(0, device="cuda")
    return torch.cat([inner.sort().values.int(), torch.full((1,), total, dtype=torch.int32, device="cuda")])


def _scattered(g, lens, P, columns, spare=0):
    """A table [B, columns] of pages anywhere in the cache for `lens` rows each, -1 behind them, and the pages that are left: enough
    for what the rows may become (all columns) and `spare` more."""
    B = lens.numel()
    total = B * columns + spare
    order = torch.randperm(total, generator=g, device="cuda").int()
    used = torch.arange(columns, device="cuda") < ((lens + P - 1) // P)[:, None]
    table = torch.where(used, order[: B * columns].view(B, columns), -1).contiguous()
    left = torch.cat([torch.where(used, -1, order[: B * columns].view(B, columns)).flatten(), order[B * columns:]])
    rank = torch.argsort((left < 0).int(), stable=True)  # those that are free come first
    return table, left[rank].contiguous(), (left >= 0).sum().int().view(1), total


def _codes(x, form):
    """8-bit rows of a normal tensor with their scales, as a cache holds them."""
    top = _LARGEST[form]
    m = x.abs().amax(-1, keepdim=True)
    y = x * (top / m)
    codes = y.round().to(torch.int8) if form == "int8" else y.to(torch.float8_e4m3fn)
    return codes, (m / top).squeeze(-1).contiguous()


def _pages(g, form, pages, Hkv, P, D, empty=False):
    t = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}.get(form) or _TYPES[form]
    out = {}
    for name in ("k", "v"):
        if empty:
            out[name] = torch.zeros((pages, Hkv, P, D), dtype=t, device="cuda")
            out[name + "_scale"] = torch.zeros((pages, Hkv, P), device="cuda") if form in _LARGEST else None
            continue
        x = torch.randn((pages, Hkv, P, D), generator=g, device="cuda")
        out[name], out[name + "_scale"] = _codes(x, form) if form in _LARGEST else (x.to(t), None)
    return out


def _paths(g, B, T):
    """Which drafted tokens each one sees, as bits: itself, its parent (an earlier one), its parent's parent, and so on."""
    parents = torch.rand((B, T), generator=g, device="cuda").cpu().tolist()
    rows = []
    for b in range(B):
        bits = []
        for t in range(T):
            bits.append(1 << t | (bits[int(parents[b][t] * t)] if t else 0))
        rows.append([m - (1 << 64) if m >= 1 << 63 else m for m in bits])
    return torch.tensor(rows, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind == "adapters":
        T, R, n, r, K, N = (case[x] for x in ("T", "R", "n", "rank", "K", "N"))
        t = _TYPES[case["dtype"]]
        s["x"], s["y"] = (torch.randn((T, w), generator=g, device="cuda").to(t) for w in (K, N))
        s["a"] = (torch.randn((n, r, K), generator=g, device="cuda") * K ** -0.5).to(t)
        s["b"] = (torch.randn((n, N, r), generator=g, device="cuda") * r ** -0.5).to(t)
        s["scales"] = torch.rand(n, generator=g, device="cuda") + 0.5
        s["requests"] = torch.searchsorted(_cut(g, T, R), torch.arange(T, dtype=torch.int32, device="cuda"), right=True).int()
        i = torch.arange(R, device="cuda")
        s["adapters"] = torch.where(i % 8 == 7, -1, torch.randperm(n, generator=g, device="cuda")[i % n]).int()
        s["out"] = torch.empty_like(s["y"])
        return s
    B, P = case["B"], case["P"]
    if kind == "assign":
        T = case["T"]
        s["counts"] = None
        if case["prompts"]:
            share = torch.rand(B, generator=g, device="cuda", dtype=torch.float64) ** 4
            share = share * (torch.rand(B, generator=g, device="cuda") > 0.1)
            s["counts"] = (share / share.sum().clamp_min(1e-9) * T).int()
        s["lens"] = _ints(g, (B,), 0, case["longest"])
        columns = (case["longest"] + T + P - 1) // P if not case["prompts"] else (case["longest"] + T // 2) // P + 2
        s["table"], s["free"], s["free_count"], _ = _scattered(g, s["lens"], P, columns)
        if case["scarce"]:
            counts = torch.ones_like(s["lens"]) if s["counts"] is None else s["counts"]
            need = ((s["lens"] + counts + P - 1) // P - (s["lens"] + P - 1) // P).sum()
            s["free_count"] = torch.minimum(s["free_count"], (need * 9 // 10).int().view(1))
        for name, n in (("new_lens", B), ("starts", B + 1), ("slots", T), ("positions", T), ("requests", T), ("free_left", 1)):
            s[name] = torch.zeros(n, dtype=torch.int32, device="cuda")
        return s
    t, D, Hq, Hkv = _TYPES[case["dtype"]], case["D"], case["Hq"], case["Hkv"]
    if kind == "append":
        S = case["S"]
        s["lens"] = _ints(g, (B,), 0, case["longest"])
        even = torch.linspace((S + 1) // 2, S, B, dtype=torch.float64, device="cuda").round().int()
        s["counts"] = even[torch.randperm(B, generator=g, device="cuda")]
        s["table"], _, _, pages = _scattered(g, s["lens"] + s["counts"], P, (case["longest"] + S + P - 1) // P)
        ends = s["counts"].cumsum(0).int()
        T = int(ends[-1])
        request = torch.searchsorted(ends, torch.arange(T, dtype=torch.int32, device="cuda"), right=True)
        s["positions"] = (s["lens"][request] + torch.arange(T, device="cuda") - (ends - s["counts"])[request]).int()
        s["slots"] = s["table"][request, (s["positions"] // P).long()] * P + s["positions"] % P
        s["starts"] = torch.cat([ends.new_zeros(1), ends])
        qkv = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda").to(t)
        s["q"], s["new_k"], s["new_v"] = qkv.split([Hq, Hkv, Hkv], dim=1)
        s["q_out"] = torch.zeros((T, Hq, D), dtype=t, device="cuda")
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, case["dims"], 2, dtype=torch.float64) / case["dims"])).float().cuda()
        s["store"] = _pages(g, case["form"], pages, Hkv, P, D, empty=True)
        s["k_out"], s["v_out"] = (torch.zeros((B, Hkv, S, D), dtype=t, device="cuda") for _ in range(2))
        return s
    T = case.get("T", 0)
    s["lens"] = _ints(g, (B,), case["lo"], case["hi"])
    s["table"], _, _, pages = _scattered(g, s["lens"] + T, P, max(1, (case["hi"] + T + P - 1) // P))
    s["store"] = _pages(g, case["form"], pages, Hkv, P, D)
    s["q"] = torch.randn((B, Hq, T, D) if T else (B, Hq, D), generator=g, device="cuda").to(t)
    s["out"] = torch.empty_like(s["q"])
    s["workspace"] = torch.zeros(_WORKSPACE, dtype=torch.uint8, device="cuda")
    if T:
        s["tree"] = _paths(g, B, T)
    return s


# ---------------------------------------------------------------------------------------------------------- the plain form
def _plain_assign(s):
    c, lens, table, free = s["case"], s["lens"].long(), s["table"], s["free"]
    P, T, (B, columns) = c["P"], c["T"], table.shape
    counts = torch.ones_like(lens) if s["counts"] is None else s["counts"].long()
    have, need = (lens + P - 1) // P, (lens + counts + P - 1) // P
    ends = counts.cumsum(0)
    fits = (need <= columns) & (ends <= T)
    new = torch.where(fits, need - have, 0)
    incl = new.cumsum(0)
    room = s["free_count"].long()
    fits = fits & ((new == 0) | (incl <= room))
    new = torch.where(fits, new, 0)
    first = incl - new  # of the pages that are handed out (where any are)
    # pages: number i of the request with first <= i < first + new
    i = torch.arange(T // P + B + 1, device="cuda")
    last = new.cumsum(0)
    b = torch.searchsorted(last, i, right=True).clamp_max(B - 1)
    page = free[(room - 1 - i).clamp_min(0)]
    at = torch.where(i < last[-1], b * columns + have[b] + i - first[b], B * columns)
    out = torch.cat([table.flatten(), table.new_zeros(1)])
    out[at] = page
    out = out[:-1].view(B, columns)
    # tokens
    t = torch.arange(T, device="cuda")
    there = t < ends[-1]
    b = torch.searchsorted(ends, t, right=True).clamp_max(B - 1)
    pos = lens[b] + t - (ends - counts)[b]
    page = out[b, (pos // P).clamp_max(columns - 1)].long()
    slots = torch.where(there & fits[b], page * P + pos % P, -1)
    starts = torch.cat([ends.new_zeros(1), ends]).clamp_max(T)
    ints = (lens + torch.where(fits, counts, 0), starts, slots, torch.where(there, pos, 0), torch.where(there, b, -1), room - last[-1:])
    return (*(x.int() for x in ints), out)


def _turned(x, positions, inv_freq, layout):
    """x [T, H, D] in 32 bits, rotated by positions [T]; angles in 64 bits."""
    n = 2 * inv_freq.numel()
    angle = positions.double()[:, None, None] * inv_freq.double()
    cos, sin = angle.cos().float(), angle.sin().float()
    y = x.clone()
    a, b = (x[..., : n // 2], x[..., n // 2: n]) if layout == "half" else (x[..., 0:n:2], x[..., 1:n:2])
    u, v = a * cos - b * sin, b * cos + a * sin
    if layout == "half":
        y[..., : n // 2], y[..., n // 2: n] = u, v
    else:
        y[..., 0:n:2], y[..., 1:n:2] = u, v
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


def _plain_append(s):
    c = s["case"]
    t = _TYPES[c["dtype"]]
    q, k = (_turned(s[x].float(), s["positions"], s["inv_freq"], c["layout"]) for x in ("q", "new_k"))
    out = [q.to(t)]
    for x, name in ((k, "k_out"), (s["new_v"].float(), "v_out")):
        x = _kept(x, c["form"]).to(t)
        i = torch.arange(c["S"], device="cuda")
        rows = x[(s["starts"][:-1, None] + i).clamp_max(x.shape[0] - 1).long()].transpose(1, 2)  # [B, Hkv, S, D]
        out.append(torch.where((i < s["counts"][:, None])[:, None, :, None], rows, s[name]))
    return tuple(out)


def _plain_attend(s):
    c, lens = s["case"], s["lens"]
    T, P, (B, columns) = c.get("T", 0), c["P"], s["table"].shape
    q = s["q"].float() if T else s["q"].float()[:, :, None]
    Hkv, D, rows = c["Hkv"], c["D"], columns * P

    def values(name):
        page = s["table"].clamp_min(0).long()
        x = s["store"][name][page].float()                     # [B, columns, Hkv, P, D]
        if s["store"][name + "_scale"] is not None:
            x = x * s["store"][name + "_scale"][page][..., None]
        return x.transpose(1, 2).reshape(B, Hkv, rows, D)

    j = torch.arange(rows, device="cuda") - lens[:, None]       # >= 0: a drafted token's row
    seen = (j < 0)[:, None].expand(B, max(T, 1), rows)
    if T:
        bit = (s["tree"][:, :, None] >> j.clamp(0, T - 1)[:, None]) & 1
        seen = seen | ((j >= 0) & (j < T))[:, None] & (bit == 1)
    scores = (q * D ** -0.5).reshape(B, Hkv, -1, D) @ values("k").transpose(2, 3)
    scores = scores.view(B, Hkv, -1, max(T, 1), rows).masked_fill(~seen[:, None, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = (scores - torch.where(m == -math.inf, 0.0, m)).exp()
    o = (p.view(B, Hkv, -1, rows) @ values("v")) / p.sum(-1).view(B, Hkv, -1, 1).clamp_min(1e-37)
    return o.reshape(s["q"].shape).to(s["q"].dtype)


def _plain_adapters(s):
    """Products with all adapters, of which each token keeps its own one's part."""
    n, r, K = s["a"].shape
    own_one = s["adapters"][s["requests"].long()]
    u = s["x"].float() @ s["a"].float().view(n * r, K).T
    mine = torch.arange(n, device="cuda") == own_one[:, None]
    u = u.view(-1, n, r) * (mine * s["scales"])[..., None]
    y = u.view(-1, n * r) @ s["b"].float().transpose(1, 2).reshape(n * r, -1)
    return (s["y"].float() + y).to(s["y"].dtype)


def _plain(s):
    kind = s["case"]["kind"]
    return {"assign": _plain_assign, "append": _plain_append, "adapters": _plain_adapters}.get(kind, _plain_attend)(s)


# ---------------------------------------------------------------------------------------------------------- the library's calls
def _handles(s, forge):
    """The handles that a program makes once: of the cache, the frequencies, the tables and a step's slots."""
    if "handles" not in s:
        h = s["handles"] = {}
        if "inv_freq" in s:
            h["rotary"] = forge.Rotary(s["inv_freq"], forge.ROTARY_HALF if s["case"]["layout"] == "half" else forge.ROTARY_INTERLEAVED)
        if "store" in s:
            h["cache"] = forge.KVPages(s["store"]["k"], s["store"]["v"], s["store"]["k_scale"], s["store"]["v_scale"])
        if "free" in s:
            h["tables"] = forge.PageTables(s["table"], s["free"], s["free_count"], s["case"]["P"])
            h["step"] = forge.PageSlots(*(s[x] for x in ("new_lens", "starts", "slots", "positions", "requests")))
    return s["handles"]


def _library(s):
    from paper_2604_16498_b200 import binding as forge
    kind, h = s["case"]["kind"], _handles(s, forge)
    if kind == "assign":
        forge.assign_pages(h["tables"], s["lens"], h["step"], counts=s["counts"], free_left=s["free_left"])
        return tuple(s[x] for x in ("new_lens", "starts", "slots", "positions", "requests", "free_left", "table"))
    if kind == "append":
        forge.kv_append_pages(h["cache"], s["new_k"], s["new_v"], s["slots"], positions=s["positions"], rotary=h["rotary"], q=s["q"],
                              q_out=s["q_out"])
        forge.kv_read_pages(h["cache"], s["table"], s["k_out"], s["v_out"], first=s["lens"], counts=s["counts"])
        return s["q_out"], s["k_out"], s["v_out"]
    if kind == "decode":
        return forge.attn_decode_pages(s["q"], h["cache"], s["table"], s["lens"], out=s["out"], workspace=s["workspace"])
    if kind == "tree":
        return forge.attn_tree_pages(s["q"], h["cache"], s["table"], s["lens"], s["tree"], out=s["out"], workspace=s["workspace"])
    return forge.linear_adapters(s["x"], s["y"], s["a"], s["b"], s["adapters"], requests=s["requests"], scales=s["scales"], out=s["out"])


def run(s):
    return _library(s) if own else _plain(s)


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_assign(s):
    c, free, room = s["case"], s["free"].tolist(), s["free_count"].item()
    P, T, table = c["P"], c["T"], s["table"].tolist()
    lens = s["lens"].tolist()
    counts = [1] * len(lens) if s["counts"] is None else s["counts"].tolist()
    slots, positions, requests, new_lens, starts = [], [], [], [], [0]
    total, short = 0, False
    for b, (n, more) in enumerate(zip(lens, counts)):
        total += more
        starts.append(min(total, T))
        want = -(-(n + more) // P) - -(-n // P)
        ok = -(-(n + more) // P) <= len(table[b]) and total <= T
        if ok and want:
            short = short or want > room
            ok = not short
        if ok:
            for i in range(want):
                room -= 1
                table[b][-(-n // P) + i] = free[room]
        new_lens.append(n + more if ok else n)
        for p in range(n, n + more):
            slots.append(table[b][p // P] * P + p % P if ok else -1)
            positions.append(p)
            requests.append(b)
    pad = T - len(slots)
    slots, positions, requests = (slots + [-1] * pad)[:T], (positions + [0] * pad)[:T], (requests + [-1] * pad)[:T]
    return tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (new_lens, starts, slots, positions, requests, [room], table))


def _exact_append(s):
    c = s["case"]
    n = c["dims"] // 2

    def turn(x):
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None, None] * s["inv_freq"].double())
        x = x.double()
        head, tail = x[..., : 2 * n], x[..., 2 * n:]
        pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if c["layout"] == "half" else head.unflatten(-1, (n, 2))
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
        return torch.cat([(y.transpose(-1, -2) if c["layout"] == "half" else y).flatten(-2), tail], -1)

    def keep(x):
        if c["form"] not in _LARGEST:
            return x.to(_TYPES[c["form"]]).double()
        step = x.abs().max(-1, keepdim=True).values / _LARGEST[c["form"]]
        y = torch.nan_to_num(x / step)
        return step * (y.round() if c["form"] == "int8" else y.float().to(torch.float8_e4m3fn).double())

    out = [turn(s["q"])]
    starts = s["starts"].tolist()
    for x in (keep(turn(s["new_k"])), keep(s["new_v"].double())):
        y = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
        for b in range(c["B"]):
            y[b, :, : starts[b + 1] - starts[b]] = x[starts[b]: starts[b + 1]].transpose(0, 1)
        out.append(y)
    return tuple(out)


def _exact_attend(s):
    c = s["case"]
    T, P, Hkv, D = c.get("T", 0), c["P"], c["Hkv"], c["D"]
    q = s["q"].double().view(c["B"], Hkv, -1, max(T, 1), D)
    out = torch.zeros_like(q)
    for b, n in enumerate(s["lens"].tolist()):
        rows = n + T
        if rows == 0:
            continue
        page = s["table"][b, : -(-rows // P)].long()
        k, v = (s["store"][x][page].double() * (1.0 if s["store"][x + "_scale"] is None else s["store"][x + "_scale"][page].double()[..., None])
                for x in ("k", "v"))
        k, v = (x.transpose(0, 1).reshape(Hkv, -1, D)[:, :rows] for x in (k, v))
        w = torch.einsum("hgtd,hjd->hgtj", q[b], k) / math.sqrt(D)
        if T:
            sees = torch.tensor([[m >> u & 1 for u in range(T)] for m in s["tree"][b].tolist()], device="cuda").bool()
            w[..., n:] = torch.where(sees, w[..., n:], -math.inf)
        out[b] = torch.einsum("hgtj,hjd->hgtd", torch.softmax(w, -1), v)
    return out.view(s["q"].shape)


def _exact_adapters(s):
    out = s["y"].double()
    which = s["adapters"][s["requests"].long()]
    for i in range(s["a"].shape[0]):
        at = (which == i).nonzero().flatten()
        if at.numel():
            out[at] += s["scales"][i].double() * torch.einsum("tr,nr->tn", torch.einsum("tk,rk->tr", s["x"][at].double(), s["a"][i].double()),
                                                              s["b"][i].double())
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    return {"assign": _exact_assign, "append": _exact_append, "adapters": _exact_adapters}.get(kind, _exact_attend)(s)


# ---------------------------------------------------------------------------------------------------------- work
def work(case):
    """Lengths and counts drawn from the seed count with their mean."""
    c, kind = case, case["kind"]
    if kind == "assign":
        return {"bytes": 4 * (3 * c["B"] + 3 * c["T"] + 2 * (c["T"] // c["P"] + 1)), "flops": 8 * c["T"]}
    if kind == "adapters":
        used = len({i % c["n"] for i in range(c["R"]) if i % 8 != 7})
        tokens = c["T"] * (1 - c["R"] // 8 / c["R"])  # with an adapter
        wide = c["K"] + c["N"]
        return {"bytes": 2 * (tokens * c["K"] + 2 * c["T"] * c["N"] + used * c["rank"] * wide), "flops": 2 * tokens * c["rank"] * wide}
    B, D, Hq, Hkv = c["B"], c["D"], c["Hq"], c["Hkv"]
    row = D + 4 if c["form"] in _LARGEST else 2 * D  # of a cache, for one token and KV head
    if kind == "append":
        n = B * ((c["S"] + 1) // 2 + c["S"]) / 2
        moved = 4 * Hq * D + 2 * Hkv * (4 * D + 2 * row) + 8  # q in and out; K and V in, kept, and back
        return {"bytes": n * moved, "flops": 3 * n * c["dims"] * (Hq + Hkv) + 4 * n * D * Hkv}
    T = c.get("T", 0)
    rows = B * ((c["lo"] + c["hi"]) // 2 + T)
    return {"bytes": 2 * Hkv * row * rows + 4 * B * Hq * max(T, 1) * D + 4 * rows // c["P"] + 8 * B * T, "flops": 4 * D * Hq * max(T, 1) * rows}
