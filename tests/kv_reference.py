"""Rotary positions, KV caches of 8-bit rows and attention over them in 64 bits, from their definitions, with the error that the
kernels' roundings allow.  A rounding to a type t is off by at most half a step, HALF[t] relative to the value."""
import math

import torch

HALF = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}
F32 = 2.0 ** -24
TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def seeded(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def rotate(x, positions, inv_freq, layout="half", amplitude=1.0, inverse=False):
    """x [B,H,S,D] (any float type), positions [B,S] -> (rotated in fp64, bound of the fp32 arithmetic's error).
    cos and sin are off by a few 2^-24 (4 are allowed), each of the two products and the sum by one rounding, the products with the
    amplitude by one more: 8 roundings of |a| + |b| in all."""
    x = x.double()
    n = inv_freq.numel()
    angle = (positions.double()[:, None, :, None] * inv_freq.double()) * (-1 if inverse else 1)
    cos, sin = angle.cos() * amplitude, angle.sin() * amplitude
    y, err = x.clone(), torch.zeros_like(x)
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    err[..., first] = err[..., second] = (a.abs() + b.abs()) * 8 * F32 * abs(amplitude)
    return y, err


def decode_values(codes, scale):
    """The values that rows of codes stand for, in fp64 (16-bit rows: themselves)."""
    return codes.double() if scale is None else codes.double() * scale.double()[..., None]


def assert_rows_kept(codes, scale, exact, err, what=""):
    """Rows [..., D] in a cache against the exact values that were to be kept, known to `err`."""
    if scale is None:
        tol = HALF[codes.dtype] * exact.abs() * (1 + 2 ** -6) + err + 2.0 ** -25
        bad = (codes.double() - exact).abs() - tol
        assert bad.max() <= 0, f"{what}: {bad.max():.3e} over the bound"
        return
    top = TOP[codes.dtype]
    m, e = exact.abs().amax(-1), err.amax(-1)
    want = torch.where(m >= 2.0 ** -100, m / top, 0.0)
    off = (scale.double() - want).abs() - (e / top + 4 * F32 * want)
    assert off.max() <= 0, f"{what}: scale {off.max():.3e} over the bound"
    step = torch.where(scale > 0, scale.double(), 1.0)[..., None]
    y = torch.where(scale[..., None] > 0, exact / step, 0.0)
    # half a step of the code, and what x * (top / max) and the scale differ by in fp32: a few roundings of at most `top`
    half = 0.5 if codes.dtype == torch.int8 else torch.maximum(y.abs() * 2.0 ** -4, torch.full_like(y, 2.0 ** -10))
    bad = (codes.double() - y).abs() - (half * (1 + 2 ** -10) + err / step + y.abs() * 8 * F32)
    assert bad.max() <= 0, f"{what}: code {bad.max():.3e} over the bound"


def quantise(x, dtype):
    """Codes and scales of rows x (fp32) for a test's cache."""
    top = TOP[dtype]
    m = x.abs().amax(-1, keepdim=True)
    y = torch.where(m > 0, x * (top / m), 0.0)
    return (y.round() if dtype == torch.int8 else y).to(dtype), (m / top).squeeze(-1).contiguous()


def make_cache(g, B, Hkv, Smax, D, form, binding, spread=1.0):
    """A full cache of normal rows; spread > 1: rows of very different sizes."""
    parts = []
    for _ in range(2):
        x = torch.randn((B, Hkv, Smax, D), generator=g, device="cuda")
        if spread > 1:
            x *= spread ** (2 * torch.rand((B, Hkv, Smax, 1), generator=g, device="cuda") - 1)
        parts.append(quantise(x, form) if form in TOP else (x.to(form), None))
    (k, ks), (v, vs) = parts
    return binding.KVCache(k, v, ks, vs)


def attention(q, cache, past, sees=None, scale=None, rows_off=0.0, half_p=None):
    """q [B,Hq,T,D]; past: rows that every token sees; sees [B,T,T] bool: which of the T rows behind them (None: those rows do not
    exist).  -> (out in fp64, bound).  The bound: every probability is rounded to the operands' type (fp16 with 8-bit rows) and the
    output once; scores are sums of D products in fp32 (2^-22 of the sum of magnitudes per term is allowed, which covers truncating
    accumulation and the scaling), and a relative change d of the weights moves the output by at most 2 d sum w |v|.
    rows_off: what each element of K and V is off by in the operator under test, relative; half_p: how P is rounded there."""
    B, Hq, T, D = q.shape
    k, v = decode_values(cache.k, cache.k_scale), decode_values(cache.v, cache.v_scale)
    Smax, G = k.shape[2], Hq // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    past = past.clamp(0, Smax)
    j = torch.arange(Smax, device="cuda")
    visible = (j < past[:, None])[:, None].expand(B, T, Smax).clone()
    if sees is not None:
        for b in range(B):
            n = min(T, Smax - int(past[b]))
            if n > 0:
                visible[b, :, int(past[b]): int(past[b]) + n] = sees[b][:, :n]
    out, bound = torch.zeros((B, Hq, T, D), dtype=torch.float64, device="cuda"), torch.zeros((B, Hq, T, D), dtype=torch.float64, device="cuda")
    u_p = (HALF[q.dtype] if cache.k_scale is None else HALF[torch.float16]) if half_p is None else half_p
    for b in range(B):
        any_row = visible[b].any(0)  # rows that nobody sees may hold anything
        kb, vb = k[b][:, any_row], v[b][:, any_row]
        vis = visible[b][:, any_row]
        qb = q[b].double().view(-1, G, T, D)
        s = torch.einsum("hgtd,hjd->hgtj", qb, kb) * scale
        mag = torch.einsum("hgtd,hjd->hgtj", qb.abs(), kb.abs()) * abs(scale)
        s = s.masked_fill(~vis, -math.inf)
        if s.shape[-1] == 0:
            continue
        w = torch.nan_to_num(torch.softmax(s, -1))
        out[b] = torch.einsum("hgtj,hjd->hgtd", w, vb).view(Hq, T, D)
        wv = torch.einsum("hgtj,hjd->hgtd", w, vb.abs()).view(Hq, T, D)
        s_err = (mag.masked_fill(~vis, 0.0).amax(-1) * ((D + 8) * 2.0 ** -22 + rows_off)).view(Hq, T, 1) if mag.numel() else 0.0
        biggest = vb.abs().amax()  # what underflows of P in fp16 (2^-39 of the largest row) and fp32 sums can be worth
        bound[b] = (u_p + rows_off + 2 * s_err + 2.0 ** -17) * wv + HALF[q.dtype] * out[b].abs() * 1.01 + biggest * 2.0 ** -25 + 2.0 ** -25
    return out, bound


def assert_within(got, want, bound, what=""):
    g = got.double()
    assert torch.isfinite(g).all(), f"{what}: not finite"
    over = (g - want).abs() - bound
    assert over.max() <= 0, f"{what}: error {(g - want).abs().max():.3e}, {over.max():.3e} over the bound"


def tree_bits(sees):
    """bool [..., T, T] -> int64 [..., T]"""
    T = sees.shape[-1]
    out = torch.zeros(sees.shape[:-1], dtype=torch.int64, device=sees.device)
    for u in range(T):
        out |= torch.where(sees[..., u], (1 << u) - (1 << 64 if u == 63 else 0), 0)
    return out


def random_tree(g, B, T):
    """sees [B,T,T]: each token sees itself and its ancestors; parents are random earlier tokens."""
    sees = torch.zeros((B, T, T), dtype=torch.bool, device="cuda")
    parents = torch.rand((B, T), generator=g, device="cuda").cpu()
    for b in range(B):
        for t in range(T):
            if t:
                sees[b, t] = sees[b, int(parents[b, t] * t)]
            sees[b, t, t] = True
    return sees
