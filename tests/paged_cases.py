"""Plain implementations of the paged cache's operators in 64 bits, and inputs for their tests."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2410_23668_amd.device import PagedKvCache

BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


def e4m3_rows(x: torch.Tensor):
    """(codes as uint8, scale bytes) of rows [..., d], from the definition in 64 bits."""
    x = x.double().cpu().numpy()
    a = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    with np.errstate(all="ignore"):
        frac, e = np.frexp(np.where(bad, 1.0, a))   # a = frac 2^e, frac in [0.5, 1)
        k = np.where(a == 0, -126, np.maximum(e - 9 + (frac > 0.875), -126))
        y = np.ldexp(np.where(bad[..., None], 0.0, x), -k[..., None])
        # nearest multiple of the spacing, halves to even
        _, ey = np.frexp(np.where(y == 0, 1e-30, np.abs(y)))
        step = np.ldexp(1.0, np.maximum(ey - 1, -6) - 3)
        y = np.rint(y / step) * step
    codes = torch.from_numpy(y).to(torch.float32).to(E4M3)   # (exact: y is a code's value)
    assert torch.equal(codes.double(), torch.from_numpy(y))
    codes = codes.view(torch.uint8).clone()
    # (the sign of a zero is the value's own)
    zero = torch.from_numpy((y == 0) & np.signbit(x))
    codes[zero] = 0x80
    codes[torch.from_numpy(bad)] = 0x7F
    return codes, torch.from_numpy(np.where(bad, 127, k + 127).astype(np.uint8))


def values(pool: PagedKvCache, name: str) -> torch.Tensor:
    """Every row of the pool in 64 bits (CPU)."""
    x = getattr(pool, name).cpu()
    if x.dtype == BF16:
        return x.double()
    s = getattr(pool, name + "_scale").cpu().double()
    return x.float().double() * torch.exp2(s - 127)[..., None]


def make_pool(layers, n_pages, kv, page, d, dtype, gen, sigma=1.0) -> PagedKvCache:
    cfg = dict(n_layers=layers, n_kv_heads=kv, head_dim=d)
    pool = PagedKvCache(cfg, n_pages, page, dtype)
    for name in ("k", "v"):
        x = torch.randn((layers, n_pages, kv, page, d), generator=gen) * sigma
        if dtype == BF16:
            getattr(pool, name).copy_(x.to(BF16))
        else:
            codes, scale = e4m3_rows(x)
            getattr(pool, name).view(torch.uint8).copy_(codes)
            getattr(pool, name + "_scale").copy_(scale)
    return pool


def make_table(lengths, page, n_pages, gen, extra=2, fill=-1) -> torch.Tensor:
    """Pages in random order; entries past a sequence's own hold 'fill'."""
    need = [-(-n // page) for n in lengths]
    t = torch.full((len(lengths), max(max(need), 1) + extra), fill, dtype=torch.int32)
    order = torch.randperm(n_pages, generator=gen).to(torch.int32)
    at = 0
    assert sum(need) <= n_pages
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    return t


def attention64(K, V, table, lengths, q, page, scale, window=0, layer=0):
    """(out, lse, tolerance) in 64 bits from pools of values (CPU).

    The tolerance of an output in 32 bits (a bound on rounding, not a fit): a
    product q.k of d terms and its scaling are off by about sqrt(d) half-steps
    of the sum of magnitudes X, a weight by as much again in its exponent, sums
    of n terms by sqrt(n) half-steps of the sum of magnitudes; eight times that
    for the spread, and 32 steps for the joins, the exponential and the
    division: 2^-24 (32 + 8 sqrt(n) + 8 X) times sum p |v| / sum p."""
    B, nq, d = q.shape
    kv = K.shape[2]
    out = torch.zeros(B, nq, d, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((B, nq), -math.inf, dtype=torch.float64)
    ltol = torch.zeros_like(lse)
    for b, n in enumerate(lengths):
        lo = max(0, n - window) if window else 0
        if n <= lo:
            continue
        j = torch.arange(lo, n)
        pg = table[b].long()[j // page]
        for h in range(nq):
            g = h // (nq // kv)
            k, v = K[layer, pg, g, j % page], V[layer, pg, g, j % page]
            x = (k @ q[b, h].double()) * scale
            X = float(((k.abs() @ q[b, h].double().abs()) * abs(scale)).max())
            p = torch.softmax(x, 0)
            out[b, h] = p @ v
            lse[b, h] = torch.logsumexp(x, 0)
            T = 2.0 ** -24 * (32 + 8 * math.sqrt(n - lo) + 8 * X)
            tol[b, h] = T * (p @ v.abs())
            ltol[b, h] = T + 2.0 ** -23 * abs(float(lse[b, h]))
    return out, lse, tol, ltol


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def check_attention(out, lse, want, what=""):
    """out within its tolerance plus half a step of its own type (fp16 values
    below its normal range: half its smallest step)."""
    o, l, tol, ltol = want
    got = out.double().cpu()
    tiny = {FP16: 2.0 ** -25}.get(out.dtype, 0.0)
    lim = tol + half_step(out.dtype) * (o.abs() + tol) + tiny
    off = (got - o).abs()
    assert torch.isfinite(got).all(), f"{what}: non-finite output"
    worst = float((off / lim.clamp(min=1e-300)).max())
    assert bool((off <= lim).all()), f"{what}: {worst:.2f} of the tolerance"
    if lse is not None:
        g = lse.double().cpu()
        same = (g == l) | ((g - l).abs() <= ltol)
        assert bool(same.all()), f"{what}: lse off by {float((g - l).abs().max()):.2e}"
    return worst
