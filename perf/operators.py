"""The operators of a paged KV cache, as cases that can be timed and compared.

A cache of pages holds the keys and values of sequences of any length: a pool
[pages][kv heads][page size][head dim] for keys and one for values, and a table
[sequence][n] of each sequence's pages in order.  Three operators work on it:

  append     rows of new keys and values (a decode step's, or a prompt's) are
             written to their positions' slots; an 8-bit cache is quantised as
             it is written, with one power of two per row and head;
  read       rows are read back, as values;
  attention  one new query token per sequence attends over its cached positions.

Each case is one call.  Head counts and dimensions are those of
``synth.workloads``, or generic.  Pages are dealt in random order, as a pool
that has been in use hands them out.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32,
          "e4m3": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}


def _attn(batch, context, heads, kv_heads, head_dim, cache, io, page=64, ragged=False, empty=0,
          window=0, **named) -> dict:
    """batch sequences (the last ``empty`` of them of no length: a padded batch)."""
    return dict(op="attention", batch=batch, context=context, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, cache=cache, io=io, page=page, ragged=ragged, empty=empty,
                window=window, **named)


def _rows(op, batch, context, kv_heads, head_dim, cache, io, page=64, rows=0, ragged=False,
          empty=0, **named) -> dict:
    """Each sequence's last ``rows`` positions (0: all of them); ``empty`` more rows are padding."""
    return dict(op=op, batch=batch, context=context, kv_heads=kv_heads, head_dim=head_dim,
                cache=cache, io=io, page=page, rows=rows, ragged=ragged, empty=empty, **named)


def listed() -> list:
    return [
        # one step of one user: a row per layer, where latency is all there is
        _rows("append", 1, 4096, 8, 128, "e4m3", "bf16", rows=1, name="append step b1"),
        # prompts of different lengths that arrive together, padded to a fixed row count
        _rows("append", 5, 1700, 8, 128, "bf16", "fp32", page=16, ragged=True, empty=77,
              name="append prompts"),
        # a long document
        _rows("append", 1, 32768, 8, 128, "e4m3", "bf16", name="append document"),
        # a sequence that leaves the pages for a contiguous cache
        _rows("read", 1, 1500, 8, 128, "e4m3", "bf16", name="read sequence"),
        # shared prefixes of a batch read back for a prompt's attention
        _rows("read", 6, 6400, 8, 128, "e4m3", "fp32", page=32, ragged=True, name="read prefixes"),
        # the smallest attention: a toy model
        _attn(1, 129, 4, 2, 64, "bf16", "fp32", page=16, name="attn tiny b1"),
        # one user of an 8B model
        _attn(1, 4096, 32, 8, 128, "bf16", "bf16", name="attn 8b b1"),
        # one user and a very long document, in 8 bits
        _attn(1, 131072, 32, 8, 128, "e4m3", "bf16", name="attn 8b b1 long"),
        # a busy server: lengths of all kinds, some places of the batch not in use
        _attn(32, 8192, 32, 8, 128, "e4m3", "bf16", page=16, ragged=True, empty=3,
              name="attn 8b b32 ragged"),
        # a large model's batch
        _attn(16, 8192, 64, 8, 128, "bf16", "fp32", name="attn 70b b16"),
        # every query head with keys of its own, head dimension 64
        _attn(48, 1999, 32, 32, 64, "e4m3", "fp16", page=16, ragged=True, name="attn mha d64 b48"),
        # three query heads per KV head, the last 1024 positions of each sequence
        _attn(7, 2999, 9, 3, 128, "bf16", "fp32", page=32, ragged=True, window=1024,
              name="attn window b7"),
    ]


def _log(rng, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(("append", "read", "attention", "attention", "attention"))
        kv, d = rng.choice((1, 2, 3, 4, 5, 8, 8, 8, 16, 32)), rng.choice((64, 128, 128))
        cache, io = rng.choice(("bf16", "e4m3")), rng.choice(("bf16", "fp16", "fp32"))
        page = rng.choice((8, 16, 32, 64, 128, 256))
        batch, ragged = _log(rng, 1, 200), rng.random() < 0.6
        empty = rng.randint(0, batch // 4) if rng.random() < 0.4 else 0
        if op == "attention":
            c = _attn(batch, _log(rng, 1, 150000), kv * rng.choice((1, 2, 3, 4, 4, 5, 8, 16)), kv,
                      d, cache, io, page=page, ragged=ragged, empty=empty,
                      window=_log(rng, 16, 4096) if rng.random() < 0.2 else 0)
            kept = _cached(c) * kv * d   # (a window's sequence is in the cache as a whole)
        else:
            c = _rows(op, batch, _log(rng, 1, 50000), kv, d, cache, io, page=page,
                      rows=rng.choice((0, 0, 1, 1, 3)), ragged=ragged, empty=empty)
            kept = _cached(c) * kv * d
        if work(c)["bytes"] <= most and kept <= 3e8:
            return c


# ---------------------------------------------------------------- lengths and slots

def _lengths(c: dict) -> list:
    """Cached positions of each sequence; ragged: spread from the whole context down to an eighth."""
    n, b = c["context"], c["batch"]
    live = b - c["empty"] if c["op"] == "attention" else b
    out = [max(1, n - n * 7 // 8 * i // b) if c["ragged"] else n for i in range(b)]
    return [x if i < live else 0 for i, x in enumerate(out)]


def _cached(c: dict) -> int:
    return sum(_lengths(c))


def _row_counts(c: dict) -> list:
    return [min(c["rows"], n) if c["rows"] else n for n in _lengths(c)]


def _pages(c: dict) -> list:
    return [-(-n // c["page"]) for n in _lengths(c)]


# ---------------------------------------------------------------- inputs

def _inputs(c: dict, seed: int) -> dict:
    """The pools with a context in them, the table and the call's tensors."""
    g = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 17)
    h = torch.Generator().manual_seed(1_000_003 * seed + 18)
    used = _pages(c)
    n_pages, d = sum(used) + 1 + sum(used) // 8, c["head_dim"]
    order = torch.randperm(n_pages, generator=h, dtype=torch.int32)
    table = torch.full((c["batch"], max(used)), -1, dtype=torch.int32)   # (-1: no page)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    s = dict(table=table.cuda())
    shape = (1, n_pages, c["kv_heads"], c["page"], d)
    for name in ("k", "v"):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        if c["cache"] == "bf16":
            s[name], s[name + "_scale"] = x.normal_(generator=g), None
        else:
            # codes and exponents as rows of standard normal values leave them
            x.normal_(0.0, 130.0, generator=g)
            s[name] = x.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
            s[name + "_scale"] = torch.randint(119, 122, shape[:-1], dtype=torch.uint8,
                                               device="cuda", generator=g)
    io = _TYPES[c["io"]]
    if c["op"] == "attention":
        s["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32).cuda()
        s["q"] = torch.empty(c["batch"], c["heads"], d, dtype=io, device="cuda").normal_(
            0.0, 1.5, generator=g)
        return s
    pos, seq = [], []
    for b, (n, r) in enumerate(zip(_lengths(c), _row_counts(c))):
        pos.append(torch.arange(n - r, n, dtype=torch.int32))
        seq.append(torch.full((r,), b, dtype=torch.int32))
    pos.append(torch.full((c["empty"],), -1, dtype=torch.int32))
    seq.append(torch.zeros(c["empty"], dtype=torch.int32))
    s["positions"], s["seq"] = torch.cat(pos).cuda(), torch.cat(seq).cuda()
    rows = s["positions"].numel()
    for name in ("k_rows", "v_rows"):
        x = torch.empty(rows, c["kv_heads"], d, dtype=io, device="cuda")
        s[name] = x.normal_(generator=g) if c["op"] == "append" else x.zero_()
    return s


def prepare(case: dict, seed: int) -> dict:
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    s["scale"] = 1.0 / math.sqrt(c["head_dim"])
    if c["op"] == "attention":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(c["batch"], c["heads"], dtype=torch.float32, device="cuda")
    if own:
        from paper_2410_23668_amd.device import PagedKvCache
        s["pool"] = PagedKvCache.from_tensors(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if c["op"] == "attention":
            s["workspace"] = s["pool"].workspace(c["batch"])
    return s


# ---------------------------------------------------------------- the plain forms

def _pow2(biased):
    """2^(biased - 127) in 32 bits, from the exponent's own bits."""
    return (biased.int() << 23).view(torch.float32)


def _values(pool, scale):
    """Values of cache entries in 32 bits."""
    if scale is None:
        return pool.float()
    return pool.view(torch.float8_e4m3fn).float() * _pow2(scale)[..., None]


def _bits(pool):
    return pool if pool.element_size() == 2 else pool.view(torch.uint8)


def _sequences(s, name):
    """Every sequence's entries in order, [batch][kv heads][table's positions][head dim]."""
    t = s["table"].clamp(min=0).long()
    scale = s[name + "_scale"]
    x = _values(_bits(s[name])[0][t], None if scale is None else scale[0][t])
    B, n, kv, ps, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, kv, n * ps, d)


def _plain_attention(s):
    c, q = s["case"], s["q"]
    B, nq, d = q.shape
    K, V = _sequences(s, "k"), _sequences(s, "v")
    kv, L = K.shape[1], K.shape[2]
    qt = q.float().view(B, kv, nq // kv, d).transpose(2, 3).contiguous()
    x = torch.matmul(K, qt).transpose(2, 3).contiguous() * s["scale"]   # [B][kv][group][L]
    j, n = torch.arange(L, device="cuda"), s["lengths"].long()[:, None]
    seen = (j < n) & (j >= n - c["window"] if c["window"] else j >= 0)
    x = x.masked_fill(~seen[:, None, None, :], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(x - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, V) / torch.where(l == 0, torch.ones_like(l), l)
    lse = (m + torch.log(l)).view(B, nq)
    return dict(out=o.view(B, nq, d).to(q.dtype), lse=lse)


def _slots(s):
    ps, pos = s["case"]["page"], s["positions"].long()
    ok = pos >= 0
    pos, seq = pos.clamp(min=0), s["seq"].long()
    return ok, s["table"][seq, pos // ps].long(), pos % ps


def _plain_append(s):
    ok, page, off = _slots(s)
    page, off = page[ok], off[ok]
    for name in ("k", "v"):
        x = s[name + "_rows"][ok].float()
        if s[name + "_scale"] is None:
            s[name][0][page, :, off] = x.to(torch.bfloat16)
            continue
        # the smallest power of two 2^e with |x| <= 448 2^e, from the value's own exponent
        frac, e = torch.frexp(x.abs().amax(-1))   # in [0.5, 1) 2^e; 448 = 0.875 2^9
        e = (e - 9 + (frac > 0.875).int()).clamp(min=-126)
        e = torch.where(frac == 0, torch.full_like(e, -126), e)
        code = (x * _pow2(127 - e)[..., None]).to(torch.float8_e4m3fn)
        _bits(s[name])[0][page, :, off] = code.view(torch.uint8)
        s[name + "_scale"][0][page, :, off] = (e + 127).to(torch.uint8)
    return _pool(s)


def _pool(s):
    return {n: s[n] for n in ("k", "v", "k_scale", "v_scale") if s[n] is not None}


def _plain_read(s):
    ok, page, off = _slots(s)
    out = {}
    for name in ("k", "v"):
        scale = s[name + "_scale"]
        x = _values(_bits(s[name])[0][page, :, off],
                    None if scale is None else scale[0][page, :, off])
        dst = s[name + "_rows"]   # (padding rows stay as they were)
        out[name] = dst.copy_(torch.where(ok[:, None, None], x.to(dst.dtype), dst))
    return out


def run(state: dict) -> dict:
    s, op = state, state["case"]["op"]
    if not own:
        return (_plain_attention if op == "attention" else
                _plain_append if op == "append" else _plain_read)(s)
    if op == "attention":
        s["pool"].attention(0, s["table"], s["lengths"], s["q"], s["out"], s["workspace"],
                            scale=s["scale"], window=s["case"]["window"], lse=s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if op == "append":
        s["pool"].append(0, s["table"], s["positions"], s["k_rows"], s["v_rows"], seq=s["seq"])
        return _pool(s)
    s["pool"].read(0, s["table"], s["positions"], s["k_rows"], s["v_rows"], seq=s["seq"])
    return dict(k=s["k_rows"], v=s["v_rows"])


# ---------------------------------------------------------------- what a pass has to do

def work(case: dict) -> dict:
    """Every cached row that counts and its scale byte, the call's rows and
    results, the table and the lengths or positions, each once."""
    c, d, kv, io = case, case["head_dim"], case["kv_heads"], _BYTES[case["io"]]
    row = 2 * kv * (d * _BYTES[c["cache"]] + (1 if c["cache"] == "e4m3" else 0))
    if c["op"] == "attention":
        seen = [min(n, c["window"]) if c["window"] else n for n in _lengths(c)]
        nbytes = sum(seen) * row + c["batch"] * c["heads"] * (2 * d * io + 4)
        nbytes += 4 * c["batch"] + 4 * sum(-(-n // c["page"]) for n in seen)
        return {"bytes": float(nbytes), "flops": 4.0 * c["heads"] * d * sum(seen)}
    rows = sum(_row_counts(c))
    return {"bytes": float(rows * (row + 2 * kv * d * io + 8)), "flops": 2.0 * rows * kv * d}


# ---------------------------------------------------------------- the same in 64 bits

def _entries64(s, name, b, n, page):
    """Sequence b's first n entries, [kv heads][n][head dim]."""
    pages = s["table"][b, :-(-n // page)].tolist()
    blocks = []
    for p in pages:
        x = s[name][0, p]
        if s[name + "_scale"] is None:
            blocks.append(x.double())
        else:
            blocks.append(x.double() * _pow2_64(s[name + "_scale"][0, p].int() - 127)[..., None])
    return torch.cat(blocks, 1)[:, :n]


def _pow2_64(e):
    """2^e, |e| < 200, exactly (pow may be a last bit off, which decides ties)."""
    return torch.tensor([2.0 ** i for i in range(-200, 200)], dtype=torch.float64,
                        device="cuda")[e.long() + 200]


def _e4m3_64(x):
    """Row by row: codes (as values) and biased exponents of x in 64 bits."""
    e = torch.ceil(torch.log2(x.abs().amax(-1).clamp(min=1e-300) / 448.0)).clamp(min=-126.0)
    # (448 = 0.875 2^9: the exponent from the quotient's logarithm may be one off next to a border)
    e = torch.where(x.abs().amax(-1) > 448.0 * _pow2_64(e), e + 1, e)
    e = torch.where((x.abs().amax(-1) <= 448.0 * _pow2_64(e - 1)) & (e > -126), e - 1, e)
    y = x * _pow2_64(-e)[..., None]
    # values of 4 significant bits from 2^-6 on, multiples of 2^-9 below
    log = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    log = torch.where(y.abs() >= _pow2_64(log + 1), log + 1, log)
    step = _pow2_64(torch.where((y.abs() < _pow2_64(log)) & (log > -6), log - 1, log) - 3)
    return torch.round(y / step) * step, (e + 127).to(torch.uint8)   # (round: half to even)


def exact(case: dict, seed: int) -> dict:
    """run() in 64 bits, from the definitions, sequence by sequence and row by row."""
    c, s = case, _inputs(case, seed)
    page = c["page"]
    if c["op"] == "attention":
        B, nq, d = s["q"].shape
        kv, out, lse = c["kv_heads"], torch.zeros(B, nq, d, dtype=torch.float64, device="cuda"), []
        for b, n in enumerate(_lengths(c)):
            if n == 0:
                lse.append(torch.full((nq,), -math.inf, dtype=torch.float64, device="cuda"))
                continue
            first = max(0, n - c["window"]) if c["window"] else 0
            K, V = (_entries64(s, x, b, n, page)[:, first:] for x in ("k", "v"))
            q = s["q"][b].double().view(kv, nq // kv, 1, d)
            x = torch.stack([(q[:, i] * K).sum(-1) for i in range(nq // kv)], 1) / math.sqrt(d)
            o = torch.matmul(torch.softmax(x, -1), V.contiguous())
            out[b] = o.reshape(nq, d)
            lse.append(torch.logsumexp(x, -1).reshape(nq))
        return dict(out=out, lse=torch.stack(lse))
    pos, seq = s["positions"].tolist(), s["seq"].tolist()
    rows = [i for i, p in enumerate(pos) if p >= 0]
    at = torch.tensor([[s_, pos[i] // page, pos[i] % page] for i, s_ in enumerate(seq) if pos[i] >= 0],
                      dtype=torch.int64).view(-1, 3).cuda()
    pages, off = s["table"].long()[at[:, 0], at[:, 1]], at[:, 2]
    res = {}
    for name in ("k", "v"):
        x, scale = s[name].double(), s[name + "_scale"]
        if c["op"] == "append":
            new = s[name + "_rows"][rows].double()
            if scale is not None:
                new, scale[0].view(-1)[_flat(scale[0], pages, off)] = _e4m3_64(new)
                res[name + "_scale"] = scale
            else:
                new = new.to(torch.bfloat16).double()   # (the value that the cache holds)
            x[0, pages, :, off] = new
            res[name] = x
        else:
            if scale is not None:
                x = x * _pow2_64(scale.int() - 127)[..., None]
            y = torch.zeros_like(s[name + "_rows"], dtype=torch.float64)
            y[rows] = x[0, pages, :, off]
            res[name] = y
    return res


def _flat(scale, pages, off):
    """Places of rows' scales, [rows][kv heads], in a flattened pool of scales."""
    n, kv, ps = scale.shape
    return (pages[:, None] * kv + torch.arange(kv, device="cuda")) * ps + off[:, None]
