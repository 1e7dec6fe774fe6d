"""The paged cache's operators on the GPU against plain implementations in 64
bits: rows quantised as they are written, rows read back, and the attention of
one new token per sequence."""
import math

import pytest
import torch

from paper_2410_23668_amd import binding as kb
from paper_2410_23668_amd.device import KvCache, PagedKvCache
from tests.paged_cases import (BF16, E4M3, FP16, FP32, attention64, check_attention, e4m3_rows,
                               half_step, make_pool, make_table, values)

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator().manual_seed(seed)


def snapshot(pool):
    return [None if x is None else x.view(torch.uint8).clone()
            for x in (pool.k, pool.v, pool.k_scale, pool.v_scale)]


def same_bits(a, b):
    return all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b))


# ---------------------------------------------------------------- append

def special_rows(n, kv, d, g):
    """Rows where quantising can go wrong: zeros, one value, ties between codes,
    magnitudes at and next to a scale's border, tiny and huge ones."""
    x = torch.randn(n, kv, d, generator=g)
    x[0] = 0.0
    x[1] = 0.0
    x[1, :, 3] = -1.0
    x[2] = torch.arange(d).float() * 0.0625 + 1.0          # (ties at 4 significant bits)
    x[3] *= 448.0 / x[3].abs().amax(-1, keepdim=True)
    x[3, :, 5] = 448.0                                     # largest code, no larger scale
    x[4, :, 5] = 450.0                                     # next scale
    x[5] *= 2.0 ** -120                                    # e near its lower bound
    x[6] *= 2.0 ** -135
    x[7] *= 2.0 ** 125
    x[8, :, 0] = 448.0 * 2.0 ** 4
    x[8, :, 1:] *= 2.0 ** -14                              # codes below the normal range
    x[9] = 2.0 ** -9 * (torch.arange(d).float() + 0.5)     # ties of those
    x[9, :, 0] = 256.0
    return x


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io", [BF16, FP16, FP32])
@pytest.mark.parametrize("d,kv,page", [(64, 3, 8), (128, 8, 16), (128, 1, 256), (64, 5, 64)])
def test_append_writes_the_rows_and_nothing_else(cache, io, d, kv, page):
    g = gen(d + kv + page)
    lengths = [37, 1, 129]
    n_pages = 64
    pool = make_pool(2, n_pages, kv, page, d, cache, g)
    table = make_table(lengths, page, n_pages, g)
    pos = torch.cat([torch.arange(n) for n in lengths] + [torch.tensor([-1, -5])]).to(torch.int32)
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(lengths)] +
                    [torch.tensor([0, 77])]).to(torch.int32)
    perm = torch.randperm(len(pos), generator=g)
    pos, seq = pos[perm], seq[perm]
    n = len(pos)
    with torch.no_grad():
        k, v = (special_rows(n, kv, d, g)[torch.randperm(n, generator=g)].to(io) for _ in range(2))
    if io != FP16:
        k[torch.nonzero(pos == 7)[0, 0], 0, 11] = math.nan
        v[torch.nonzero(pos == 9)[0, 0], kv - 1, 0] = -math.inf
    want = snapshot(pool)
    ok = pos >= 0
    pg, off = table[seq[ok].long(), pos[ok].long() // page].long(), pos[ok].long() % page
    for i, x in enumerate((k, v)):
        if cache == BF16:
            w = want[i].view(BF16)
            w[1][pg.cuda(), :, off.cuda()] = x[ok].float().to(BF16).cuda()
        else:
            codes, scale = e4m3_rows(x[ok])
            want[i][1][pg.cuda(), :, off.cuda()] = codes.cuda()
            want[i + 2][1][pg.cuda(), :, off.cuda()] = scale.cuda()
    pool.append(1, table.cuda(), pos.cuda(), k.cuda(), v.cuda(), seq=seq.cuda())
    got = snapshot(pool)
    for a, b, what in zip(got, want, ("k", "v", "k_scale", "v_scale")):
        if a is None:
            continue
        if cache == BF16 and what in ("k", "v"):   # (a NaN may be any NaN)
            fa, fb = a.view(BF16).float(), b.view(BF16).float()
            assert torch.equal(torch.isnan(fa), torch.isnan(fb)), what
            a, b = fa.nan_to_num(), fb.nan_to_num()
        assert torch.equal(a, b), f"{what}: {int((a != b).sum())} differ"
    assert pool.device_error() == 0


def test_append_takes_any_strides_and_alignment():
    g = gen(5)
    kv, d, page, n = 3, 64, 16, 21
    table = make_table([n], page, 4, g).cuda()
    pos = torch.arange(n, dtype=torch.int32).cuda()
    seq = torch.zeros(n, dtype=torch.int32).cuda()
    for io in (BF16, FP16, FP32):
        flat = torch.randn(4 * n * kv * d, generator=g).to(io).cuda()
        layouts = [flat.as_strided((n, kv, d), (kv * d + 1, d, 1), 1),          # misaligned
                   flat.as_strided((n, kv, d), (d, n * d, 1), 0),               # heads outermost
                   flat.as_strided((n, kv, d), (0, d + 3, 1), 5),               # one row for all
                   flat.as_strided((n, kv, d), (3 * kv * d + 8, 2 * d, 1), 8)]  # gaps
        for cache in (BF16, E4M3):
            for x in layouts:
                a, b = (make_pool(1, 4, kv, page, d, cache, gen(1)) for _ in range(2))
                a.append(0, table, pos, x, x, seq=seq)
                b.append(0, table, pos, x.contiguous(), x.contiguous(), seq=seq)
                assert same_bits(snapshot(a), snapshot(b))


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("d", [64, 128])
def test_keys_and_values_of_their_own_strides_and_types(cache, d):
    g = gen(6)
    kv, page, n = 3, 16, 21
    table = make_table([n], page, 4, g).cuda()
    pos = torch.arange(n, dtype=torch.int32).cuda()
    seq = torch.zeros(n, dtype=torch.int32).cuda()
    k = torch.randn(4 * n * kv * d, generator=g).to(FP16).cuda().as_strided(
        (n, kv, d), (3 * kv * d + 8, 2 * d, 1), 8)
    v = torch.randn(n, kv, d, generator=g).cuda()
    a, b = (make_pool(1, 4, kv, page, d, cache, gen(1)) for _ in range(2))
    a.append(0, table, pos, k, v, seq=seq)
    b.append(0, table, pos, k.float().contiguous(), v, seq=seq)
    assert same_bits(snapshot(a), snapshot(b))
    outs = []
    for ko, vo in ((torch.full((n, kv, d), 7.0, dtype=FP16, device="cuda"),
                    torch.full((kv, n, d), 7.0, device="cuda").transpose(0, 1)),
                   (torch.full((n, kv, d), 7.0, dtype=FP16, device="cuda"),
                    torch.full((n, kv, d), 7.0, device="cuda"))):
        a.read(0, table, pos, ko, vo, seq=seq)
        outs.append((ko, vo))
    for x, y in zip(*outs):
        assert torch.equal(x, y) and bool((x != 7.0).any())
    want = [values(a, w)[0, table.cpu()[0].long()[torch.arange(n) // page], :, torch.arange(n) % page]
            for w in "kv"]
    assert torch.equal(outs[1][0].cpu(), want[0].to(FP16)) and torch.equal(outs[1][1].cpu(), want[1].float())


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_bad_rows_are_skipped_and_reported(cache):
    g = gen(6)
    kv, d, page = 2, 64, 8
    pool = make_pool(1, 6, kv, page, d, cache, g)
    table = torch.tensor([[0, 6, 2], [3, -1, 5]], dtype=torch.int32).cuda()
    x = torch.randn(4, kv, d, generator=g).cuda()
    before = snapshot(pool)

    def call(pos, seq):
        pool.append(0, table, torch.tensor(pos, dtype=torch.int32).cuda(), x[:len(pos)], x[:len(pos)],
                    seq=torch.tensor(seq, dtype=torch.int32).cuda())
        return pool.device_error()

    assert call([24, 1 << 30], [0, 1]) == kb.KL_DEVERR_POSITION
    assert call([0, 0], [2, -1]) == kb.KL_DEVERR_POSITION
    assert call([8, 15], [0, 1]) == kb.KL_DEVERR_PAGE
    assert same_bits(snapshot(pool), before)
    assert call([-1, -1, 8, 30], [0, 9, 1, 0]) == kb.KL_DEVERR_PAGE | kb.KL_DEVERR_POSITION
    assert same_bits(snapshot(pool), before)
    out = torch.full((4, kv, d), 7.0, device="cuda")
    pool.read(0, table, torch.tensor([0, 8, -1, 99], dtype=torch.int32).cuda(), out, out.clone(),
              seq=torch.tensor([0, 0, 0, 1], dtype=torch.int32).cuda())
    assert pool.device_error() == kb.KL_DEVERR_PAGE | kb.KL_DEVERR_POSITION
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1]).all() and torch.isnan(out[3]).all()
    assert bool((out[2] == 7.0).all())


def test_append_and_read_of_no_rows():
    pool = make_pool(1, 2, 1, 8, 64, E4M3, gen(2))
    table = torch.zeros(1, 1, dtype=torch.int32).cuda()
    before = snapshot(pool)
    none = torch.empty(0, 1, 64, device="cuda")
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    pool.append(0, table, pos, none, none)
    pool.read(0, table, pos, none, none)
    assert same_bits(snapshot(pool), before) and pool.device_error() == 0


# ---------------------------------------------------------------- read

@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io", [BF16, FP16, FP32])
@pytest.mark.parametrize("d,kv,page", [(64, 3, 8), (128, 8, 32), (128, 2, 4096)])
def test_read_gives_the_values_back(cache, io, d, kv, page):
    g = gen(d + kv + page + 1)
    lengths = [50, 0, 33]
    n_pages = 20 if page < 100 else 3
    pool = make_pool(2, n_pages, kv, page, d, cache, g)
    table = make_table(lengths, page, n_pages, g)
    pos = torch.cat([torch.arange(n) for n in lengths] + [torch.tensor([-1])]).to(torch.int32)
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(lengths)] +
                    [torch.tensor([0])]).to(torch.int32)
    n = len(pos)
    pg, off = table[seq[:-1].long(), pos[:-1].long() // page].long(), pos[:-1].long() % page
    for strided in (False, True):
        if strided:   # heads outermost, at an odd offset of a larger buffer
            buf = [torch.full((kv * n * d + 9,), 3.0, dtype=io, device="cuda") for _ in range(2)]
            out = [x.as_strided((n, kv, d), (d, n * d, 1), 3) for x in buf]
        else:
            out = [torch.full((n, kv, d), 3.0, dtype=io, device="cuda") for _ in range(2)]
        pool.read(1, table.cuda(), pos.cuda(), out[0], out[1], seq=seq.cuda())
        for o, name in zip(out, ("k", "v")):
            want = values(pool, name)[1][pg, :, off].to(io)   # (one rounding)
            assert torch.equal(o[:-1].cpu(), want)
            assert bool((o[-1] == 3.0).all())
        if strided:
            for x in buf:
                assert bool((x[:3] == 3.0).all()) and bool((x[-6:] == 3.0).all())
    assert pool.device_error() == 0


@pytest.mark.parametrize("io", [BF16, FP16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_read_of_the_smallest_scales_rounds_once(io, d):
    # every code at scale bytes 1 to 4 (and the largest that append writes): exact in fp32,
    # in bf16 rounded where codes are multiples of less than 2^-133
    page, kv = 16, 2
    for rows in (3, 2000):   # (few and many: different kernels)
        n_pages = -(-rows // page)
        pool = make_pool(1, n_pages, kv, page, d, E4M3, gen(2))
        for name in ("k", "v"):
            codes = torch.randint(0, 127, pool.k.shape, generator=gen(10), dtype=torch.uint8)
            codes += 128 * torch.randint(0, 2, codes.shape, generator=gen(12), dtype=torch.uint8)
            getattr(pool, name).view(torch.uint8).copy_(codes)
            scale = torch.randint(1, 5, codes.shape[:-1], generator=gen(11), dtype=torch.uint8)
            scale[..., 0] = 246   # (448 2^119 is a number of every type but fp16)
            getattr(pool, name + "_scale").copy_(scale)
        table = make_table([rows], page, n_pages, gen(4))
        pos = torch.arange(rows, dtype=torch.int32)
        out = [torch.full((rows, kv, d), 3.0, dtype=io, device="cuda") for _ in range(2)]
        pool.read(0, table.cuda(), pos.cuda(), out[0], out[1], seq=torch.zeros_like(pos).cuda())
        pg, off = table[0, pos.long() // page].long(), pos.long() % page
        for o, name in zip(out, ("k", "v")):
            assert torch.equal(o.cpu(), values(pool, name)[0][pg, :, off].to(io))


# ---------------------------------------------------------------- attention

def run_attention(pool, table, lengths, q, page, layer=0, scale=None, window=0, dtype=None, ws=None):
    B, nq, d = q.shape
    out = torch.full((B, nq, d), 9.0, dtype=dtype or q.dtype, device="cuda")
    lse = torch.full((B, nq), 9.0, device="cuda")
    ws = pool.workspace(B) if ws is None else ws
    pool.attention(layer, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), q.cuda(),
                   out, ws, scale=scale, window=window, lse=lse)
    return out, lse


CASES = [   # heads, kv, d, page, lengths, window
    (4, 2, 64, 16, [1], 0),
    (1, 1, 128, 8, [2], 0),
    (32, 8, 128, 64, [129], 0),
    (8, 8, 64, 8, [31, 32, 33, 0, 1], 0),
    (6, 2, 128, 16, [63, 64, 65, 127, 128, 129, 255, 257], 0),
    (15, 3, 128, 32, [500, 1, 0, 77], 0),
    (16, 1, 128, 16, [1000, 3], 0),
    (16, 1, 64, 256, [700, 300], 0),
    (64, 8, 128, 128, [513, 40], 0),
    (32, 32, 64, 16, [90, 200, 7], 0),
    (24, 8, 128, 64, [0, 0], 0),
    (8, 4, 64, 4096, [4100, 4096, 4095], 0),
    (6, 2, 128, 8, [100, 50, 9, 3, 1], 8),
    (4, 4, 64, 16, [300, 299, 17, 16, 0], 33),
    (12, 4, 128, 32, [2000, 100, 1024, 1025], 1024),
    (4, 2, 128, 64, [90, 10], 1),
]


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io", [BF16, FP16, FP32])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"h{c[0]}-{c[1]}-d{c[2]}-p{c[3]}-n{max(c[4])}-w{c[5]}")
def test_attention_matches_64_bits(cache, io, case):
    nq, kv, d, page, lengths, window = case
    g = gen(nq + d + page)
    n_pages = sum(-(-n // page) for n in lengths) + 3
    pool = make_pool(2, n_pages, kv, page, d, cache, g)
    table = make_table(lengths, page, n_pages, g)
    q = (torch.randn(len(lengths), nq, d, generator=g) * 2).to(io)
    scale = 1 / math.sqrt(d)
    want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, page, scale, window, 1)
    out, lse = run_attention(pool, table, lengths, q, page, 1, window=window)
    check_attention(out, lse, want, "attention")
    for b, n in enumerate(lengths):
        if n == 0:
            assert bool((out[b] == 0).all()) and bool((lse[b] == -math.inf).all())
    assert pool.device_error() == 0


@pytest.mark.parametrize("q_type,out_type", [(BF16, FP32), (FP32, BF16), (FP16, FP32), (FP32, FP16)])
def test_attention_output_type_is_its_own(q_type, out_type):
    g = gen(12)
    pool = make_pool(1, 20, 2, 16, 128, E4M3, g)
    lengths = [150, 60]
    table = make_table(lengths, 16, 20, g)
    q = torch.randn(2, 8, 128, generator=g).to(q_type)
    want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, 16, 128 ** -0.5)
    out, lse = run_attention(pool, table, lengths, q, 16, dtype=out_type)
    check_attention(out, lse, want)


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_attention_scales(cache, scale):
    # (scale 4: one position has nearly all the weight, and the running maximum moves)
    g = gen(13)
    pool = make_pool(1, 70, 2, 8, 64, cache, g)
    lengths = [500]
    table = make_table(lengths, 8, 70, g)
    q = torch.randn(1, 4, 64, generator=g)
    want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, 8, scale)
    out, lse = run_attention(pool, table, lengths, q, 8, scale=scale)
    check_attention(out, lse, want)


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("scale,query,key", [(2.0 ** 127, 2.0 ** -100, 2.0 ** -29),
                                             (-2.0 ** 127, 2.0 ** -100, 2.0 ** -29),
                                             (2.0 ** -126, 2.0 ** 62, 2.0 ** 60),
                                             (2.0 ** -140, 2.0 ** 62, 2.0 ** 60)])
def test_attention_of_the_largest_and_smallest_scales(cache, scale, query, key):
    # keys are multiples of 'key' of 4 significant bits: scores in steps of 1/4 (or, of the
    # smallest scale, next to none)
    d, n, page = 64, 300, 16
    pool = make_pool(1, 20, 1, page, d, cache, gen(3))
    table = make_table([n], page, 20, gen(4))
    k = torch.zeros(n, 1, d)
    k[:, 0, 0] = torch.randint(-15, 16, (n,), generator=gen(8)).float() * key
    pos = torch.arange(n, dtype=torch.int32).cuda()
    pool.append(0, table.cuda(), pos, k.cuda(), torch.randn(n, 1, d, generator=gen(9)).cuda(),
                seq=torch.zeros_like(pos))
    q = torch.zeros(1, 3, d)
    q[:, 0, 0], q[:, 1, 0] = query, -query
    want = attention64(values(pool, "k"), values(pool, "v"), table, [n], q, page, scale)
    out, lse = run_attention(pool, table, [n], q, page, scale=scale)
    check_attention(out, lse, want)


def test_attention_rising_and_falling_scores():
    # the running maximum rises at every position, or never after the first
    d, n, page = 128, 700, 16
    for sign in (1.0, -1.0):
        pool = make_pool(1, 50, 1, page, d, BF16, gen(3))
        k = torch.zeros(n, 1, d)
        k[:, 0, 0] = sign * torch.arange(n).float() * 0.25
        table = make_table([n], page, 50, gen(4))
        pos = torch.arange(n, dtype=torch.int32).cuda()
        v = torch.randn(n, 1, d, generator=gen(9)).cuda()
        pool.append(0, table.cuda(), pos, k.cuda(), v, seq=torch.zeros_like(pos))
        q = torch.zeros(1, 2, d)
        q[:, :, 0] = 30.0
        want = attention64(values(pool, "k"), values(pool, "v"), table, [n], q, page, d ** -0.5)
        out, lse = run_attention(pool, table, [n], q, page)
        check_attention(out, lse, want)


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_attention_of_large_and_tiny_values(cache):
    # sums stay below the largest value where the weights do not pass 1, also
    # while scores rise; tiny values keep their precision
    d, n, page = 128, 300, 16
    for mag in (1.2e36, 1e-30):
        pool = make_pool(1, 20, 1, page, d, cache, gen(3))
        k = torch.zeros(n, 1, d)
        k[:, 0, 0] = torch.arange(n).float() * 0.125
        v = (torch.rand(n, 1, d, generator=gen(9)) + 0.5) * mag
        table = make_table([n], page, 20, gen(4))
        pos = torch.arange(n, dtype=torch.int32).cuda()
        pool.append(0, table.cuda(), pos, k.cuda(), v.cuda(), seq=torch.zeros_like(pos))
        q = torch.zeros(1, 2, d)
        q[:, 0, 0], q[:, 1, 0] = 10.0, -4.0
        want = attention64(values(pool, "k"), values(pool, "v"), table, [n], q, page, d ** -0.5)
        out, lse = run_attention(pool, table, [n], q, page)
        check_attention(out, lse, want)


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io", [BF16, FP32])
@pytest.mark.parametrize("key,query,scale", [(2.0 ** 20, 2.0 ** 20, 0.125), (2.0 ** 20, 2.0 ** 20, -0.125),
                                             (2.0 ** 100, 2.0 ** 26, 1.0)])
def test_attention_of_scores_far_apart(cache, io, key, query, scale):
    # scores are multiples of 2^37 (or 2^126): the largest have all the weight, shared
    # equally, whatever the rounding of scores in log2 units
    d, page, lengths = 64, 16, [1, 40, 1500, 5000]
    pool = make_pool(1, 450, 2, page, d, cache, gen(3))
    table = make_table(lengths, page, 450, gen(4))
    out_of = torch.empty(4, 6, d, dtype=torch.float64)
    tol, lse_of = torch.empty_like(out_of), torch.empty(4, 6, dtype=torch.float64)
    rows = []
    for b, n in enumerate(lengths):
        m = torch.randint(-3, 2, (n, 2), generator=gen(b)).float()
        m[n // 2:] += 1   # (the maximum of the first half is passed)
        k = torch.zeros(n, 2, d)
        k[:, :, 0] = m * key
        v = torch.randn(n, 2, d, generator=gen(20 + b))
        pos = torch.arange(n, dtype=torch.int32)
        seq = torch.full_like(pos, b)
        pool.append(0, table.cuda(), pos.cuda(), k.cuda(), v.cuda(), seq=seq.cuda())
        rows.append(m)
    V = values(pool, "v")
    for b, n in enumerate(lengths):
        pg, off = table[b].long()[torch.arange(n) // page], torch.arange(n) % page
        for h in range(6):
            x = rows[b][:, h // 3] * (1 if scale > 0 else -1)
            top = x == x.max()
            v = V[0, pg, h // 3, off][top]
            out_of[b, h] = v.mean(0)
            tol[b, h] = 2.0 ** -24 * (32 + 8 * math.sqrt(n)) * v.abs().mean(0)
            lse_of[b, h] = float(x.max()) * key * query * abs(scale) + math.log(int(top.sum()))
    ltol = 2.0 ** -23 * lse_of.abs() + 2.0 ** -24 * (32 + 8 * math.sqrt(5000))
    q = torch.zeros(4, 6, d)
    q[:, :, 0] = query
    out, lse = run_attention(pool, table, lengths, q.to(io), page, scale=scale)
    check_attention(out, lse, (out_of, lse_of, tol, ltol))


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io", [BF16, FP32])
def test_attention_of_scores_that_overflow(cache, io):
    # a score below every number (its sum of products overflows) has no weight: at the
    # sequence's start, for whole tiles and workgroups, in between, or everywhere (NaN)
    d, page, n = 128, 16, 3000
    for where in (slice(0, 2000), slice(1, None, 2), slice(0, 2999), slice(10, None), slice(0, None)):
        pool = make_pool(1, 200, 1, page, d, cache, gen(3))
        table = make_table([n], page, 200, gen(4))
        k = torch.zeros(n, 1, d)
        k[where, 0, 0] = -2.0 ** 100
        v = torch.randn(n, 1, d, generator=gen(9))
        pos = torch.arange(n, dtype=torch.int32).cuda()
        pool.append(0, table.cuda(), pos, k.cuda(), v.cuda(), seq=torch.zeros_like(pos))
        q = torch.zeros(1, 2, d)
        q[:, 0, 0] = 2.0 ** 100   # (the other head: all scores 0)
        out, lse = run_attention(pool, table, [n], q.to(io), page)
        V = values(pool, "v")[0, table[0].long()[torch.arange(n) // page], 0, torch.arange(n) % page]
        some = torch.ones(n, dtype=torch.bool)
        some[where] = False
        for h, left in ((0, some), (1, torch.ones_like(some))):
            if not bool(left.any()):
                assert bool(torch.isnan(out[0, h]).all()) and float(lse[0, h]) == -math.inf
                continue
            x = V[left]
            tol = 2.0 ** -24 * (32 + 8 * math.sqrt(n)) * x.abs().mean(0)
            want = (x.mean(0), torch.tensor(math.log(len(x)), dtype=torch.float64), tol,
                    torch.tensor(2.0 ** -24 * (32 + 8 * math.sqrt(n) + 16)))
            check_attention(out[0, h], lse[0, h], want, f"{where}, head {h}")


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io,query,key", [(FP32, 2.0 ** 100 * (2 - 2.0 ** -10), -2.0 ** 100),
                                          (FP32, 3.4e38, -2.0),
                                          (FP32, 2.0 ** 70 * (1 + 2.0 ** -8 + 2.0 ** -9), -2.0 ** 70),
                                          (FP16, 2.0 ** 14 * (2 - 2.0 ** -10), -2.0 ** 126)])
def test_attention_of_scores_that_overflow_whatever_the_query_rounds_to(cache, io, query, key):
    # products of query and key are below every number, of queries that are no bf16 values:
    # their bf16 terms must not overflow to both sides, nor where the query itself does not
    d, page, n = 64, 16, 1200
    pool = make_pool(1, 80, 1, page, d, cache, gen(3))
    table = make_table([n], page, 80, gen(4))
    k = torch.zeros(n, 1, d)
    k[::2, 0, 0] = key
    v = torch.randn(n, 1, d, generator=gen(9))
    pos = torch.arange(n, dtype=torch.int32).cuda()
    pool.append(0, table.cuda(), pos, k.cuda(), v.cuda(), seq=torch.zeros_like(pos))
    q = torch.zeros(1, 3, d)
    q[:, 0, 0], q[:, 1, 0] = query, -query   # (head 1: above every number; head 2: all scores 0)
    out, lse = run_attention(pool, table, [n], q.to(io), page, scale=1.0)
    V = values(pool, "v")[0, table[0].long()[torch.arange(n) // page], 0, torch.arange(n) % page]
    for h, x in ((0, V[1::2]), (2, V)):
        m = x.shape[0]
        tol = 2.0 ** -24 * (32 + 8 * math.sqrt(m)) * x.abs().mean(0)
        want = (x.mean(0), torch.tensor(math.log(m), dtype=torch.float64), tol,
                torch.tensor(2.0 ** -24 * (32 + 8 * math.sqrt(m) + 16)))
        check_attention(out[0, h], lse[0, h], want, f"head {h}")
    assert bool(torch.isnan(out[0, 1]).all())


def cancelling(pool, group, kv, B, page, d):
    """Sequences of six positions of which the last five cancel, head by head:
    keys k0 (the largest score, value 0), kA (value 1) and four times kB, whose
    values add up to -pA / pB of head e % group in element e."""
    rows_k, rows_v, qh = [], [], 1 + torch.arange(group).double() / 16
    step = 2.0 ** -3
    for b in range(B):
        a, c = step * (1 + b % 16), step * (2 + (5 * b) % 15)
        k = torch.zeros(6, kv, d, dtype=torch.float64)
        k[1, :, 0], k[2:, :, 0] = -a, -c
        v = torch.zeros(6, kv, d, dtype=torch.float64)
        v[1] = 1.0
        left = -torch.exp(qh * (c - a))[torch.arange(d) % group].expand(kv, d)
        for i in range(2, 6):
            if pool.k.dtype == BF16:
                v[i] = left.to(BF16).double()
            else:
                codes, s = e4m3_rows(left)
                v[i] = codes.view(E4M3).float().double() * torch.exp2(s.double() - 127)[..., None]
            left = left - v[i]
        rows_k.append(k)
        rows_v.append(v)
    table = torch.arange(B, dtype=torch.int32)[:, None].contiguous()
    pos = torch.arange(6, dtype=torch.int32).repeat(B)
    seq = torch.arange(B, dtype=torch.int32).repeat_interleave(6)
    pool.append(0, table.cuda(), pos.cuda(), torch.cat(rows_k).float().cuda(),
                torch.cat(rows_v).float().cuda(), seq=seq.cuda())
    q = torch.zeros(B, kv * group, d, dtype=torch.float64)
    q[:, :, 0] = qh.repeat(kv)
    return table, q


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io", [BF16, FP16, FP32])
@pytest.mark.parametrize("d,group", [(64, 4), (128, 8), (128, 16)])
def test_attention_where_values_cancel(cache, io, d, group):
    # Outputs of a 2^-15th of sum p |v| or less: half a step of any type is far below
    # what the weights' own rounding leaves.  Scores are exact (one product of 4 and 8
    # significant bits, at most 4 in magnitude).  A weight: its exponent c (s - m) - 8, below
    # 16 in magnitude, is rounded by 2^-21 (times ln 2), c by 2^-24 of 5.8 in either of two
    # roundings, the exponential by 2^-23: 2^-20.5 together; the six products that count are
    # added in fp32, 2^-23 of sum p |v| each: 2^-20.4.  Together 2^-19.4, of sum p |v|.
    # (Weights of 16 bits would be off by up to 2^-17.)
    B, kv, page = 32, 2, 8
    pool = make_pool(1, B, kv, page, d, cache, gen(5))
    table, q = cancelling(pool, group, kv, B, page, d)
    q = q.to(io)
    want = attention64(values(pool, "k"), values(pool, "v"), table, [6] * B, q, page, 1.0)
    K, V = values(pool, "k")[0], values(pool, "v")[0]
    out, lse = run_attention(pool, table, [6] * B, q, page, scale=1.0)
    mag = torch.zeros_like(want[0])
    for b in range(B):
        for h in range(kv * group):
            p = torch.softmax(K[b, h // group, :6] @ q[b, h].double(), 0)
            mag[b, h] = p @ V[b, h // group, :6].abs()
    hit = torch.arange(d)[None] % group == (torch.arange(kv * group) % group)[:, None]
    assert float((want[0].abs() / mag)[:, hit].max()) < 2.0 ** -15
    check_attention(out, lse, (want[0], want[1], 2.0 ** -19.4 * mag, want[3]))


@pytest.mark.parametrize("io", [BF16, FP32])
@pytest.mark.parametrize("d,group", [(64, 1), (128, 4), (128, 16)])
def test_attention_of_the_smallest_scales(io, d, group):
    # An e4m3 pool's smallest scales, beside large ones or alone.  The weights are 2^-8
    # times p or less, and nearly equal (scores differ by 0.05 at most): of n values three
    # products each are rounded by 2^-150 at most, 3 2^-142 / 0.95 < 2^-140 of the output.
    # Values are taken as bf16, whose smallest step is 2^-133: at scale bytes 1 and 2
    # (random codes) off by 2^-134 at most, as a bf16 output of that size is.
    n, page = 300, 16
    pos = torch.arange(n, dtype=torch.int32).cuda()
    for what in (448 * 2.0 ** -126, 1e-34, 1e-32, 1e-28, "apart", "codes"):
        pool = make_pool(1, 20, 1, page, d, E4M3, gen(3))
        k = torch.zeros(n, 1, d)
        k[:, 0, 0] = torch.arange(n).float() * 0.125
        v = torch.rand(n, 1, d, generator=gen(9)) * 0.5 + 0.5
        if what == "apart":
            v *= 1e-34
            v[::2] = 0.0
            v[:, :, 0] = 0.0
            v[::2, :, 0] = 1e30
        elif what != "codes":
            v *= what
        table = make_table([n], page, 20, gen(4))
        pool.append(0, table.cuda(), pos, k.cuda(), v.cuda(), seq=torch.zeros_like(pos))
        if what == "codes":
            codes = torch.randint(0, 127, pool.v.shape, generator=gen(10), dtype=torch.uint8)
            codes += 128 * torch.randint(0, 2, codes.shape, generator=gen(12), dtype=torch.uint8)
            pool.v.view(torch.uint8).copy_(codes)
            pool.v_scale.copy_(torch.randint(1, 4, pool.v_scale.shape, generator=gen(11), dtype=torch.uint8))
        q = torch.zeros(1, group, d)
        q[:, 0, 0] = 0.01
        q = q.to(io)
        o, l, tol, ltol = attention64(values(pool, "k"), values(pool, "v"), table, [n], q, page, d ** -0.5)
        tol = tol + 2.0 ** -140 + (2.0 ** -133 if what == "codes" else 0.0)
        out, lse = run_attention(pool, table, [n], q, page)
        check_attention(out, lse, (o, l, tol, ltol), f"{what}")


def garbage(pool, used):
    """Everything that no attended position uses: NaN, infinities, and scale bytes of all kinds."""
    for name in ("k", "v"):
        x = getattr(pool, name)
        keep = used.cuda()
        if x.dtype == BF16:
            bad = torch.full_like(x, math.nan)
            bad[..., ::2] = math.inf
            x.copy_(torch.where(keep[None, :, None, :, None], x, bad))
        else:
            b = x.view(torch.uint8)
            b.copy_(torch.where(keep[None, :, None, :, None], b, torch.full_like(b, 0x7F)))
            s = getattr(pool, name + "_scale")
            junk = torch.randint(0, 2, s.shape, dtype=torch.uint8, device="cuda") * 255
            s.copy_(torch.where(keep[None, :, None, :], s, junk))


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [0, 45])
def test_attention_ignores_what_it_does_not_attend(cache, d, window):
    page, kv, nq = 16, 2, 8
    lengths = [100, 1, 0, 47, 333, 64]
    g = gen(d + window)
    n_pages = 50
    pool = make_pool(1, n_pages, kv, page, d, cache, g)
    table = make_table(lengths, page, n_pages, g, fill=2 ** 30)
    used = torch.zeros(n_pages, page, dtype=torch.bool)
    for b, n in enumerate(lengths):
        j = torch.arange(max(0, n - window) if window else 0, n)
        used[table[b].long()[j // page], j % page] = True
        if window:   # (pages before the window have been given back)
            table[b, :max(0, n - window) // page] = -7
    garbage(pool, used)
    q = torch.randn(len(lengths), nq, d, generator=g)
    want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, page, d ** -0.5, window)
    out, lse = run_attention(pool, table, lengths, q, page, window=window)
    check_attention(out, lse, want)
    assert pool.device_error() == 0


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("n,kv,batch", [(1, 1, 1), (31, 8, 3), (1023, 2, 5), (4097, 8, 1),
                                        (100003, 1, 1), (20011, 3, 2), (131, 4, 300)])
def test_attention_counts_every_position_once(cache, n, kv, batch):
    # equal scores, values 1: the output is 1 and the lse ln n (a missing or
    # doubled position is 1 / n off, and the sum of up to 2^24 ones is exact)
    page, d = 64, 64
    need = -(-n // page)
    n_pages = need * min(batch, 4)
    pool = PagedKvCache(dict(n_layers=1, n_kv_heads=kv, head_dim=d), n_pages, page, cache)
    pool.k.view(torch.uint8).zero_()
    pool.v.copy_(torch.ones(1, device="cuda").expand(pool.v.shape).to(cache))
    table = torch.stack([torch.randperm(need, generator=gen(b)).to(torch.int32) + need * (b % 4)
                         for b in range(batch)])
    lengths = [n - b % 7 if n > 7 else n for b in range(batch)]
    q = torch.randn(batch, 2 * kv, d, generator=gen(1))
    out, lse = run_attention(pool, table, lengths, q, page)
    want = torch.log(torch.tensor(lengths, dtype=torch.float64))[:, None]
    # (an fp32 logarithm: a step or two of its value)
    assert float(((lse.double().cpu() - want).abs() / want.clamp(min=1)).max()) <= 3 * 2.0 ** -23
    assert float((out - 1).abs().max()) <= 4 * 2.0 ** -24


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_attention_reports_bad_sequences(cache):
    g = gen(21)
    page, kv, nq, d = 16, 2, 4, 128
    pool = make_pool(1, 30, kv, page, d, cache, g)
    lengths = [100, 90, 80, 70, 60, 10]
    table = make_table(lengths, page, 30, g, extra=0)
    bad = table.clone()
    bad[1, 3] = 30           # one page past the pool
    bad[4, 0] = -1
    lens = list(lengths)
    lens[2] = table.shape[1] * page + 1
    lens[3] = -4
    q = torch.randn(6, nq, d, generator=g)
    want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, page, d ** -0.5)
    out, lse = run_attention(pool, bad, lens, q, page)
    assert pool.device_error() == kb.KL_DEVERR_PAGE | kb.KL_DEVERR_POSITION
    for b in (1, 2, 3, 4):
        assert torch.isnan(out[b]).all() and torch.isnan(lse[b]).all()
    keep = [0, 5]
    check_attention(out[keep], lse[keep], [w[keep] for w in want])


def test_attention_strides_and_untouched_places():
    g = gen(22)
    page, kv, nq, d = 16, 2, 6, 64
    pool = make_pool(1, 30, kv, page, d, E4M3, g)
    lengths = [100, 33, 0]
    table = make_table(lengths, page, 30, g)
    for io in (BF16, FP16, FP32):
        big = torch.randn(4000, generator=g).to(io).cuda()
        q = big.as_strided((3, nq, d), (nq * (d + 5) + 3, d + 5, 1), 1)
        buf = torch.full((3000,), 5.0, dtype=io, device="cuda")
        out = buf.as_strided((3, nq, d), (d + 1, 3 * (d + 1), 1), 7)   # heads outermost
        table_wide = torch.full((3, 20), -1, dtype=torch.int32)
        table_wide[:, :table.shape[1]] = table
        t = table_wide.cuda()[:, :table.shape[1]]
        pool.attention(0, t, torch.tensor(lengths, dtype=torch.int32).cuda(), q, out,
                       pool.workspace(3))
        want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q.cpu(), page, d ** -0.5)
        check_attention(out, None, want)
        mark = torch.zeros(3000, dtype=torch.bool)
        mark.as_strided((3, nq, d), (d + 1, 3 * (d + 1), 1), 7).fill_(True)
        assert bool((buf.cpu()[~mark] == 5.0).all())


def test_offsets_past_32_bits():
    # K and V of 5 GiB each: pages at both ends
    kv, page, d = 8, 64, 128
    n_pages = 5 * 2 ** 30 // (kv * page * d * 2)
    pool = PagedKvCache.from_tensors(*(torch.empty(1, n_pages, kv, page, d, dtype=BF16, device="cuda")
                                       for _ in range(2)))
    g = gen(30)
    n = 300
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, n_pages // 2, n_pages - 3]], dtype=torch.int32)
    rows = [torch.randn(n, kv, d, generator=g).to(BF16) for _ in range(2)]
    pos = torch.arange(n, dtype=torch.int32).cuda()
    seq = torch.zeros_like(pos)
    pool.append(0, table.cuda(), pos, rows[0].cuda(), rows[1].cuda(), seq=seq)
    back = [torch.empty(n, kv, d, dtype=BF16, device="cuda") for _ in range(2)]
    pool.read(0, table.cuda(), pos, back[0], back[1], seq=seq)
    assert torch.equal(back[0].cpu(), rows[0]) and torch.equal(back[1].cpu(), rows[1])
    q = torch.randn(1, 32, d, generator=g)
    small = torch.zeros(2, 1, 5, kv, page, d, dtype=torch.float64)
    for i in range(2):
        full = torch.zeros(5 * page, kv, d, dtype=torch.float64)
        full[:n] = rows[i].double()
        small[i, 0] = full.view(5, page, kv, d).transpose(1, 2)
    want = attention64(small[0], small[1], torch.arange(5).view(1, 5), [n], q, page, d ** -0.5)
    out, lse = run_attention(pool, table, [n], q, page)
    check_attention(out, lse, want)
    assert pool.device_error() == 0


def test_attention_is_deterministic_and_leaves_its_workspace_ready():
    g = gen(31)
    page = 16
    pool = make_pool(1, 700, 8, page, 128, E4M3, g)
    many = [(37 * i) % 300 + 1 for i in range(40)]
    few = [9000]
    ws = pool.workspace(40)
    ref = {}
    for turn in range(3):
        for name, lengths, nq in (("many", many, 32), ("few", few, 64), ("many8", many, 8)):
            table = make_table(lengths, page, 700, gen(5))
            q = torch.randn(len(lengths), nq, 128, generator=gen(6))
            out, lse = run_attention(pool, table, lengths, q, page, ws=ws)
            got = (out.cpu(), lse.cpu())
            if turn == 0:
                ref[name] = got
                want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, page,
                                   128 ** -0.5)
                check_attention(out, lse, want, name)
            assert torch.equal(got[0], ref[name][0]) and torch.equal(got[1], ref[name][1])


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("io", [BF16, FP32])
def test_prompt_then_decode_then_read(cache, io):
    """Prompts go in together, then tokens one by one across page borders, each
    attending over what is cached so far; at the end everything is read back."""
    g = gen(40)
    page, kv, nq, d, B = 8, 2, 8, 128, 3
    prompts, steps = [13, 1, 30], 11
    total = [n + steps for n in prompts]
    pool = make_pool(1, 40, kv, page, d, cache, g)
    table = make_table(total, page, 40, g)
    rows = [[torch.randn(n, kv, d, generator=g).to(io) for n in total] for _ in range(2)]
    pos = torch.cat([torch.arange(n) for n in prompts]).to(torch.int32).cuda()
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(prompts)]).to(torch.int32).cuda()
    first = [torch.cat([r[b][:prompts[b]] for b in range(B)]).cuda() for r in rows]
    pool.append(0, table.cuda(), pos, first[0], first[1], seq=seq)
    ws = pool.workspace(B)
    for s in range(steps):
        at = torch.tensor([n + s for n in prompts], dtype=torch.int32)
        new = [torch.stack([r[b][prompts[b] + s] for b in range(B)]).cuda() for r in rows]
        pool.append(0, table.cuda(), at.cuda(), new[0], new[1])
        q = torch.randn(B, nq, d, generator=g).to(io)
        lengths = (at + 1).tolist()
        out, lse = run_attention(pool, table, lengths, q, page, ws=ws)
        want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, page, d ** -0.5)
        check_attention(out, lse, want, f"step {s}")
    pos = torch.cat([torch.arange(n) for n in total]).to(torch.int32).cuda()
    seq = torch.cat([torch.full((n,), b) for b, n in enumerate(total)]).to(torch.int32).cuda()
    back = [torch.empty(sum(total), kv, d, device="cuda") for _ in range(2)]
    pool.read(0, table.cuda(), pos, back[0], back[1], seq=seq)
    for got, r in zip(back, rows):
        x = torch.cat(r)
        if cache == BF16:
            assert torch.equal(got.cpu(), x.float().to(BF16).float())
        else:
            codes, scale = e4m3_rows(x)
            want = codes.view(E4M3).float() * torch.exp2(scale.float() - 127)[..., None]
            assert torch.equal(got.cpu(), want)
    assert pool.device_error() == 0


def test_graph_replays_beside_eager_calls():
    """append and attention captured together; replays between eager calls on
    the same pool, each checked, and two graphs side by side on two streams."""
    g = gen(41)
    page, kv, nq, d, B = 16, 8, 32, 128, 4
    pool = make_pool(1, 200, kv, page, d, E4M3, g)
    lengths = [600, 33, 0, 250]
    table = make_table([n + 10 for n in lengths], page, 200, g)
    t = table.cuda()
    stat = dict(pos=torch.zeros(B, dtype=torch.int32).cuda(), n=torch.zeros(B, dtype=torch.int32).cuda(),
                k=torch.empty(B, kv, d, device="cuda"), v=torch.empty(B, kv, d, device="cuda"),
                q=torch.empty(B, nq, d, device="cuda"))
    outs = [torch.empty(B, nq, d, device="cuda") for _ in range(2)]
    spaces = [pool.workspace(B) for _ in range(3)]

    def fill(s):
        at = torch.tensor([n + s if n else -1 for n in lengths], dtype=torch.int32)
        stat["pos"].copy_(at)
        stat["n"].copy_(at + 1)
        for name in ("k", "v", "q"):
            stat[name].copy_(torch.randn(stat[name].shape, generator=gen(100 + s)))
        return (at + 1).tolist()

    def body(i, stream):
        if i == 0:
            pool.append(0, t, stat["pos"], stat["k"], stat["v"], stream=stream)
        pool.attention(0, t, stat["n"], stat["q"], outs[i], spaces[i], stream=stream)

    fill(0)
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            body(i, streams[i])
    for s in range(5):
        n = fill(s)
        torch.cuda.synchronize()
        graphs[0].replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(outs[0])
        pool.attention(0, t, stat["n"], stat["q"], eager, spaces[2])
        torch.cuda.synchronize()
        want = attention64(values(pool, "k"), values(pool, "v"), table, n, stat["q"].cpu(), page,
                           d ** -0.5)
        check_attention(outs[0], None, want, f"replay {s}")
        assert torch.equal(eager, outs[0])
        # both graphs at once, each with its own workspace
        outs[0].zero_()
        outs[1].zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], eager) and torch.equal(outs[1], eager)
    assert pool.device_error() == 0


def test_a_stream_of_the_caller():
    g = gen(42)
    pool = make_pool(1, 30, 2, 16, 64, BF16, g)
    table = make_table([200], 16, 30, g).cuda()
    q = torch.randn(1, 4, 64, generator=g).cuda()
    n = torch.tensor([200], dtype=torch.int32).cuda()
    ws, a, b = pool.workspace(1), torch.zeros(1, 4, 64, device="cuda"), torch.zeros(1, 4, 64, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    pool.attention(0, table, n, q, a, ws, stream=s)
    s.synchronize()
    pool.attention(0, table, n, q, b, ws)
    assert torch.equal(a, b)


def test_device_error_sees_calls_of_other_streams():
    pool = make_pool(1, 4, 2, 16, 64, BF16, gen(44))
    table = torch.tensor([[0, 9]], dtype=torch.int32).cuda()   # (no page 9)
    pos = torch.tensor([20], dtype=torch.int32).cuda()
    row = torch.zeros(1, 2, 64, device="cuda")
    side, work = torch.cuda.Stream(), torch.zeros(2048, 2048, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(40):
                work @ work
        pool.append(0, table, pos, row, row, stream=side)
        assert pool.device_error() == kb.KL_DEVERR_PAGE
        assert pool.device_error() == 0


def test_a_pool_and_its_workspace_are_ready_for_any_stream():
    # made while the current stream is busy, used at once on another
    g = gen(45)
    n, q = torch.tensor([900], dtype=torch.int32).cuda(), torch.randn(1, 16, 128, generator=g).cuda()
    base = make_pool(1, 60, 2, 16, 128, E4M3, g)
    table = make_table([900], 16, 60, g).cuda()
    want, out = torch.empty_like(q), torch.empty_like(q)
    base.attention(0, table, n, q, want, base.workspace(1))
    side, work = torch.cuda.Stream(), torch.zeros(2048, 2048, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        out.fill_(5.0)
        torch.cuda.synchronize()
        for _ in range(40):
            work @ work
        pool = PagedKvCache.from_tensors(base.k, base.v, base.k_scale, base.v_scale)
        pool.attention(0, table, n, q, out, pool.workspace(1), stream=side)
        side.synchronize()
        assert torch.equal(out, want)
        assert pool.device_error() == 0


def test_a_workspace_made_in_a_capture():
    g = gen(46)
    pool = make_pool(1, 60, 2, 16, 128, BF16, g)
    table = make_table([900], 16, 60, g).cuda()
    n, q = torch.tensor([900], dtype=torch.int32).cuda(), torch.randn(1, 16, 128, generator=g).cuda()
    want, out = torch.empty_like(q), torch.empty_like(q)
    pool.attention(0, table, n, q, want, pool.workspace(1))
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        pool.attention(0, table, n, q, out, pool.workspace(1), stream=stream)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_the_contiguous_cache_and_pages():
    """A sequence goes from a contiguous cache into pages and back, bit for bit."""
    g = gen(43)
    cfg = dict(n_layers=2, n_kv_heads=3, head_dim=64)
    kv = KvCache(cfg, 2, 128)
    for x in (kv.k, kv.v):
        x.copy_(torch.randn(x.shape, generator=g).to(BF16).view(torch.int16))
    pool = PagedKvCache(cfg, 12, 16)
    n = 101
    table = make_table([n], 16, 12, g).cuda()
    pos = torch.arange(n, dtype=torch.int32).cuda()
    seq = torch.zeros_like(pos)
    other = KvCache(cfg, 2, 128)
    for l in range(2):
        rows = [x[l, 1].view(BF16).transpose(0, 1)[:n] for x in (kv.k, kv.v)]
        pool.append(l, table, pos, rows[0], rows[1], seq=seq)
        back = [x[l, 0].view(BF16).transpose(0, 1)[:n] for x in (other.k, other.v)]
        pool.read(l, table, pos, back[0], back[1], seq=seq)
    for a, b in ((kv.k, other.k), (kv.v, other.v)):
        assert torch.equal(a[:, 1, :, :n], b[:, 0, :, :n])
        assert not b[:, 1].any() and not b[:, 0, :, n:].any()


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("window", [0, 19])
def test_more_sequences_than_a_wave_has_lanes(cache, window):
    # lengths of all kinds, empty and bad ones among them, bad pages of one
    g = gen(50)
    page, kv, nq, d, B = 8, 3, 12, 64, 150
    lengths = [(53 * i * i) % 97 if i % 9 else 0 for i in range(B)]
    n_pages = sum(-(-n // page) for n in lengths)
    pool = make_pool(1, n_pages, kv, page, d, cache, g)
    table = make_table(lengths, page, n_pages, g, extra=0)
    q = torch.randn(B, nq, d, generator=g)
    want = attention64(values(pool, "k"), values(pool, "v"), table, lengths, q, page, d ** -0.5, window)
    ws = pool.workspace(B)
    out, lse = run_attention(pool, table, lengths, q, page, window=window, ws=ws)
    check_attention(out, lse, want)
    assert pool.device_error() == 0
    lens, bad = list(lengths), table.clone()
    lens[70] = -1
    lens[149] = table.shape[1] * page + 1
    victim = max(range(71, 149), key=lambda b: lengths[b])
    bad[victim, (lengths[victim] - 1) // page] = n_pages
    out, lse = run_attention(pool, bad, lens, q, page, window=window, ws=ws)
    assert pool.device_error() == kb.KL_DEVERR_PAGE | kb.KL_DEVERR_POSITION
    keep = torch.tensor([b for b in range(B) if b not in (70, 149, victim)])
    assert torch.isnan(out[[70, 149, victim]]).all() and torch.isnan(lse[[70, 149, victim]]).all()
    check_attention(out[keep.cuda()], lse[keep.cuda()], [w[keep] for w in want])


def test_the_largest_batch_and_group():
    g = gen(51)
    page, kv, nq, d, B = 16, 1, 16, 128, 4096
    lengths = [(i * 7) % 33 for i in range(B)]
    pool = make_pool(1, 400, kv, page, d, E4M3, g)
    table = torch.randint(0, 400, (B, 3), generator=g).to(torch.int32)   # (pages shared by many)
    q = torch.randn(B, nq, d, generator=g).to(BF16)
    out, lse = run_attention(pool, table, lengths, q, page)
    pick = torch.cat([torch.arange(40), torch.randint(0, B, (60,), generator=g), torch.arange(B - 40, B)])
    want = attention64(values(pool, "k"), values(pool, "v"), table[pick],
                       [lengths[int(i)] for i in pick], q[pick], page, d ** -0.5)
    check_attention(out[pick.cuda()], lse[pick.cuda()], want)
    assert torch.isfinite(out).all() and pool.device_error() == 0


def test_sequences_that_share_their_pages_agree():
    g = gen(52)
    page, kv, d = 32, 2, 128
    pool = make_pool(1, 40, kv, page, d, E4M3, g)
    one = make_table([1000], page, 40, g)
    q = torch.randn(1, 8, d, generator=g)
    a, la = run_attention(pool, one.expand(5, -1).contiguous(), [1000, 17, 1000, 0, 1000],
                          q.expand(5, -1, -1).contiguous(), page)
    want = attention64(values(pool, "k"), values(pool, "v"), one, [1000], q, page, d ** -0.5)
    for b in (0, 2, 4):
        check_attention(a[b:b + 1], la[b:b + 1], want)
    # one query for all of them, by a row stride of zero
    b_, lb = run_attention(pool, one.expand(5, -1).contiguous(), [1000, 17, 1000, 0, 1000],
                           q.cuda().expand(5, -1, -1), page)
    assert torch.equal(a, b_) and torch.equal(la, lb)


def test_two_streams_append_and_attend_at_once():
    """Rows of some sequences are written while others are attended over."""
    g = gen(53)
    page, kv, nq, d = 16, 4, 16, 128
    pool = make_pool(1, 600, kv, page, d, E4M3, g)
    table = make_table([4000, 3000], page, 600, g).cuda()
    q = torch.randn(2, nq, d, generator=g).cuda()
    n = torch.tensor([4000, 0], dtype=torch.int32).cuda()
    outs = [torch.empty(2, nq, d, device="cuda") for _ in range(2)]
    wss = [pool.workspace(2) for _ in range(2)]
    rows = torch.randn(3000, kv, d, generator=g).to(BF16).cuda()
    pos = torch.arange(3000, dtype=torch.int32).cuda()
    seq = torch.ones_like(pos)
    pool.attention(0, table, n, q, outs[0], wss[0])
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        pool.append(0, table, pos, rows, rows, seq=seq, stream=s1)
        pool.attention(0, table, n, q, outs[1], wss[1], stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    back = [torch.empty(3000, kv, d, device="cuda") for _ in range(2)]
    pool.read(0, table, pos, back[0], back[1], seq=seq)
    codes, scale = e4m3_rows(rows)
    want = codes.view(E4M3).float() * torch.exp2(scale.float() - 127)[..., None]
    assert torch.equal(back[0].cpu(), want) and torch.equal(back[1].cpu(), want)


def test_wrong_device_index_is_refused():
    pool = make_pool(1, 2, 1, 8, 64, BF16, gen(1))
    pool.c.device = 1
    x = torch.zeros(1, 1, 64, device="cuda")
    t = torch.zeros(1, 1, dtype=torch.int32).cuda()
    with pytest.raises(kb.KlError) as e:
        pool.append(0, t, torch.zeros(1, dtype=torch.int32).cuda(), x, x)
    assert e.value.status == kb.KL_ERR_INVALID_ARGUMENT and "device" in str(e.value)
    assert half_step(BF16) == 2.0 ** -8
