"""kl_decode_step_paged: a step over pages against the CPU oracle (the decode
step's own tolerances) and against the step over the contiguous cache."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_23668_amd import binding as kb
from paper_2410_23668_amd.device import KvCache, PagedKvCache
from synth.workloads import TINY
from tests.gpu_cases import (REL_L2_TOL, Case, assert_bit_exact, check_against_oracle,
                             check_vectors, say)
from tests.paged_cases import BF16, E4M3, e4m3_rows, make_table

pytestmark = pytest.mark.gpu


def rows_of(kv, l, b, n):
    return [x[l, b].view(BF16).transpose(0, 1)[:n] for x in (kv.k, kv.v)]


def to_pages(case, page, dtype, seed=1):
    """The case's filled positions in a pool, and the table (room for the capacity)."""
    B, cap, cfg = case.batch, case.capacity, case.cfg
    g = torch.Generator().manual_seed(seed)
    need = B * (-(-cap // page))
    pool = PagedKvCache(cfg, need + 3, page, dtype)
    table = make_table([cap] * B, page, need + 3, g, extra=0).cuda()
    kv = KvCache(cfg, B, cap, k_host=case.K0, v_host=case.V0)
    for l in range(cfg["n_layers"]):
        for b in range(B):
            n = cap   # (the zeros behind the filled positions too: what must stay)
            pos = torch.arange(n, dtype=torch.int32).cuda()
            k, v = rows_of(kv, l, b, n)
            pool.append(l, table, pos, k, v, seq=torch.full_like(pos, b))
    return pool, table


def from_pages(case, pool, table):
    kv = KvCache(case.cfg, case.batch, case.capacity)
    for l in range(case.cfg["n_layers"]):
        for b in range(case.batch):
            pos = torch.arange(case.capacity, dtype=torch.int32).cuda()
            k, v = rows_of(kv, l, b, case.capacity)
            pool.read(l, table, pos, k, v, seq=torch.full_like(pos, b))
    assert pool.device_error() == 0
    return kv


def paged_step(case, pool, table, tokens=None, positions=None):
    B = case.batch
    toks = torch.from_numpy(case.tokens if tokens is None else np.asarray(tokens, np.int32)).cuda()
    pos = torch.from_numpy(case.positions if positions is None else
                           np.asarray(positions, np.int32)).cuda()
    logits = torch.full((B, case.cfg["vocab"]), 7.0, device="cuda")
    hidden = torch.full((B, case.cfg["hidden"]), 7.0, device="cuda")
    case.model.step_paged(toks, pos, pool, table, logits, hidden)
    torch.cuda.synchronize()
    return logits.cpu().numpy(), hidden.cpu().numpy()


D128 = dict(n_layers=2, hidden=512, n_heads=8, n_kv_heads=2, head_dim=128, ffn_dim=768, vocab=999,
            rope_theta=10000.0, rms_eps=1e-5)
THREE = dict(D128, n_heads=6, qkv_bias=True)
EIGHT = dict(D128, n_heads=16)
MHA = dict(TINY, n_layers=2, n_kv_heads=4)


@pytest.mark.parametrize("model,filled,page", [
    (TINY, [128], 16),
    (TINY, [0, 5, 63, 64, 130, 31], 8),
    (D128, [77, 0, 128], 64),
    (D128, [(37 * i) % 190 for i in range(33)], 32),
    (THREE, [100, 3, 180, 64, 1], 16),
    (EIGHT, [150, 20], 128),
    (MHA, [90] * 7, 16),
], ids=["tiny-b1", "tiny-b6", "d128-b3", "d128-b33", "three-b5", "eight-b2", "mha-b7"])
def test_matches_the_oracle(model, filled, page):
    say(f"[paged step] batch {len(filled)} page {page}")
    case = Case(model, len(filled), 192, filled, seed=31, max_batch=max(len(filled), 8), max_seq=256)
    pool, table = to_pages(case, page, BF16)
    lg, hd = paged_step(case, pool, table)
    kv = from_pages(case, pool, table)
    check_against_oracle(case, (lg, hd, *kv.host()), case.oracle_step())
    assert case.model.device_error() == 0
    # the same bits again, and an ordinary step of the same model in between
    a = case.gpu_step(kb.KL_MODE_LOOPED)
    lg2, hd2 = paged_step(case, pool, table)
    assert np.array_equal(lg, lg2) and np.array_equal(hd, hd2)
    assert_bit_exact(a, case.gpu_step(kb.KL_MODE_LOOPED), "ordinary step around a paged one")


def test_skips_bad_sequences():
    filled = [40, 60, 80, 100, 20, 10]
    case = Case(TINY, 6, 128, filled, seed=33, max_batch=8)
    pool, table = to_pages(case, 16, BF16)
    bad = table.clone()
    bad[4, 1] = pool.c.n_pages      # (its position 20 is in page 1)
    bad[5, 1] = -9                  # (not read: its position 10 is in page 0)
    tokens, pos = case.tokens.copy(), case.positions.copy()
    tokens[1] = TINY["vocab"]
    pos[2], pos[3] = 128, -1
    got = paged_step(case, pool, bad, tokens, pos)
    assert case.model.device_error() == (kb.KL_DEVERR_TOKEN | kb.KL_DEVERR_POSITION |
                                         kb.KL_DEVERR_PAGE)
    case.tokens, case.positions = tokens, pos
    case.tokens[1], case.positions[2:4] = 0, [0, 0]   # (the oracle evaluates these too; not compared)
    ref = case.oracle_step(sample=[0, 5])
    kv = from_pages(case, pool, table)
    check_against_oracle(case, (*got, *kv.host()), ref, skip=(1, 2, 3, 4))
    # a bad page alone
    got = paged_step(case, pool, bad, tokens * 0, filled)
    assert case.model.device_error() == kb.KL_DEVERR_PAGE | kb.KL_DEVERR_POSITION
    assert np.isnan(got[0][4]).all() and np.isfinite(got[0][[0, 1, 2, 3, 5]]).all()


def test_8_bit_pool():
    filled = [128, 140, 190, 150, 133]
    case = Case(D128, 5, 192, filled, seed=35, max_batch=8)
    pool, table = to_pages(case, 16, E4M3)
    held = from_pages(case, pool, table)      # what the pool holds, exact in bf16
    case.K0, case.V0 = held.host()
    say("[paged step] e4m3")
    step = case.gpu_step(kb.KL_MODE_PER_OP)   # (matrix-core path at this batch)
    lg, hd = paged_step(case, pool, table)
    # the first layer's new rows do not depend on the cache: the contiguous
    # step's rows, quantised
    for b, p in enumerate(filled):
        pg = int(table[b, p // 16])
        for name, new in (("k", step[2]), ("v", step[3])):
            row = torch.from_numpy(oracle.bf16_to_f64(new[0, b, :, p]))
            codes, scale = e4m3_rows(row)
            assert torch.equal(getattr(pool, name).view(torch.uint8)[0, pg, :, p % 16].cpu(), codes)
            assert torch.equal(getattr(pool, name + "_scale")[0, pg, :, p % 16].cpu(), scale)
    # the outputs differ by the new rows' quantising alone: 2^-4 of one row of
    # more than 128, within the step's tolerance
    rl, rh, _, _ = case.oracle_step()
    errs = {f"logits[{b}]": oracle.rel_l2(lg[b], rl[b]) for b in range(5)}
    errs.update({f"hidden[{b}]": oracle.rel_l2(hd[b], rh[b]) for b in range(5)})
    check_vectors(errs, {})
    # and nothing else was written
    kv = from_pages(case, pool, table)
    for got, had in zip(kv.host(), (case.K0, case.V0)):
        for b, p in enumerate(filled):
            mask = np.arange(192) != p
            assert np.array_equal(got[:, b, :, mask], had[:, b, :, mask])
    assert case.model.device_error() == 0


def test_steps_across_pages_follow_the_contiguous_ones():
    filled = [13, 6, 30, 15, 7]
    case = Case(TINY, 5, 64, filled, seed=37, max_batch=8)
    pool, table = to_pages(case, 8, BF16)
    kv = KvCache(case.cfg, 5, 64, k_host=case.K0, v_host=case.V0)
    rng = np.random.RandomState(3)
    for s in range(6):
        tokens = rng.randint(0, TINY["vocab"], 5).astype(np.int32)
        pos = (np.asarray(filled) + s).astype(np.int32)
        lg, hd = paged_step(case, pool, table, tokens, pos)
        want = case.gpu_step(kb.KL_MODE_LOOPED, positions=pos, tokens=tokens, kv=kv)
        for b in range(5):
            assert oracle.rel_l2(lg[b], want[0][b]) <= REL_L2_TOL
            assert oracle.rel_l2(hd[b], want[1][b]) <= REL_L2_TOL
    got = from_pages(case, pool, table).host()
    for g, w in zip(got, kv.host()):
        for b, n in enumerate(filled):
            assert np.array_equal(g[:, b, :, n + 6:], w[:, b, :, n + 6:])
            a, r = (oracle.bf16_to_f64(x[:, b, :, n:n + 6]) for x in (g, w))
            assert oracle.rel_l2(a, r) <= REL_L2_TOL


def test_refusals():
    case = Case(TINY, 2, 64, [3, 4], seed=39, max_batch=8)
    pool, table = to_pages(case, 16, BF16)
    lg = torch.empty(2, TINY["vocab"], device="cuda")
    tok, pos = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))

    def call(model=case.model, pool=pool, table=table):
        with pytest.raises(kb.KlError) as e:
            model.step_paged(tok, pos, pool, table, lg)
        return e.value.status, str(e.value)

    other = PagedKvCache(dict(TINY, n_kv_heads=1), 4, 16)
    assert call(pool=other)[0] == kb.KL_ERR_INVALID_ARGUMENT
    assert call(pool=PagedKvCache(dict(TINY, n_layers=3), 4, 16))[0] == kb.KL_ERR_INVALID_ARGUMENT
    st, msg = call(table=table[:1])
    assert st == kb.KL_ERR_INVALID_ARGUMENT and "table batch 1" in msg
    small = Case(TINY, 2, 64, [3, 4], seed=39, max_batch=2)
    st, msg = call(model=small.model)
    assert st == kb.KL_ERR_UNSUPPORTED and "max_batch" in msg
    moe = dict(TINY, n_layers=1, n_experts=4, top_k=2, ffn_dim=256)
    moe_case = Case(moe, 2, 64, [3, 4], seed=41, max_batch=7)
    st, msg = call(model=moe_case.model, pool=PagedKvCache(moe, 8, 16))
    assert st == kb.KL_ERR_UNSUPPORTED
    assert kb.lib().kl_decode_step_paged(None, 16, 16, 1, pool.c, pool._table(table), 16, None,
                                         None) == kb.KL_ERR_INVALID_ARGUMENT


def test_room_for_more_tiles_than_32_bits_count_is_refused():
    cfg = dict(TINY, n_layers=1, n_heads=16, n_kv_heads=16)
    case = Case(cfg, 2, 64, [3, 4], seed=43, max_batch=4096, max_seq=2 ** 20)
    pool = PagedKvCache(cfg, 2, 4096)
    B = 4096
    table = torch.zeros(B, 256, dtype=torch.int32, device="cuda")
    tok, pos = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    lg = torch.empty(B, cfg["vocab"], device="cuda")
    with pytest.raises(kb.KlError) as e:
        case.model.step_paged(tok, pos, pool, table, lg)
    assert e.value.status == kb.KL_ERR_UNSUPPORTED and "2^35" in str(e.value)


def test_captured_steps_replay_between_eager_ones():
    # two graphs of one model (a bf16 and an 8-bit pool), replayed in turn, each replay
    # checked against the eager step's bits; inputs change in place
    case = Case(TINY, 6, 256, [0, 5, 63, 64, 130, 31], seed=44, max_batch=8)
    B, cfg = case.batch, case.cfg
    tok, pos = torch.from_numpy(case.tokens).cuda(), torch.from_numpy(case.positions).cuda()
    runs = []
    for dtype in (BF16, E4M3):
        pool, table = to_pages(case, 16, dtype)
        out = [torch.zeros(B, cfg["vocab"], device="cuda"), torch.zeros(B, cfg["hidden"], device="cuda")]
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            case.model.step_paged(tok, pos, pool, table, *out, stream=stream)
        runs.append((pool, table, out, graph))
    for i in range(4):
        for pool, table, out, graph in runs:
            tokens, at = (case.tokens + 3 * i) % cfg["vocab"], case.positions + i
            tok.copy_(torch.from_numpy(tokens))
            pos.copy_(torch.from_numpy(at))
            for o in out:
                o.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            got, k = [o.cpu().numpy() for o in out], pool.k.view(torch.uint8).clone()
            want = paged_step(case, pool, table, tokens, at)   # (writes the same rows again)
            assert_bit_exact(got, want, f"replay {i}")
            assert torch.equal(k, pool.k.view(torch.uint8))
        assert case.model.device_error() == 0
    # a replay reports and skips what an eager step would
    pool, table, out, graph = runs[0]
    table[2, 0] = -1
    graph.replay()
    torch.cuda.synchronize()
    assert case.model.device_error() == kb.KL_DEVERR_PAGE | kb.KL_DEVERR_POSITION
    assert bool(torch.isnan(out[0][2]).all()) and bool(torch.isfinite(out[0][3]).all())
