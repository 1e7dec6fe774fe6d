"""PagedKvCache's and GpuModel's own part of a call, with the library and the GPU stubbed (CPU only)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2410_23668_amd import binding as kb
from paper_2410_23668_amd.device import GpuModel, PagedKvCache


def bare_pool():
    """A pool without memory of its own."""
    pool = PagedKvCache.__new__(PagedKvCache)
    pool.device = torch.device("cuda", 0)
    pool.error = torch.zeros(1, dtype=torch.int32)
    return pool


def test_device_error_waits_for_every_stream(monkeypatch):
    # a call that is still running when device_error() is called reports as it ends
    pool, seen = bare_pool(), []

    def synchronize(device=None):
        seen.append((device, int(pool.error)))
        if len(seen) == 1:
            pool.error |= kb.KL_DEVERR_PAGE

    monkeypatch.setattr(torch.cuda, "synchronize", synchronize)
    assert pool.device_error() == kb.KL_DEVERR_PAGE
    # (and once more behind the clearing, so that no later call's bits go with it)
    assert seen == [(pool.device, 0), (pool.device, 0)] and int(pool.error) == 0
    assert pool.device_error() == 0 and len(seen) == 3


@pytest.mark.parametrize("capturing", [False, True])
def test_a_workspace_is_filled_before_it_is_handed_out(monkeypatch, capturing):
    pool, order = bare_pool(), []

    class Stream:
        def synchronize(self):
            order.append("wait")

    def zeros(*a, **k):
        order.append("fill")
        return "workspace"

    monkeypatch.setattr(kb, "kl_paged_attention_workspace", lambda c, batch: 64 * batch)
    monkeypatch.setattr(torch, "zeros", zeros)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream())
    pool.c = None
    assert pool.workspace(3) == "workspace"
    assert order == (["fill"] if capturing else ["fill", "wait"])


B, VOCAB, HIDDEN = 3, 7, 5
INT = torch.int32
GOOD = dict(tokens=torch.zeros(B, dtype=INT), positions=torch.zeros(B, dtype=INT),
            logits=torch.zeros(B, VOCAB), hidden=torch.zeros(B, HIDDEN),
            tokens_out=torch.zeros(4, B, dtype=INT))


def call(monkeypatch, method, **over):
    """The library calls that a GpuModel method makes of these tensors (the cache is on the CPU)."""
    made = []
    for name in ("kl_decode_step", "kl_decode_step_paged", "kl_decode_greedy"):
        monkeypatch.setattr(kb, name, lambda *a, name=name: made.append(name))
    model = GpuModel.__new__(GpuModel)
    model.state, model.model_cfg = None, dict(vocab=VOCAB, hidden=HIDDEN)
    a, stream = dict(GOOD, **over), SimpleNamespace(cuda_stream=0)
    x = torch.zeros(1)
    kv = SimpleNamespace(k=x, v=x, batch=B, capacity=8)
    if method == "step":
        model.step(a["tokens"], a["positions"], kv, a["logits"], a["hidden"], 1, stream)
    elif method == "step_paged":
        pool = SimpleNamespace(c=None, device=x.device, _table=lambda t: t)
        model.step_paged(a["tokens"], a["positions"], pool, None, a["logits"], a["hidden"], stream)
    else:
        model.greedy(a["tokens"], a["positions"], kv, 4, a["tokens_out"], a["logits"], 1, stream)
    return made


METHODS = {"step": "kl_decode_step", "step_paged": "kl_decode_step_paged", "greedy": "kl_decode_greedy"}
BAD = dict(short_positions=dict(positions=torch.zeros(B - 1, dtype=INT)),
           long_positions=dict(positions=torch.zeros(B + 1, dtype=INT)),
           strided_positions=dict(positions=torch.zeros(2 * B, dtype=INT)[::2]),
           strided_tokens=dict(tokens=torch.zeros(2 * B, dtype=INT)[::2]),
           strided_logits=dict(logits=torch.zeros(VOCAB, B).t()),
           other_device_tokens=dict(tokens=torch.zeros(B, dtype=INT, device="meta")),
           other_device_positions=dict(positions=torch.zeros(B, dtype=INT, device="meta")),
           other_device_logits=dict(logits=torch.zeros(B, VOCAB, device="meta")))
BAD_HIDDEN = dict(strided=torch.zeros(HIDDEN, B).t(), device=torch.zeros(B, HIDDEN, device="meta"))
BAD_OUT = dict(strided=torch.zeros(B, 4, dtype=INT).t(), device=torch.zeros(4, B, dtype=INT, device="meta"))


@pytest.mark.parametrize("method", METHODS)
@pytest.mark.parametrize("bad", BAD)
def test_steps_refuse_tensors_that_the_library_would_misread(monkeypatch, method, bad):
    with pytest.raises(AssertionError):
        call(monkeypatch, method, **BAD[bad])
    assert call(monkeypatch, method) == [METHODS[method]]


@pytest.mark.parametrize("method", ["step", "step_paged"])
@pytest.mark.parametrize("bad", BAD_HIDDEN)
def test_steps_refuse_hidden_outputs_that_the_library_would_miswrite(monkeypatch, method, bad):
    with pytest.raises(AssertionError):
        call(monkeypatch, method, hidden=BAD_HIDDEN[bad])
    assert call(monkeypatch, method, hidden=None) == [METHODS[method]]


@pytest.mark.parametrize("bad", BAD_OUT)
def test_the_token_loop_refuses_outputs_that_the_library_would_miswrite(monkeypatch, bad):
    with pytest.raises(AssertionError):
        call(monkeypatch, "greedy", tokens_out=BAD_OUT[bad])
