"""PagedKvCache's and GpuModel's own part of a call, with the library and the GPU stubbed (CPU only)."""
import pytest
import torch

from paper_2410_23668_amd import binding as kb
from paper_2410_23668_amd.device import PagedKvCache


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
