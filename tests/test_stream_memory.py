"""Calls that are given a stream and no memory for their results: what they allocate comes from that stream's pool, not from the
current stream's, whose queued kernels may still be at work on what its pool hands out."""
import contextlib
import types

import pytest
import torch

from paper_2409_15104_amd import binding as pec

S = types.SimpleNamespace(cuda_stream=0x51)
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Library:
    """Every entry point succeeds and does nothing; sizes are 0."""

    def __getattr__(self, name):
        return lambda *args: 0


@pytest.fixture
def world(monkeypatch):
    """The binding on CPU tensors that pass for GPU ones.  Collects (shape, stream) of every allocation and the streams that
    tensors are held for."""
    seen = types.SimpleNamespace(allocated=[], held=[], now=None)
    make = torch.empty

    @contextlib.contextmanager
    def on(stream):
        before, seen.now = seen.now, stream
        yield
        seen.now = before

    def empty(*args, device=None, **kw):
        t = make(*args, **kw)
        seen.allocated.append((tuple(t.shape), seen.now))
        return t

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: seen.held.append((tuple(t.shape), s)), raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(pec, "_require", lambda t, dtype, name: None)
    monkeypatch.setattr(pec, "_current_stream", lambda: 0)
    monkeypatch.setattr(pec, "_call", lambda fn, name, index, stream, *args: None)
    monkeypatch.setattr(pec, "lib", Library)
    return seen


def rows(n, heads):
    return torch.zeros(n, heads, 128, dtype=BF16)


CACHE = types.SimpleNamespace(index=0, n_kv_heads=2, ref=None)
TURN = types.SimpleNamespace(index=None, ref=None)
META = (torch.zeros(3, 2, dtype=I32), torch.zeros(4, dtype=I32), torch.zeros(3, dtype=I32))
PAGED = {
    "pec_qk_norm_rope": lambda **kw: pec.pec_qk_norm_rope(rows(5, 4), rows(5, 2), TURN, **kw),
    "pec_paged_append": lambda **kw: pec.pec_paged_append(rows(5, 2), rows(5, 2), CACHE, *META, q=rows(5, 4), **kw),
    "pec_attn_paged": lambda **kw: pec.pec_attn_paged(rows(5, 4), CACHE, *META, **kw),
}
CU = torch.zeros(4, dtype=I32)
IN_A_ROW = {
    "pec_attn_chunk": lambda **kw: pec.pec_attn_chunk(rows(5, 4), rows(9, 2), rows(9, 2), 4, 0, **kw),
    "pec_finalize": lambda **kw: pec.pec_finalize(rows(5, 4), **kw),
    "pec_sp_prefill": lambda **kw: pec.pec_sp_prefill(rows(5, 4), rows(9, 2), rows(9, 2), 0, 5, flags=pec.PEC_FLAG_SP_STEP_LAUNCHES, **kw),
    "pec_decode_splitkv": lambda **kw: pec.pec_decode_splitkv(rows(1, 4), rows(9, 2), rows(9, 2), **kw),
    "pec_ulysses_layout": lambda **kw: pec.pec_ulysses_layout(rows(4, 4), 2, True, **kw),
    "pec_attn_colocated": lambda **kw: pec.pec_attn_colocated(rows(5, 4), rows(9, 2), rows(9, 2), CU, CU, **kw),
    "pec_attn_varlen": lambda **kw: pec.pec_attn_varlen(rows(5, 4), rows(5, 2), rows(5, 2), CU, 5, **kw),
}
CALLS = {**PAGED, **IN_A_ROW}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_is_its_streams(world, name):
    CALLS[name](stream=S)
    assert world.allocated and all(stream is S for _, stream in world.allocated)
    # results are held for the stream that they are read on, a workspace (16 bytes: its size is 0 here) for no other
    assert world.held == [(shape, "current") for shape, _ in world.allocated if shape != (16,)]
    n = len(world.allocated)
    CALLS[name]()
    assert len(world.allocated) == 2 * n and all(stream is None for _, stream in world.allocated[n:])
