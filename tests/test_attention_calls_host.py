"""Calls beside the sparse decode that are refused before any launch (no GPU needed)."""
import pytest
import torch

import paper_2502_12216_amd as T
from paper_2502_12216_amd import _capi as C
from tests.test_attention_host import prompt, scored, shared, weights


@pytest.mark.parametrize("call", [prompt, weights, scored, shared])
@pytest.mark.parametrize("cap", [2.0 ** -121, 1e-40, 2.0 ** 121, 3e38])
def test_caps_that_leave_the_normal_numbers(call, cap):
    assert call(mod=C.ScoreMod(cap)) == 1
    assert b"cap" in C.lib().tactic_last_error()
    with pytest.raises(ValueError, match="cap"):
        T.ScoreMod(cap=cap)


@pytest.mark.parametrize("cap", [0.0, 2.0 ** -120, 1e-6, 50.0, 2.0 ** 120])
def test_caps_at_the_ends_of_their_range(cap):
    T.ScoreMod(cap=cap)
    assert scored(mod=C.ScoreMod(cap), n=1000) == 3  # the next check: the workspace


def test_a_workspace_that_is_not_one_piece_of_memory_is_not_used():
    """A view that repeats or skips bytes has as many elements as asked for, and less memory, or another one's between."""
    batch = T.RaggedBatch([900, 300], 8, 2, device="cpu")
    size = T.PromptAttention(batch, [20, 20]).workspace.numel()
    whole = torch.zeros(2 * size + 64, dtype=torch.uint8)
    assert T.PromptAttention(batch, [20, 20], workspace=whole).workspace is whole
    assert whole.data_ptr() % 16 == 0
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(size), whole[::2], whole[1:], whole[:size - 1], whole.float()):
        got = T.PromptAttention(batch, [20, 20], workspace=bad).workspace
        assert got is not bad and got.is_contiguous() and got.numel() == size and got.dtype is torch.uint8


KB = 1 << 30  # far apart: eight arrays of at most 1000 x 2 rows


def _evict(**at):
    """tactic_evict over arrays at made-up addresses (1000 rows in, 100 out, 2 KV heads); no refusal, no launch: not called so."""
    names = ("K", "V", "weights", "positions", "K_out", "V_out", "weights_out", "positions_out")
    p = {**{x: KB * (i + 1) for i, x in enumerate(names)}, **at}
    shape = C.KVShape(2, 8, 2, 128, 1000, 700, 0x1000, None)
    return C.lib().tactic_evict(p["K"], p["V"], C.ctypes.byref(shape), p["weights"], p["positions"], 0x1000, None, 5, 0x1000, 100,
                                60, p["K_out"], p["V_out"], p["weights_out"], p["positions_out"], 0x1000, 0x1000, 1 << 40, None)


@pytest.mark.parametrize("out,size", [("K_out", 100 * 2 * 256), ("V_out", 100 * 2 * 256), ("weights_out", 800), ("positions_out", 800)])
@pytest.mark.parametrize("other,other_size", [("K", 1000 * 2 * 256), ("V", 1000 * 2 * 256), ("weights", 8000), ("positions", 8000),
                                              ("K_out", 100 * 2 * 256), ("V_out", 100 * 2 * 256), ("weights_out", 800),
                                              ("positions_out", 800)])
def test_evict_refuses_outputs_that_overlap(out, size, other, other_size):
    """Workgroups write rows while others still read theirs, so that one byte in common is too much."""
    if out == other:
        return
    at = KB * 100
    for off in (0, 256, other_size - 16, 16 - size):
        assert _evict(**{other: at, out: at + off}) == 1, off
        assert b"overlap" in C.lib().tactic_last_error()


def _pages(**other):
    """A cache of 3 pages of 16 tokens with other parts in place of its own (host memory: no call gets as far as a launch)."""
    c = object.__new__(T.PagedCache)
    c.num_pages, c.page_size, c.max_pages, c.perm = 3, 16, 2, None
    c.K_pages, c.V_pages = (torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16) for _ in range(2))
    c.page_table = torch.zeros(2, 2, dtype=torch.int32)
    for part, x in other.items():
        setattr(c, part, x)
    return c


@pytest.mark.parametrize("part", ["K_pages", "V_pages"])
@pytest.mark.parametrize("bad,error,match", [
    (torch.zeros(3, 2, 16, 128, dtype=torch.float16), TypeError, "bfloat16"),
    (torch.zeros(3, 2, 16, 128, dtype=torch.uint8), TypeError, "bfloat16"),  # half the memory that is read
    (torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16), ValueError, "must be"),  # fewer pages than the table may name
    (torch.zeros(3, 2, 8, 128, dtype=torch.bfloat16), ValueError, "must be"),
    (torch.zeros(3, 1, 16, 128, dtype=torch.bfloat16), ValueError, "must be"),
])
def test_pages_that_were_replaced(part, bad, error, match, monkeypatch):
    """Parts of a paged cache are checked at the call, for every paged form."""
    _paged_calls_refuse(monkeypatch, {part: bad}, error, match)


@pytest.mark.parametrize("bad,error,match", [(torch.zeros(2, 2, dtype=torch.int64), TypeError, "int32"),
                                             (torch.zeros(2, 1, dtype=torch.int32), ValueError, "must be"),
                                             (torch.zeros(1, 2, dtype=torch.int32), ValueError, "must be")])
def test_page_tables_that_were_replaced(bad, error, match, monkeypatch):
    _paged_calls_refuse(monkeypatch, dict(page_table=bad), error, match)


def _paged_calls_refuse(monkeypatch, part, error, match):
    batch = T.RaggedBatch([20, 30], 8, 2, device="cpu")
    # (tensors of the host stand in for the device's: only the place is let pass)
    from paper_2502_12216_amd import attention as A
    place = A._Call.tensor

    def on_host(self, t, name, dtype, shape=None, optional=False):
        try:
            return place(self, t, name, dtype, shape, optional)
        except ValueError as e:
            if "must live on the GPU" not in str(e):
                raise
    monkeypatch.setattr(A._Call, "tensor", on_host)
    monkeypatch.setattr(A._Call, "run", lambda self, name, *args: pytest.fail(f"{name} was not refused"))
    q, prompt_q = torch.zeros(2, 8, 128, dtype=torch.bfloat16), torch.zeros(50, 8, 128, dtype=torch.bfloat16)
    shared_dec = T.SharedPrefixDecoder(batch, [20, 25], [0, 1])
    for call in (lambda c: T.PromptAttention(batch, [20, 30]).paged(prompt_q, c), lambda c: T.ScoredDecoder(batch).paged(q, c),
                 lambda c: shared_dec.paged(q, c, _pages()), lambda c: shared_dec.paged(q, _pages(), c)):
        with pytest.raises(error, match=match):
            call(_pages(**part))


def test_append_that_is_refused_leaves_the_positions():
    """Tokens off their 16-byte alignment, or that the insertion refuses for whatever reason."""
    c = T.EvictingCache(8, 2, 2, 16, recent=4, device="cpu")
    k = torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    off = torch.zeros(2 * 2 * 128 + 1, dtype=torch.bfloat16)[1:].view(2, 2, 128)
    assert off.is_contiguous() and off.data_ptr() % 16
    for bad in ((off, k), (k, off), (k, k)):  # (the last: host memory)
        with pytest.raises((ValueError, C.TacticError)):
            c.append(*bad)
        assert c.newest.tolist() == [-1, -1] and c.batch.seq_lens == [0, 0]


@pytest.mark.parametrize("n", [1 << 30, (1 << 31) - 1])  # (times two KV heads: 2^31 or more)
def test_shared_prefixes_of_more_workgroups_than_a_launch_has(n):
    pre = C.Prefixes(n, 2, 500, 300, 0x1000, 0x1000, 0x1000, 0x1000, 2)
    assert shared(pre=pre) == 2
    assert b"workgroups" in C.lib().tactic_last_error()


def test_a_stream_of_another_device_is_refused(monkeypatch):
    from types import SimpleNamespace

    from paper_2502_12216_amd import attention as A
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    call = A._Call(here, SimpleNamespace(device=there, cuda_stream=0))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="stream"):
        call.run("tactic_last_error")


def test_evicting_cache_stays_on_the_device_it_was_made_on():
    """Not on whichever is current at a later prefill ("cuda" names that one)."""
    c = T.EvictingCache(8, 2, 2, 16, recent=4, device="cpu")
    assert isinstance(c.device, torch.device) and c.device == c.K.device
