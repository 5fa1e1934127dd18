"""The binding's own checks of prompt, score and page calls, on stand-ins for device tensors (nothing is launched)."""
from __future__ import annotations

import contextlib
import weakref

import pytest
import torch

from paper_2607_27269_gb300 import abi

F32, BF16, F16, I32, I64 = torch.float32, torch.bfloat16, torch.float16, torch.int32, torch.int64
GPU = torch.device("cuda", 0)


class Fake:
    """What the binding asks of a tensor on a GPU."""
    is_cuda = True

    def __init__(self, *shape, dtype=F32, device=GPU, strides=None, stream=None):
        self.shape, self.dtype, self.device, self.stream = torch.Size(shape), dtype, device, stream
        dense = [1]
        for n in reversed(shape[1:]):
            dense.insert(0, dense[0] * n)
        self._strides = tuple(dense[:len(shape)]) if strides is None else strides
        self._dense = strides is None

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def size(self, i):
        return self.shape[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return self._dense

    def data_ptr(self):
        return 0x10000

    def __getitem__(self, at):
        shape = (1, *self.shape) if at is None else (len(range(*at.indices(self.shape[0]))), *self.shape[1:])
        return Fake(*shape, dtype=self.dtype, device=self.device, stream=self.stream)


class Calls:
    """The library: every call is noted and succeeds."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            return abi.MLA_OK
        return call


@pytest.fixture
def calls(monkeypatch):
    """The library's calls; torch.empty makes stand-ins that know the stream on which they were allocated."""
    made, on = Calls(), ["current"]

    @contextlib.contextmanager
    def stream_of(s):
        on.append(s)
        yield
        on.pop()

    def empty(*shape, dtype=None, device=None):
        return Fake(*(shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape), dtype=dtype,
                    device=torch.device(device), stream=on[-1])

    monkeypatch.setattr(abi, "lib", lambda: made)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", stream_of)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, **kw: ("external", handle))
    monkeypatch.setattr(abi, "_stream", lambda s: 0 if s is None else s if isinstance(s, int) else s.cuda_stream)
    return made


@pytest.mark.parametrize("name,bad", [
    (name, bad) for name in ("logprob", "entropy", "lse")
    for bad in (Fake(3, dtype=BF16), Fake(3, dtype=F16), Fake(3, dtype=torch.float64), Fake(2), Fake(0), Fake(1),
                Fake(3, device=torch.device("cuda", 1)), Fake(3, 2))
] + [("top_index", bad) for bad in (Fake(3, 4, dtype=I32), Fake(2, 5, dtype=I32), Fake(14, dtype=I32), Fake(3, 5, dtype=I64),
                                    Fake(3, 5), Fake(5, 3, dtype=I32), Fake(3, 5, dtype=I32, strides=(8, 1)))]
  + [("top_logprob", bad) for bad in (Fake(3, 4), Fake(2, 5), Fake(3, 5, dtype=BF16), Fake(3, 6), Fake(3))])
def test_score_outputs_that_do_not_fit_are_refused(calls, name, bad):
    x, tokens = Fake(3, 100), Fake(3, dtype=I32)
    good = dict(logprob=Fake(3), entropy=Fake(3), lse=Fake(3), top_index=Fake(3, 5, dtype=I32), top_logprob=Fake(3, 5))
    abi.token_logprobs(x, tokens, 5, **good)
    assert len(calls.made) == 1
    with pytest.raises(ValueError):
        abi.token_logprobs(x, tokens, 5, **{**good, name: bad})
    assert len(calls.made) == 1  # (nothing was called)


def test_score_inputs_that_do_not_fit_are_refused(calls):
    for tokens in (Fake(2, dtype=I32), Fake(3, dtype=I64), Fake(3, dtype=I32, strides=(2,)),
                   Fake(3, dtype=I32, device=torch.device("cuda", 1))):
        with pytest.raises(ValueError):
            abi.token_logprobs(Fake(3, 100), tokens, 0)
    assert not calls.made


def test_score_outputs_with_room_to_spare_are_taken(calls):
    out = abi.token_logprobs(Fake(3, 100), Fake(3, dtype=I32), 5, Fake(4), Fake(3, 1), Fake(9, 5, dtype=I32), Fake(15))
    assert len(calls.made) == 1 and [t.numel() for t in out] == [4, 3, 45, 15]
    assert abi.token_logprobs(Fake(3, 100), None, 0, top_index=Fake(1, dtype=I32))[2].numel() == 1  # (not written)


def test_score_results_are_made_where_none_are_given(calls):
    out = abi.token_logprobs(Fake(3, 100, dtype=BF16), Fake(3, dtype=I32), 4)
    assert [tuple(t.shape) for t in out] == [(3,), (3,), (3, 4), (3, 4)]
    assert [t.dtype for t in out] == [F32, F32, I32, F32]
    assert abi.token_logprobs(Fake(3, 100), None)[0] is None


class Stream:
    cuda_stream = 77


@pytest.mark.parametrize("stream", [None, Stream(), 77])
def test_results_are_allocated_on_the_stream_that_writes_them(calls, monkeypatch, stream):
    """Memory of the current stream may still be in use by work queued there: what a call on another stream writes comes
    from that stream's memory."""
    want = "current" if stream is None else stream if isinstance(stream, Stream) else ("external", 77)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    x, rows = Fake(3, 100), Fake(3, 64, dtype=BF16)
    made = [*abi.token_logprobs(x, Fake(3, dtype=I32), 4, stream=stream), *abi.acceptance_stats(x, x, stream=stream),
            abi.e2e_loss(rows, rows, stream=stream)]
    assert len(made) == 9 and all(t.stream == want for t in made)
    given = abi.token_logprobs(x, None, 0, entropy=(e := Fake(3)), stream=stream)
    assert given[1] is e


def handle(monkeypatch, max_tokens=10):
    monkeypatch.setattr(abi, "gqa_prompt_workspace_size", lambda *a: (0, 0, 1))
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    dims = abi.GqaDims(4, 2, 64, 0.125)
    cache = abi.Cache(Fake(4, 64, 64, dtype=BF16), Fake(4, 64, 64, dtype=BF16), 64)
    return abi.GqaPrompt(dims, cache, 2, max_tokens, 64)


def test_prompt_buffers_are_allocated_on_the_stream_that_writes_them(calls, monkeypatch):
    """Buffers that a handle makes at their first use, too."""
    h, side = handle(monkeypatch), Stream()
    cu, pos = Fake(3, dtype=I32), Fake(2, dtype=I32)
    rot = h.append(Fake(7, 4, 64, dtype=BF16), *(Fake(7, 2, 64, dtype=BF16) for _ in range(2)), cu, pos, stream=side)
    assert rot.stream is side
    w = [Fake(n * 64, 96, dtype=BF16) for n in (4, 2, 2)] + [Fake(96, 256, dtype=BF16)]
    out = h.from_hidden(Fake(7, 96, dtype=BF16), *w, cu, pos, pos, stream=side)
    assert out.stream is side and out.shape == (7, 96)
    written = {name: args for name, args in calls.made}
    assert {"mla_gqa_prompt_append", "mla_gqa_prompt_attn", "mla_gqa_prompt_out_proj", "mla_gqa_project"} <= set(written)


def test_prompt_buffers_live_as_long_as_their_handle(calls, monkeypatch):
    """Another width of hidden states does not give back what work still queued may be writing."""
    h = handle(monkeypatch)
    made, empty = [], torch.empty

    def noted(*shape, **kw):
        t = empty(*shape, **kw)
        made.append(weakref.ref(t))
        return t

    monkeypatch.setattr(torch, "empty", noted)
    cu, pos = Fake(3, dtype=I32), Fake(2, dtype=I32)
    for hidden in (96, 128, 96, 128):
        w = [Fake(n * 64, hidden, dtype=BF16) for n in (4, 2, 2)] + [Fake(hidden, 256, dtype=BF16)]
        assert h.from_hidden(Fake(5, hidden, dtype=BF16), *w, cu, pos, pos).shape == (5, hidden)
    assert len(made) == 5  # q, k, v; an output for either width
    assert all(t() is not None for t in made)


def test_prompt_projection_operands_that_do_not_fit_are_refused(calls):
    dims = abi.GqaDims(4, 2, 64, 0.125)
    good = dict(o=Fake(7, 4, 64, dtype=BF16), w_o=Fake(96, 256, dtype=BF16), out=Fake(7, 96, dtype=BF16))
    assert abi.gqa_prompt_out_proj(dims, **good) is good["out"]
    assert abi.gqa_prompt_out_proj(dims, **{**good, "out": Fake(9, 96, dtype=BF16)}).shape == (9, 96)
    for name, bad in (("o", Fake(7, 4, 64)),                                 # fp32, as the decode step's o is
                      ("o", Fake(7, 4, 32, dtype=BF16)), ("o", Fake(7, 256, dtype=BF16)), ("out", Fake(6, 96, dtype=BF16)),
                      ("out", Fake(7, 96)), ("out", Fake(7, 100, dtype=BF16)), ("w_o", Fake(96, 128, dtype=BF16)),
                      ("w_o", Fake(96, 256))):
        with pytest.raises(ValueError):
            abi.gqa_prompt_out_proj(dims, **{**good, name: bad})
    assert len(calls.made) == 2
