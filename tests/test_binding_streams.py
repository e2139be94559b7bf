"""What the tensor-level calls make for themselves (outputs that are not given, scratch memory) is made on the stream that the
call's kernels run on, and what they return is kept for the stream that is current.  On the CPU, with stand-ins for torch's streams
and for the library's entry points."""
import contextlib

import pytest
import torch

from paper_2606_17107_amd import pkv


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


CURRENT, OTHER = Stream(11), Stream(22)


@pytest.fixture
def made(monkeypatch):
    """Fake streams; the list gets (maker, stream) of every tensor that a call makes."""
    state, made = [CURRENT], []

    @contextlib.contextmanager
    def on(stream):
        state.append(stream)
        yield
        state.pop()

    def logged(name, real):
        def make(*a, **k):
            made.append((name, state[-1].cuda_stream))
            return real(*a, **k)
        return make

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: state[-1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle))
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: made.append(("kept", s.cuda_stream)))
    for name in ("empty", "zeros"):
        monkeypatch.setattr(torch, name, logged(name, getattr(torch, name)))
    monkeypatch.setattr(pkv, "_gpu_device", lambda t, name: t.device)
    for name in ("pkv_tree_masks", "pkv_tree_verify", "pkv_tree_attention", "pkv_suffix_attention", "pkv_suffix_attention_paged",
                 "pkv_suffix_attention_quant", "pkv_pages_fork", "pkv_pages_compact"):
        monkeypatch.setattr(pkv, name, lambda *a, **k: 0)
    return made


def i32(*shape):
    return torch.ones(shape, dtype=torch.int32)


def bf16(*shape):
    return torch.ones(shape, dtype=torch.bfloat16)


def codes(*shape):
    return torch.ones(shape, dtype=torch.uint8)


def masks(stream):
    pkv.tree_masks(i32(4), i32(1), stream=stream)


def verify(stream):
    pkv.tree_verify(torch.ones(4, 10), i32(4), i32(4), torch.ones(4), torch.ones(1), 4, stream=stream)


def tree(stream):
    x = bf16(1, 2, 4, 64)
    pkv.tree_attention(bf16(1, 4, 2, 64), bf16(1, 2, 90, 64), bf16(1, 2, 90, 64), x, x, bf16(1, 4, 2, 64), i32(4), i32(1), 1.0, 90,
                       stream=stream)


def suffix(stream):
    k = bf16(1, 2, 5000, 64)
    pkv.suffix_attention(bf16(1, 40, 2, 64), k, k, bf16(1, 40, 2, 64), i32(40), i32(1), 1.0, 5000, n_splits=2, stream=stream)


def paged(stream):
    k = bf16(1, 100, 64, 2, 64)
    pkv.suffix_attention_paged(bf16(1, 40, 2, 64), k, k, bf16(1, 40, 2, 64), i32(40), i32(1), i32(1, 80), 1.0, 5000, n_splits=2,
                               stream=stream)


def quant(stream):
    k, e = codes(1, 100, 64, 2, 64), codes(1, 100, 2, 2)
    pkv.suffix_attention_quant(bf16(1, 40, 2, 64), k, k, e, e, bf16(1, 40, 2, 64), i32(40), i32(1), i32(1, 80), 1.0, 5000, n_splits=2,
                               stream=stream)


def fork(stream):
    pkv.pages_fork([bf16(1, 9, 32, 2, 64)], i32(9), i32(3, 3), 32, torch.ones(16, dtype=torch.uint8), 1, stream=stream)


def compact(stream):
    pkv.pages_compact([bf16(1, 9, 32, 2, 64)], i32(9), i32(3, 3), 32, stream=stream)


# How many tensors a call makes, and how many of them it returns.
CALLS = [(masks, 2, 2), (verify, 4, 3), (tree, 1, 0), (suffix, 1, 0), (paged, 1, 0), (quant, 1, 0), (fork, 1, 0), (compact, 2, 1)]


@pytest.mark.parametrize("call,n,returned", CALLS)
@pytest.mark.parametrize("handle", [False, True])
def test_made_on_the_stream_of_the_call(made, call, n, returned, handle):
    call(OTHER.cuda_stream if handle else OTHER)
    assert [s for what, s in made if what != "kept"] == [OTHER.cuda_stream] * n
    assert [s for what, s in made if what == "kept"] == [CURRENT.cuda_stream] * returned


@pytest.mark.parametrize("call,n,returned", CALLS)
@pytest.mark.parametrize("stream", [None, CURRENT, CURRENT.cuda_stream])
def test_made_on_the_current_stream(made, call, n, returned, stream):
    call(stream)
    assert [s for what, s in made if what != "kept"] == [CURRENT.cuda_stream] * n
    assert not [s for what, s in made if what == "kept"]
