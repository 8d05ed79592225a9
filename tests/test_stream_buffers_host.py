"""Where the buffers that a call makes itself come from, without a GPU: the
library's calls and torch's streams are stood in for, tensors are host memory
that says it is on the card."""
import contextlib

import pytest
import torch

import paper_2608_23429_amd as cheb

CARD = torch.device("cuda", 0)


class OnCard(torch.Tensor):
    is_cuda = property(lambda self: True)
    device = property(lambda self: CARD)

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.recorded = getattr(self, "recorded", []) + [stream]


class Stream:
    device, cuda_stream = CARD, 7


USER, SIDE = Stream(), Stream()


@pytest.fixture
def card(monkeypatch):
    """torch.empty gives tensors that know the stream they were made on."""
    now = [USER]
    empty = torch.empty

    def make(*size, dtype=None, device=None):
        t = empty(*size, dtype=dtype).as_subclass(OnCard)
        t.made_on = now[-1]
        return t

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    monkeypatch.setattr(torch, "empty", make)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(cheb, "_raw_stream", lambda device: 0)
    for name in ("cheb_add_norm", "cheb_residual_norm", "cheb_cache_read", "cheb_extrapolate",
                 "cheb_extrapolate_at", "cheb_extrapolate_multi", "cheb_extrapolate_at_multi",
                 "cheb_extrapolate_steps"):
        monkeypatch.setattr(cheb, name, lambda *a, **k: None)
    monkeypatch.setattr(cheb._binding, "weights_at", lambda h, t: [1.0])


def on_card(*size, dtype=torch.float32):
    return torch.zeros(*size, dtype=dtype).as_subclass(OnCard)


def cache(quant=None):
    c = object.__new__(cheb.ChebCache)
    c._h, c.n_slots, c.dtype, c.quant, c.layout = None, 1, torch.bfloat16, quant, "slots"
    c.seg_numel, c.slot_numel, c.device, c.arena = [128], 128, CARD, on_card(4)
    return c


def history():
    h = object.__new__(cheb.ResidualHistory)
    h.cache = cache()
    return h


class Table:
    handle = None


def made(result):
    """The tensors a call returned, however nested."""
    if isinstance(result, torch.Tensor):
        return [result]
    if isinstance(result, (tuple, list)):
        return [t for r in result for t in made(r)]
    return []


CALLS = {
    "add_norm": lambda s: cheb.add_norm([on_card(2, 64)], [1.0], stream=s),
    "add_norm_mxfp8": lambda s: cheb.add_norm([on_card(2, 64)], [1.0], out="mxfp8", stream=s),
    "add_norm_row": lambda s: cheb.add_norm([on_card(2, 64)], [1.0], out="fp8_row", stream=s),
    "residual_norm": lambda s: cache().residual_norm([1.0], 0, dim=64, stream=s),
    "predict_norm": lambda s: history().predict_norm(0.5, dim=64, stream=s),
    "read": lambda s: cache().read(0, stream=s),
    "read_8bit": lambda s: cache("mxint8").read(0, stream=s),
    "extrapolate": lambda s: cache().extrapolate([1.0], stream=s),
    "extrapolate_8bit": lambda s: cache("mxfp8").extrapolate([1.0], stream=s),
    "extrapolate_at": lambda s: cache().extrapolate_at(0.5, stream=s),
    "extrapolate_multi": lambda s: cache().extrapolate_multi([[1.0], [2.0]], stream=s),
    "extrapolate_at_multi": lambda s: cache().extrapolate_at_multi([0.5, 0.6], stream=s),
    "extrapolate_steps": lambda s: cache().extrapolate_steps(Table(), 0, 2, stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_buffers_come_from_the_calls_stream(card, name):
    """A buffer made within a call on another stream is that stream's, and is
    held back until the current stream is done with it."""
    tensors = made(CALLS[name](SIDE))
    assert tensors
    for t in tensors:
        assert t.made_on is SIDE and t.recorded == [USER]


@pytest.mark.parametrize("name", CALLS)
def test_buffers_of_the_current_stream(card, name):
    tensors = made(CALLS[name](None))
    assert tensors
    for t in tensors:
        assert t.made_on is USER and not hasattr(t, "recorded")
