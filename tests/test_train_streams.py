"""Where the training step's operators stand in the order of torch's streams, checked without a GPU: a library and streams that
write down what is asked of them."""
import pytest
import torch

import paper_2601_02311_b200.ps as ps

OWN, OTHER = 7, 5


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


class Library:
    """Sizes of work buffers come from the library itself; a call is written down."""

    def __init__(self, log, code):
        self.log, self.code = log, code

    def __getattr__(self, name):
        if name.endswith("_bytes") or name == "ps_strerror":
            return getattr(REAL, name)

        def call(*args):
            self.log.append(name)
            return self.code
        return call


REAL = ps._lib


@pytest.fixture
def setup(monkeypatch):
    def make(current, code=ps.OK, own=OWN):
        log = []
        c = ps.Context.__new__(ps.Context)
        c.torch_device, c.device, c._h, c._raw_stream = torch.device("cpu"), -1, None, own    # a host tensor's device is -1
        c.stream = Stream("own", log) if own else None
        monkeypatch.setattr(ps, "_lib", Library(log, code))
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: current, raising=False)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream("current", log))
        monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream("default", log))
        return c, log
    return make


def calls():
    x, tokens = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    q, k = torch.zeros(2, 5, 4, 16, dtype=torch.bfloat16), torch.zeros(2, 6, 2, 16, dtype=torch.bfloat16)
    one, far = torch.zeros(1, 1, 2, 16, dtype=torch.bfloat16), torch.zeros(1, 5000, 2, 16, dtype=torch.bfloat16)
    lse = torch.zeros(2, 4, 5)
    return {
        "dropout_into": ("ps_dropout", lambda c: c.dropout_into(x, x.clone(), 0.1, 1)),
        "dropout": ("ps_dropout", lambda c: c.dropout(x, 0.1, 1, residual=x)),
        "embed_forward_into": ("ps_embed_forward", lambda c: c.embed_forward_into(x, tokens, torch.zeros(4, 8))),
        "embed_forward": ("ps_embed_forward", lambda c: c.embed_forward(x, tokens)),
        "embed_backward_into": ("ps_embed_backward", lambda c: c.embed_backward_into(x, tokens, torch.zeros(9, 8))),
        "embed_backward": ("ps_embed_backward", lambda c: c.embed_backward(x, tokens, 9)),
        "attention_forward_into": ("ps_attention_forward", lambda c: c.attention_forward_into(q, k, k, q.clone(), lse)),
        "attention_forward": ("ps_attention_forward", lambda c: c.attention_forward(q, k, k)),
        "attention_forward, in chunks": ("ps_attention_forward", lambda c: c.attention_forward(one, far, far)),
        "attention_backward_into": ("ps_attention_backward",
                                    lambda c: c.attention_backward_into(q, k, k, q, lse, q, q.clone(), k.clone(), k.clone())),
        "attention_backward": ("ps_attention_backward", lambda c: c.attention_backward(q, k, k, q, lse, q)),
    }


@pytest.mark.parametrize("name", calls())
def test_a_call_takes_its_place_in_the_current_streams_order(setup, name):
    call, run = calls()[name]
    c, log = setup(OTHER)
    run(c)
    assert log == [("own", "waits for", "current"), call, ("current", "waits for", "own")]


@pytest.mark.parametrize("name", calls())
def test_a_call_on_the_contexts_own_stream_waits_for_nothing(setup, name):
    call, run = calls()[name]
    c, log = setup(OWN)
    run(c)
    assert log == [call]


def test_a_context_without_a_stream_is_the_default_streams(setup):
    call, run = calls()["dropout"]
    c, log = setup(OTHER, own=0)
    run(c)
    assert log == [("default", "waits for", "current"), call, ("current", "waits for", "default")]


@pytest.mark.parametrize("name", calls())
def test_a_refused_call_leaves_the_streams_in_order(setup, name):
    call, run = calls()[name]
    c, log = setup(OTHER, code=ps.E_DEVICE)
    with pytest.raises(ps.PsError) as e:
        run(c)
    assert e.value.code == ps.E_DEVICE
    assert log == [("own", "waits for", "current"), call, ("current", "waits for", "own")]
