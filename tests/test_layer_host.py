"""MoeLayer's own decisions without a GPU: which stream its work is given to and
which tensors it takes.  The library's calls are recorded instead of made, so
tensors on the CPU stand in for the device's."""
import inspect

import pytest

torch = pytest.importorskip("torch")

from paper_2607_26444_amd import layer as mod  # noqa: E402
from paper_2607_26444_amd import moe  # noqa: E402

CALLS = ("moe_rmsnorm", "moe_route", "moe_layout", "moe_dispatch", "moe_expert_matmul",
         "moe_quantize", "moe_combine")
T, H, I, E, K = 6, 256, 32, 8, 2


class Stream:
    """A stream of another library: an address, as the binding takes it."""
    cuda_stream = 0x7F00DEADB000


class Record(list):
    """(name, arguments by name, torch's current stream) of every call."""
    current = None

    def names(self):
        return [name for name, _, _ in self]

    def arguments(self, name):
        return next(args for n, args, _ in self if n == name)


@pytest.fixture
def record(monkeypatch):
    calls = Record()

    def stand_in(name):
        signature = inspect.signature(getattr(moe, name))

        def call(*args, **kw):
            bound = signature.bind(*args, **kw)
            bound.apply_defaults()
            calls.append((name, bound.arguments, calls.current))
        return call

    class Current:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.before, calls.current = calls.current, self.stream.cuda_stream

        def __exit__(self, *_):
            calls.current = self.before

    class External:
        def __init__(self, address, **_):
            self.cuda_stream = address

    for name in CALLS:
        monkeypatch.setattr(moe, name, stand_in(name))
    # host memory has not the alignment of a workspace; an empty one has
    monkeypatch.setattr(moe, "moe_layout_workspace_bytes", lambda *_: 0)
    monkeypatch.setattr(torch.cuda, "stream", Current)
    monkeypatch.setattr(torch.cuda, "ExternalStream", External)
    return calls


def _layer(T=T, E=E, K=K):
    def int8(*shape):
        return torch.ones(*shape, dtype=torch.int8)
    return mod.MoeLayer(T, H, I, E, K, torch.ones(H), int8(E, 2 * I, H), torch.ones(E, 2 * I),
                        int8(E, H, I), torch.ones(E, H), device="cpu")


def _rows(T=T):
    return [torch.zeros(T, H, dtype=torch.bfloat16) for _ in range(2)]


@pytest.mark.parametrize("stream", [None, Stream()])
def test_a_gate_runs_on_the_stream_of_the_calls(record, stream):
    """The gate reads what the norm left and the routing reads what it returns:
    torch's work has to be on the stream that both are enqueued on, after the
    one and before the other."""
    layer = _layer()

    def gate(normed):
        assert normed is layer.normed
        record.append(("gate", {}, record.current))
        return torch.zeros(T, E)
    layer.forward(*_rows(), gate, stream=stream)
    names = record.names()
    assert names.index("moe_rmsnorm") < names.index("gate") < names.index("moe_route")
    assert all(args["stream"] is stream for name, args, _ in record if name != "gate")
    want = None if stream is None else stream.cuda_stream
    assert [on for name, _, on in record if name == "gate"] == [want]
    assert record.current is None              # the caller's stream is current again


def test_logits_whose_rows_lie_on_each_other(record):
    """A row expanded to all tokens has row pitch 0, which the call takes as packed rows:
    it would read T times the storage.  Overlapping rows have a pitch under E."""
    layer = _layer()
    storage = torch.zeros(T + E)
    for logits in (storage[:E].expand(T, E), storage.as_strided((T, E), (1, 1)),
                   storage[:1].expand(T, E), torch.zeros(E, T).t()):
        with pytest.raises(ValueError, match="logits"):
            layer.forward(*_rows(), logits)
        assert "moe_route" not in record.names()


@pytest.mark.parametrize("tokens,experts", [(1, E), (T, K), (1, K)])
def test_logits_pitch(record, tokens, experts):
    """The pitch is that of the rows; of one row the stride says nothing."""
    layer = _layer(T=tokens, E=experts)
    wide = torch.zeros(tokens, experts + 3)
    for logits, pitch in ((torch.zeros(tokens, experts), experts), (wide[:, 2:2 + experts], experts + 3)):
        record.clear()
        layer.forward(*_rows(tokens), logits)
        got = record.arguments("moe_route")["logits_pitch"]
        assert got == pitch if tokens > 1 else got >= experts
    if tokens == 1:
        for logits in (torch.zeros(experts, 1).t(), torch.zeros(experts).expand(1, experts),
                       torch.zeros(experts).as_strided((1, experts), (0, 1))):
            record.clear()
            layer.forward(*_rows(tokens), logits)
            assert record.arguments("moe_route")["logits_pitch"] == experts


def test_logits_of_one_expert(record):
    """Of one column the stride says nothing either."""
    layer = _layer(E=1, K=1)
    for logits, pitch in ((torch.zeros(1, T).t(), 1), (torch.zeros(T, 5)[:, 3:4], 5)):
        record.clear()
        layer.forward(*_rows(), logits)
        assert record.arguments("moe_route")["logits_pitch"] == pitch


def test_token_mask_strides(record):
    """The call reads T neighbouring bytes: a column of a table would give other
    tokens' bytes, an expanded one bytes past its storage."""
    layer = _layer()
    table = torch.ones(T, 3, dtype=torch.uint8)
    for mask in (table[:, 1], table[0, :1].expand(T), torch.ones(2 * T, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="token_mask"):
            layer.forward(*_rows(), torch.zeros(T, E), token_mask=mask)
        assert "moe_route" not in record.names()
    good = table.t().contiguous()[1]
    layer.forward(*_rows(), torch.zeros(T, E), token_mask=good)
    assert record.arguments("moe_route")["token_mask"] is good


@pytest.mark.parametrize("stride", [0, 7])
def test_token_mask_of_one_token(record, stride):
    """Of one token the stride says nothing."""
    layer = _layer(T=1)
    mask = torch.ones(9, dtype=torch.uint8).as_strided((1,), (stride,))
    layer.forward(*_rows(1), torch.zeros(1, E), token_mask=mask)
    assert record.arguments("moe_route")["token_mask"] is mask
