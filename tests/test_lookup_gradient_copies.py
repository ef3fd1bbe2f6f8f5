"""A gradient of more dimensions that is not contiguous is copied once, on the
stream of the call; no GPU is needed (CPU tensors that say they are on one)."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

import paper_2402_01964_amd as nlb  # noqa: E402
from tests.test_operator_binding import Kept, OnDevice, library_keeps, on_device  # noqa: E402,F401

ids = on_device(torch.zeros(4, 3, dtype=torch.int32))
buffers = dict(grads=on_device(torch.zeros(12, 5)), row_ids=on_device(torch.zeros(12, dtype=torch.int32)),
               count=on_device(torch.zeros(1, dtype=torch.int32)))


@pytest.mark.parametrize("call,copies", [
    (lambda d, **k: nlb.lookup_work(d, ids, 9, listed=True), 0),
    (lambda d, **k: nlb.lookup_backward(d, ids, 9, dtable=on_device(torch.zeros(9, 5)), **k), 1),
    (lambda d, **k: nlb.lookup_backward_listed(d, ids, 9, **buffers, **k), 1)], ids=["work", "whole", "listed"])
@pytest.mark.parametrize("with_stream", [False, True])
def test_copied_once_on_the_calls_stream(library_keeps, monkeypatch, call, copies, with_stream):  # noqa: F811
    now, seen = ["current"], []

    class Watched(OnDevice):
        def reshape(self, *shape):
            seen.append(now[0])
            return torch.Tensor.reshape(self, *shape)

    @contextlib.contextmanager
    def on(stream, device):
        now[0] = stream
        yield
        now[0] = "current"
    monkeypatch.setattr(nlb, "_on", on)
    dout = torch.Tensor._make_subclass(Watched, torch.zeros(3, 4, 5).transpose(0, 1))
    with pytest.raises(Kept):
        call(dout, **({"stream": "side"} if with_stream else {}))
    assert seen == ["side" if with_stream else "current"] * copies


@pytest.mark.gpu
def test_the_copy_on_another_stream_is_the_gradient():
    side = torch.cuda.Stream()
    i = torch.randint(-1, 9, (40, 30), dtype=torch.int32, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                             # made on that stream, after some work on it
        dout = torch.randn(500, 30, 40, 5, device="cuda").sum(0).transpose(0, 1)
    got = nlb.lookup_backward(dout, i, 9, 2.0, stream=side)
    grads, row_ids, count = nlb.lookup_backward_listed(dout, i, 9, 2.0, stream=side)
    side.synchronize()
    assert torch.equal(got, nlb.lookup_backward(dout.contiguous(), i, 9, 2.0))
    n = int(count)
    assert n == 9 and torch.equal(grads[:n], got[row_ids[:n].long()])
