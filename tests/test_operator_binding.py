"""What the Python binding of the operators without a table refuses before the
library sees the call; no GPU is needed (CPU tensors that say they are on one)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2402_01964_amd as nlb  # noqa: E402


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", 0))


def on_device(t):
    return torch.Tensor._make_subclass(OnDevice, t, t.requires_grad)


def rows(*shape):
    """A tensor of any size that takes a row's memory."""
    return on_device(torch.zeros(*(1,) * (len(shape) - 1), shape[-1]).expand(*shape))


@pytest.fixture
def no_library(monkeypatch):
    """A call that reaches the library fails its test."""
    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was called")
    monkeypatch.setattr(nlb, "load_library", lambda: Library())
    monkeypatch.setattr(nlb, "_current_stream", lambda device: 0)


@pytest.mark.parametrize("q,k,batch", [
    ((2, 1, 8), (2**32 + 2, 1, 8), 1), ((2**32 + 2, 1, 8), (2, 1, 8), 1), ((2, 1, 8), (2, 1, 8), 2**32 + 1),
    ((2, 1, 8), (2, 1, 8), -1), ((2, 2**32 + 1, 8), (2, 1, 8), 1), ((2, 1, 8), (2, 2**32 + 1, 8), 1)],
    ids=["k rows", "q rows", "batch", "negative batch", "heads", "kv heads"])
def test_attention_refuses_sizes_beyond_32_bits(no_library, q, k, batch):
    """They would arrive in the library as what is left of them in 32 bits."""
    with pytest.raises(ValueError, match="2\\^31"):
        nlb.attention_work(rows(*q), rows(*k), rows(*k), batch=batch)


@pytest.mark.parametrize("shape", [(2**32 + 2, 4), (2, 2**32 + 4)])
def test_layer_norm_refuses_sizes_beyond_32_bits(no_library, shape):
    x = on_device(torch.empty(shape[1]).expand(shape))        # (memory that nothing touches)
    stats = on_device(torch.empty(shape[0]))
    with pytest.raises(ValueError, match="2\\^31"):
        nlb.layer_norm(x, out=x, mean=stats, rstd=stats)


class Kept(Exception):
    """The call came as far as the library."""


@pytest.fixture
def library_keeps(monkeypatch):
    class Library:
        def __getattr__(self, name):
            raise Kept(name)
    monkeypatch.setattr(nlb, "load_library", lambda: Library())
    monkeypatch.setattr(nlb, "_current_stream", lambda device: 0)


@pytest.mark.parametrize("leaf", ["q", "k", "v", "bias", "x", "w", "b"])
def test_calls_that_would_lose_gradients_are_refused(library_keeps, leaf):
    """The operators keep no autograd graph: with inputs that require
    gradients they are refused, but not under no_grad or within a Function."""
    def t(name, *shape):
        return on_device(torch.zeros(shape).requires_grad_(name == leaf))

    def call():
        if leaf in ("x", "w", "b"):
            return nlb.layer_norm(t("x", 3, 4), t("w", 4), t("b", 4), out=t("y", 3, 4), mean=t("m", 3), rstd=t("r", 3))
        return nlb.attention(t("q", 2, 1, 8), t("k", 2, 1, 8), t("v", 2, 1, 8), bias=t("bias", 1, 1),
                             out=t("o", 2, 1, 8), lse=t("l", 2, 1))

    with pytest.raises(RuntimeError, match="_backward"):
        call()
    with torch.no_grad(), pytest.raises(Kept):
        call()

    class Function(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return call()
    with pytest.raises(Kept):
        Function.apply(torch.zeros(1, requires_grad=True))
    leaf = None
    with pytest.raises(Kept):
        call()
