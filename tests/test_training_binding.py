"""What the Python binding of the operators that train a retrieval layer refuses
before the library sees the call; no GPU is needed (CPU tensors that say they are
on one)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2402_01964_amd as nlb  # noqa: E402
from tests.test_operator_binding import Kept, library_keeps, no_library, on_device, rows  # noqa: E402,F401


def t(*shape, dtype=torch.float32):
    return on_device(torch.zeros(*shape, dtype=dtype))


def ints(*shape):
    return t(*shape, dtype=torch.int32)


def huge(*shape, dtype=torch.float32):
    """A tensor of any size that takes a value's memory."""
    return on_device(torch.zeros((1,) * len(shape), dtype=dtype).expand(*shape))


@pytest.mark.parametrize("call", [
    lambda: nlb.lookup(huge(2**32 + 2, 4), ints(3)),
    lambda: nlb.lookup_work(t(3, 4), ints(3), 2**32 + 1),
    lambda: nlb.lookup_work(t(3, 4), ints(3), -1),
    lambda: nlb.lookup_backward(huge(2**32 + 2, 1), huge(2**32 + 2, dtype=torch.int32), 5),
    lambda: nlb.gated_scan_work(huge(2**32 + 2, 4), huge(2**32 + 2, 4)),
    lambda: nlb.gated_scan_work(t(4, 4), t(4, 4), batch=2**32 + 4),
    lambda: nlb.gated_scan_work(t(4, 4), t(4, 4), batch=-1),
    lambda: nlb.norm_rotate(huge(2**32 + 2, 1, 8), None, None, None, None),
    lambda: nlb.norm_rotate(t(2, 1, 8), huge(2**32 + 2, 1, 8), None, None, None),
], ids=range(9))
def test_sizes_beyond_32_bits(no_library, call):  # noqa: F811
    with pytest.raises(ValueError, match="2\\^31"):
        call()


x3, q3 = (5, 4), (5, 2, 8)


@pytest.mark.parametrize("error,call", [
    (TypeError, lambda: nlb.lookup(torch.zeros(3, 4), ints(3))),
    (TypeError, lambda: nlb.lookup(t(3, 4, dtype=torch.float16), ints(3))),
    (ValueError, lambda: nlb.lookup(t(3, 4, 2), ints(3))),
    (TypeError, lambda: nlb.lookup(t(3, 4), t(3, dtype=torch.int64))),
    (TypeError, lambda: nlb.lookup(t(3, 4), torch.zeros(3, dtype=torch.int32))),
    (ValueError, lambda: nlb.lookup(t(3, 4), on_device(torch.zeros(6, dtype=torch.int32)[::2]))),
    (ValueError, lambda: nlb.lookup(t(3, 4), ints(3), out=t(3, 5))),
    (ValueError, lambda: nlb.lookup(on_device(torch.zeros(4, 3).T), ints(3), out=t(3, 4))),
    (TypeError, lambda: nlb.lookup(t(3, 4), ints(3), out=t(3, 4, dtype=torch.bfloat16))),
    (ValueError, lambda: nlb.lookup_work(t(4, 4), ints(3), 9)),
    (ValueError, lambda: nlb.gated_scan(t(5, 4, 2), t(5, 4, 2))),
    (ValueError, lambda: nlb.gated_scan(t(*x3), t(5, 5))),
    (TypeError, lambda: nlb.gated_scan(t(*x3), t(*x3, dtype=torch.bfloat16))),
    (TypeError, lambda: nlb.gated_scan(t(*x3), t(*x3), start=t(3, dtype=torch.int64))),
    (ValueError, lambda: nlb.gated_scan(t(*x3), t(*x3), batch=3, start=ints(3))),
    (ValueError, lambda: nlb.gated_scan(t(*x3), t(*x3), h0=t(2, 4))),
    (TypeError, lambda: nlb.gated_scan(t(*x3), t(*x3), h0=t(1, 4, dtype=torch.bfloat16))),
    (ValueError, lambda: nlb.norm_rotate(t(5, 8), None, None, None, None)),
    (ValueError, lambda: nlb.norm_rotate(t(*q3), t(5, 2, 9), None, None, None)),
    (TypeError, lambda: nlb.norm_rotate(t(*q3), t(*q3, dtype=torch.bfloat16), None, None, None)),
    (ValueError, lambda: nlb.norm_rotate(t(*q3), None, t(4), None, None)),
    (ValueError, lambda: nlb.norm_rotate(t(*q3), t(*q3), t(4), ints(5), None)),
    (ValueError, lambda: nlb.norm_rotate(t(*q3), t(*q3), t(5), ints(5), ints(5))),
    (ValueError, lambda: nlb.norm_rotate(t(*q3), t(*q3), t(4), ints(4), ints(5))),
    (TypeError, lambda: nlb.norm_rotate(t(*q3), t(*q3), t(4), t(5), ints(5))),
    (ValueError, lambda: nlb.norm_rotate(t(*q3), t(*q3), None, None, None, t(9))),
    (ValueError, lambda: nlb.norm_rotate(t(*q3), None, None, None, ints(5))),
], ids=range(27))
def test_wrong_tensors(no_library, error, call):  # noqa: F811
    with pytest.raises(error):
        call()


@pytest.mark.parametrize("leaf", ["table", "x", "g", "h0", "q", "k", "freq", "wq", "wk"])
def test_calls_that_would_lose_gradients_are_refused(library_keeps, leaf):  # noqa: F811
    def t(name, *shape):
        return on_device(torch.zeros(shape).requires_grad_(name == leaf))

    def call():
        if leaf == "table":
            return nlb.lookup(t("table", 3, 4), ints(2), out=on_device(torch.zeros(2, 4)))
        if leaf in ("x", "g", "h0"):
            return nlb.gated_scan(t("x", 3, 4), t("g", 3, 4), h0=t("h0", 1, 4), out=t("o", 3, 4), last=t("l", 1, 4),
                                  states=t("s", 1, 4))
        return nlb.norm_rotate(t("q", 2, 1, 8), t("k", 2, 1, 8), t("freq", 4), ints(2), ints(2), t("wq", 8), t("wk", 8),
                               q_out=t("a", 2, 1, 8), k_out=t("b", 2, 1, 8))
    with pytest.raises(RuntimeError, match="_backward"):
        call()
    with torch.no_grad(), pytest.raises(Kept):
        call()
    leaf = None
    with pytest.raises(Kept):
        call()
