"""Norm and rotation of heads of which any number of pairs turn, on the GPU
(nlb_norm_rotate), against 64 bits; bounds as in test_gpu_norm_rotate.py."""
import pytest

from tests.test_gpu_norm_rotate import DTYPES, case, check, cuda, run

pytestmark = pytest.mark.gpu


@DTYPES
@pytest.mark.parametrize("dim,freqs", [
    (128, 1), (128, 5), (128, 25), (128, 30), (128, 31), (128, 33), (128, 59), (128, 60), (128, 63), (127, 33), (126, 6),
    (126, 30), (126, 58), (124, 5), (124, 29), (124, 57), (122, 29), (112, 37), (100, 21), (72, 13), (64, 9), (50, 7),
    (36, 5), (20, 5)])
def test_any_number_of_pairs_turns(dtype, dim, freqs):
    check(case(dtype, 9, 13, 3, 2, dim, freqs, seed=dim + freqs, fill=0.8))
    check(case(dtype, 40, 40, 4, 2, dim, freqs, seed=freqs, joint=True, gap=3))
    check(case(dtype, 700, 1, 2, 1, dim, freqs, weights=False))


@DTYPES
@pytest.mark.parametrize("dim,freqs", [(128, 31), (126, 30), (124, 29), (128, 5)])
def test_in_place(dtype, dim, freqs):
    import torch
    import paper_2402_01964_amd as nlb
    c = case(dtype, 300, 200, 4, 2, dim, freqs, fill=0.7)
    want = run(c)
    args = [cuda(c[n]) for n in ("q", "k", "freq", "q_pos", "k_pos", "wq", "wk")]
    dq, dk = cuda(c["dq"]), cuda(c["dk"])
    got = nlb.norm_rotate_backward(dq, dk, *args, dq=dq, dk=dk)
    assert got[0] is dq and all(torch.equal(a, want[k]) for a, k in zip(got, ("dq", "dk", "dwq", "dwk")))
    q, k = nlb.norm_rotate(*args, q_out=args[0], k_out=args[1])
    assert q is args[0] and torch.equal(q, want["q"]) and torch.equal(k, want["k"])
