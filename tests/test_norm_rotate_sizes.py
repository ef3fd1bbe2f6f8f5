"""Which kernel a norm and rotation of each size takes, without a GPU: a stand-in
for HIP's launch calls records the launches."""
from tests.test_operator_launches import stand_in  # noqa: F401
from tests.test_training_launches import run


def test_every_size_that_is_allowed_runs(stand_in):  # noqa: F811
    """Heads of 1 to 128 values, of which any number of pairs turn, in both types."""
    run(stand_in, """
n, refused = ctypes.c_size_t(), []
for dtype in (nlb.DTYPE_BF16, nlb.DTYPE_F32):
    for dim in range(1, nlb.ATT_MAX_DIM + 1):
        for freqs in range(dim // 2 + 1):
            c = rotate(dtype=dtype, dim=dim, freqs=freqs)
            assert lib.nlb_norm_rotate_work(c, n) == nlb.NLB_OK and n.value > 0
            got = turned(c), len(sizes()), rotate_backward(lib, c, size=n.value), len(sizes())
            if got != (nlb.NLB_OK, 1, nlb.NLB_OK, 2):
                refused.append((dtype, dim, freqs, got))
assert not refused, (len(refused), refused[:5], sorted({r[1] for r in refused}))
""")
