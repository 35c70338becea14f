"""Refusals of rwkvq_lowrank, through the C ABI on the CPU (every check is made before a launch), and the binding's own."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2505_03803_b200 import binding as B

EINVAL, ESHAPE, EALIGN, EUNSUPPORTED = 1, 2, 3, 7
FIELDS = ["x", "A", "B", "y", "adapter", "seq_start", "ranks", "scale", "x_prev", "xprev0", "x_row", "y_row", "x_prev_row", "tokens", "n_seq", "ic", "oc", "rank", "n_adapters",
          "x_dtype", "w_dtype", "y_dtype"]
MEM = np.zeros(1 << 20, np.uint8)
P = (MEM.ctypes.data + 255) // 256 * 256
GOOD = dict(x=P, A=P + 65536, B=P + 131072, y=P + 196608, adapter=P, seq_start=P, ranks=P, scale=P, x_prev=0, xprev0=0, x_row=128, y_row=64, x_prev_row=0, tokens=8, n_seq=2,
            ic=128, oc=64, rank=16, n_adapters=3, x_dtype=1, w_dtype=2, y_dtype=0)
MU = B.Desc(method=B.RWKVQ_VQ, bits=6, oc=1, ic=128, group=0, vec_dim=2, tile=0, entries=64)


def status(mu=None, image=None, **kw):
    a = dict(GOOD, **kw)
    return B.lib().rwkvq_lowrank(B._LOWRANK_ARGS.pack(*(a[f] for f in FIELDS)), None if mu is None else C.byref(mu), image, None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=0), EINVAL), (dict(A=0), EINVAL), (dict(B=0), EINVAL), (dict(y=0), EINVAL), (dict(adapter=0), EINVAL), (dict(x_dtype=3), EINVAL), (dict(x_dtype=-1), EINVAL),
    (dict(w_dtype=0), EINVAL), (dict(y_dtype=3), EINVAL), (dict(tokens=-1), EINVAL), (dict(n_seq=0), EINVAL), (dict(ic=0), EINVAL), (dict(oc=-8), EINVAL), (dict(rank=0), EINVAL),
    (dict(n_adapters=0), EINVAL), (dict(seq_start=0), EINVAL), (dict(x_prev=P, x_prev_row=128), EINVAL), (dict(xprev0=P), EINVAL), (dict(rank=136), EUNSUPPORTED),
    (dict(n_seq=65536), EUNSUPPORTED), (dict(tokens=(1 << 24) + 1), EUNSUPPORTED), (dict(ic=(1 << 24) + 8), EUNSUPPORTED), (dict(oc=(1 << 24) + 8), EUNSUPPORTED),
    (dict(ic=124), ESHAPE), (dict(oc=60), ESHAPE), (dict(rank=12), ESHAPE), (dict(x_row=120), EINVAL), (dict(y_row=56), EINVAL), (dict(x_row=132), EALIGN), (dict(y_row=66), EALIGN),
    (dict(x=P + 8), EALIGN), (dict(A=P + 65538), EALIGN), (dict(B=P + 131076), EALIGN), (dict(y=P + 196616), EALIGN), (dict(y=P), EINVAL)], ids=str)
def test_refusals(kw, want):
    assert status(**kw) == want


def test_refusals_of_the_token_shift():
    assert status(image=P) == EINVAL                                                  # no description
    assert status(mu=MU, image=P + 8) == EALIGN
    assert status(mu=MU, image=P, x_prev=P, x_prev_row=128, xprev0=P) == EINVAL       # one of the two
    assert status(mu=MU, image=P, x_prev=P, x_prev_row=64) == EINVAL
    assert status(mu=MU, image=P, x_prev=P, x_prev_row=132) == EALIGN
    assert status(mu=MU, image=P, x_prev=P + 4, x_prev_row=128) == EALIGN
    assert status(mu=MU, image=P, xprev0=P + 4) == EALIGN
    assert status(mu=MU, image=P, ic=256, x_row=256) == ESHAPE                        # a vector of another length
    assert status(mu=B.Desc(method=B.RWKVQ_VQ, bits=5, oc=1, ic=128, vec_dim=2, entries=32), image=P) == EUNSUPPORTED
    assert status(mu=MU, image=P, y=P, x_prev=P, x_prev_row=128) == EINVAL            # y is an input


def test_null_arguments_and_no_rows():
    assert B.lib().rwkvq_lowrank(None, None, None, None) == EINVAL
    assert status(tokens=0, x=0, y=0) == 0
    assert status(tokens=0, x=0, y=0, seq_start=0, n_seq=1) == 0


def test_binding_refuses():
    x, A, Bm, y, adapter = torch.zeros((4, 128)), torch.zeros((2, 16, 128)).half(), torch.zeros((2, 64, 16)).half(), torch.zeros((4, 64)), torch.zeros(1, dtype=torch.int32)
    for args in ((x, A, Bm, y, adapter), (x[0], A, Bm, y, adapter), (x, A[0], Bm, y, adapter), (x, A, Bm, y[:2], adapter)):
        with pytest.raises(B.RwkvqError) as e:
            B.rwkvq_lowrank(*args)            # not on the device, or of another shape
        assert e.value.status == EINVAL
