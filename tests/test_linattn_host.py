"""Refusals of rwkvq_linattn, through the C ABI on the CPU (every check is made before a launch), and the binding's own."""
import numpy as np
import pytest
import torch

from paper_2505_03803_b200 import binding as B

EINVAL, EALIGN, ENOMEM, EUNSUPPORTED = 1, 3, 5, 7
FIELDS = ["r", "k", "v", "logw", "u", "out", "state", "state_out", "seq_start", "slots", "r_row", "k_row", "v_row", "logw_row", "out_row", "tokens", "n_seq",
          "heads", "n", "n_slots", "dtype", "decay_dtype", "decay_per_head"]
MEM = np.zeros(1 << 22, np.uint8)
P = (MEM.ctypes.data + 255) // 256 * 256
GOOD = dict(r=P, k=P + 65536, v=P + 131072, logw=P + 196608, u=P, out=P + 262144, state=P + (1 << 20), state_out=P + (1 << 20), seq_start=P, slots=P, r_row=128,
            k_row=128, v_row=128, logw_row=128, out_row=128, tokens=8, n_seq=2, heads=2, n=64, n_slots=4, dtype=2, decay_dtype=0, decay_per_head=0)


def status(ws_at=P + (1 << 21), ws_bytes=1 << 20, **kw):
    a = dict(GOOD, **kw)
    return B.lib().rwkvq_linattn(B._LINATTN_ARGS.pack(*(a[f] for f in FIELDS)), ws_at, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(r=0), EINVAL), (dict(k=0), EINVAL), (dict(v=0), EINVAL), (dict(logw=0), EINVAL), (dict(out=0), EINVAL),
    (dict(out=P), EINVAL), (dict(out=P + 65536), EINVAL), (dict(out=P + 131072), EINVAL), (dict(out=P + 196608), EINVAL),
    (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(decay_dtype=1), EINVAL), (dict(decay_dtype=3), EINVAL), (dict(tokens=-1), EINVAL),
    (dict(n_seq=0), EINVAL), (dict(heads=0), EINVAL), (dict(n=0), EINVAL), (dict(n_slots=-1), EINVAL), (dict(n=32), EUNSUPPORTED), (dict(n=256), EUNSUPPORTED),
    (dict(n_seq=65536), EUNSUPPORTED), (dict(heads=65536), EUNSUPPORTED), (dict(tokens=(1 << 30) + 1), EUNSUPPORTED), (dict(tokens=5000, r_row=0), EINVAL), (dict(seq_start=0), EINVAL), (dict(slots=0, n_slots=1), EINVAL),
    (dict(n_slots=0), EINVAL), (dict(state=0, state_out=0), EINVAL), (dict(r_row=120), EINVAL), (dict(k_row=0), EINVAL), (dict(v_row=64), EINVAL),
    (dict(out_row=127), EINVAL), (dict(logw_row=64), EINVAL), (dict(decay_per_head=1, logw_row=1), EINVAL), (dict(r_row=132), EALIGN),
    (dict(logw_row=130), EALIGN), (dict(r=P + 8), EALIGN), (dict(k=P + 65538), EALIGN), (dict(v=P + 131076), EALIGN), (dict(out=P + 262146), EALIGN),
    (dict(logw=P + 196612), EALIGN), (dict(u=P + 4), EALIGN), (dict(state=P + (1 << 20) + 4), EALIGN), (dict(state_out=P + (1 << 20) + 16), EINVAL),
    (dict(state_out=P + (1 << 20) + 4 * 32768 - 16), EINVAL)], ids=str)
def test_refusals(kw, want):
    assert status(**kw) == want


def test_null_arguments():
    assert B.lib().rwkvq_linattn(None, None, 0, None) == EINVAL


def test_binding_refuses():
    T, H, n = 4, 2, 64
    x = [torch.zeros((T, H, n)) for _ in range(5)]
    with pytest.raises(B.RwkvqError) as e:
        B.rwkvq_linattn(*x[:4], None, x[4], None)        # not on the device
    assert e.value.status == EINVAL
    with pytest.raises(B.RwkvqError):
        B.rwkvq_linattn(x[0][0], *x[1:4], None, x[4], None)


def test_workspace():
    size = B.rwkvq_linattn_workspace_bytes
    assert size(1, 1, 4, 64) == size(8, 8, 4, 64) == size(100, 1, 4, 32) == size(-1, 1, 4, 64) == size(5, 0, 4, 64) == 0
    for heads, n in ((1, 64), (32, 64), (64, 64), (300, 64), (5, 128)):
        last = 0
        for tokens in list(range(9, 700, 7)) + [1000, 2048, 4100, 9999, 70001]:
            assert size(tokens, 1, heads, n) >= last, (tokens, heads, n)
            assert size(tokens, tokens, heads, n) >= size(tokens, 1, heads, n)
            last = size(tokens, 1, heads, n)
    need = size(5000, 2, 2, 64)
    assert need > 0
    assert status(tokens=5000, ws_bytes=need - 1) == ENOMEM and status(tokens=5000, ws_at=0, ws_bytes=need) == ENOMEM
    assert status(tokens=5000, ws_at=P + (1 << 21) + 4, ws_bytes=need) == EALIGN


def test_a_long_sequence_among_short_ones_is_not_gone_through_token_by_token():
    # whatever the average length: a list that leaves room for a long sequence takes the chunks' passes, which need the workspace
    assert status(tokens=600, n_seq=400, n_slots=400, ws_at=0, ws_bytes=0) == ENOMEM
    assert status(tokens=2000, n_seq=1000, n_slots=1000, ws_at=0, ws_bytes=0) == ENOMEM
    assert status(tokens=400, n_seq=400, n_slots=400, ws_at=0, ws_bytes=0) != ENOMEM       # single tokens do not


def test_few_sequences_take_the_chunks_from_nine_tokens_on():
    for n_seq, tokens in ((1, 9), (1, 16), (2, 9), (3, 12), (4, 19), (8, 17), (16, 33)):
        assert status(tokens=tokens, n_seq=n_seq, n_slots=n_seq, ws_at=0, ws_bytes=0) == ENOMEM, (n_seq, tokens)
    for n_seq, tokens in ((1, 8), (5, 10), (8, 16), (16, 31), (96, 111)):
        assert status(tokens=tokens, n_seq=n_seq, n_slots=n_seq, ws_at=0, ws_bytes=0) != ENOMEM, (n_seq, tokens)
