"""Refusals of rwkvq_beam_select and rwkvq_state_reorder, through the C ABI on the CPU (every check is made before a launch), and the binding's own."""
import struct

import numpy as np
import pytest
import torch

from paper_2505_03803_b200 import binding as B

EINVAL, EALIGN, ENOMEM, EUNSUPPORTED = 1, 3, 5, 7
MEM = np.zeros(1 << 20, np.uint8)
P = (MEM.ctypes.data + 255) // 256 * 256
FIELDS = ["logits", "scores", "finished", "next_scores", "parents", "tokens", "finished_out", "logits_row", "requests", "beams", "vocab", "picks", "eos", "dtype"]
GOOD = dict(logits=P, scores=P + 4096, finished=P + 8192, next_scores=P + 12288, parents=P + 16384, tokens=P + 20480, finished_out=P + 24576, logits_row=100, requests=2, beams=3,
            vocab=100, picks=6, eos=7, dtype=0)


def status(ws_at=P + 65536, ws_bytes=1 << 19, **kw):
    a = dict(GOOD, **kw)
    return B.lib().rwkvq_beam_select(B._BEAM_SELECT_ARGS.pack(*(a[f] for f in FIELDS)), ws_at, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(logits=0), EINVAL), (dict(scores=0), EINVAL), (dict(next_scores=0), EINVAL), (dict(parents=0), EINVAL), (dict(tokens=0), EINVAL), (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL),
    (dict(requests=0), EINVAL), (dict(beams=0), EINVAL), (dict(vocab=0), EINVAL), (dict(picks=0), EINVAL), (dict(vocab=1, logits_row=1, picks=4, eos=0), EINVAL), (dict(eos=-1), EINVAL),
    (dict(eos=100), EINVAL), (dict(eos=100, finished=0), EINVAL), (dict(eos=-1, finished_out=0), EINVAL), (dict(logits_row=99), EINVAL), (dict(next_scores=P + 4096), EINVAL),
    (dict(finished_out=P + 8192), EINVAL), (dict(beams=65), EUNSUPPORTED), (dict(picks=65), EUNSUPPORTED), (dict(vocab=(1 << 24) + 1, logits_row=1 << 25), EUNSUPPORTED),
    (dict(requests=32768, beams=2), EUNSUPPORTED), (dict(logits=P + 2), EALIGN), (dict(dtype=2, logits=P + 1), EALIGN), (dict(scores=P + 4098), EALIGN), (dict(next_scores=P + 12290), EALIGN),
    (dict(parents=P + 16385), EALIGN), (dict(tokens=P + 20482), EALIGN), (dict(ws_at=0), ENOMEM), (dict(ws_bytes=64), ENOMEM), (dict(ws_at=P + 65544), EALIGN)], ids=str)
def test_refusals(kw, want):
    assert status(**kw) == want


def test_workspace_is_enough_for_less():
    size = B.rwkvq_beam_select_workspace_bytes
    assert size(0, 1, 10, 1) == size(1, 0, 10, 1) == size(1, 1, 0, 1) == size(1, 1, 10, 0) == size(1, 1, 10, 11) == size(1, 65, 10, 1) == size(1, 1, 100, 65) == 0
    assert B.lib().rwkvq_beam_select(None, None, 0, None) == EINVAL
    last = 0
    for requests in (1, 2, 5, 16, 40, 100, 592, 593, 4000):
        assert size(requests, 4, 65536, 8) >= last
        last = size(requests, 4, 65536, 8)
        assert last >= max(size(requests, 3, 65536, 8), size(requests, 4, 65535, 8), size(requests, 4, 2049, 8), size(requests, 4, 65536, 7)) and size(requests, 4, 2049, 8) >= size(requests, 4, 2048, 8)


def reorder(parts, n_slots=4, parents=P, slots=0, requests=1, beams=4, n=None):
    data = struct.pack(f"@{3 * len(parts)}Q", *(v for p in parts for v in p))
    return B.lib().rwkvq_state_reorder(data, len(parts) if n is None else n, n_slots, parents, slots, requests, beams, None)


@pytest.mark.parametrize("kw,want", [
    (dict(parents=0), EINVAL), (dict(n=0), EINVAL), (dict(n_slots=0), EINVAL), (dict(requests=0), EINVAL), (dict(beams=0), EINVAL), (dict(requests=2), EINVAL), (dict(beams=65, n_slots=65), EUNSUPPORTED),
    (dict(requests=(1 << 18) + 1, slots=P), EUNSUPPORTED), (dict(n_slots=(1 << 20) + 1, slots=P), EUNSUPPORTED), (dict(parts=[(0, 64, 64)]), EINVAL), (dict(parts=[(P, 64, 0)]), EINVAL), (dict(parts=[(P, 48, 64)]), EINVAL), (dict(parts=[(P + 8, 64, 64)]), EALIGN),
    (dict(parts=[(P, 72, 64)]), EALIGN), (dict(parts=[(P, 64, 40)]), EALIGN), (dict(parts=[(P, 1 << 46, 64)]), EUNSUPPORTED), (dict(parts=[(P, 1 << 40, 1 << 40)]), EUNSUPPORTED),
    # the same buffer twice; one that begins in another; layers that lie between one another's slots and overlap; such with another distance
    (dict(parts=[(P, 64, 64), (P, 64, 64)]), EINVAL), (dict(parts=[(P, 64, 64), (P + 240, 64, 64)]), EINVAL), (dict(parts=[(P, 256, 64), (P + 48, 256, 64)]), EINVAL),
    (dict(parts=[(P + 64, 256, 64), (P, 256, 96)]), EINVAL), (dict(parts=[(P, 256, 64), (P + 224, 256, 64)]), EINVAL), (dict(parts=[(P, 256, 64), (P + 64, 128, 64)]), EINVAL),
    (dict(parts=[(P, 256, 64), (P + 64, 256, 64), (P + 128, 256, 64), (P + 192 + 256, 256, 80)]), EINVAL), (dict(parts=[(P, 256, 64), (P + 256, 256, 64)]), EINVAL)], ids=str)
def test_reorder_refusals(kw, want):
    assert reorder(kw.pop("parts", [(P, 64, 64)]), **kw) == want


def test_binding_refuses():
    with pytest.raises(B.RwkvqError):
        B.make_state_parts([])
    with pytest.raises(B.RwkvqError):
        B.make_state_parts([torch.zeros((4, 16))])           # not on the device
    x = torch.zeros((2, 10))
    with pytest.raises(B.RwkvqError) as e:
        B.rwkvq_beam_select(x, torch.zeros((1, 2)), torch.zeros((1, 2)), torch.zeros((1, 2), dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32))
    assert e.value.status == EINVAL
