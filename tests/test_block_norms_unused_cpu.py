"""What a call of the norms around a block does not use is neither checked nor passed on."""
import pytest
import torch

CONTIGUOUS, SLICE = torch.zeros((2, 32)), torch.zeros((2, 96))[:, 32:64]
BAD = torch.zeros((1, 7), dtype=torch.float64)


@pytest.fixture
def sent(orch_lib, monkeypatch):
    """The binding up to its call, which notes the struct that it is given."""
    calls = []
    monkeypatch.setattr(orch_lib, "_stream_here", lambda stream, device, *others: others)

    class Library:
        @staticmethod
        def orch_op_block_norms(p, code, others):
            calls.append((orch_lib.BlockNorms.from_buffer_copy(p), others))
            return 0
    monkeypatch.setattr(orch_lib, "lib", Library)

    def run(*a, **kw):
        orch_lib.block_norms(*a, rows_per_batch=3, **kw)
        return calls.pop()
    return run


H, Y = torch.zeros((6, 32)), torch.zeros((6, 32), dtype=torch.bfloat16)


def test_gate_of_another_stride_without_a_block_that_ends(sent):
    """No y: gate is not used, so the rows' stride is that of shift and scale."""
    p, _ = sent(H, None, None, H.clone(), gate=CONTIGUOUS, shift=SLICE, scale=SLICE)
    assert p.mod_stride == 96 and p.shift == SLICE.data_ptr() and not p.gate


def test_shift_and_scale_of_another_stride_without_a_block_that_follows(sent):
    p, _ = sent(H, Y, H.clone(), None, gate=SLICE, shift=CONTIGUOUS, scale=CONTIGUOUS)
    assert p.mod_stride == 96 and p.gate == SLICE.data_ptr() and not p.shift and not p.scale


def test_unused_tensors_are_not_checked(orch_lib, sent):
    """Of any shape and type, as the norms that no block asks for."""
    weights = orch_lib.norm("rms", 1e-6, torch.zeros(7))
    p, others = sent(H, None, H.clone(), None, gate=BAD, shift=BAD, scale=BAD, post=weights, pre=weights)
    assert not p.gate and not p.shift and not p.scale and not p.post.weight and not p.pre.weight
    assert len(others) == 1         # (h_out's device alone)


def test_used_ones_are_checked(orch_lib, sent):
    for kw in (dict(y=Y, gate=BAD), dict(out=H.clone(), shift=BAD), dict(out=H.clone(), scale=BAD)):
        with pytest.raises(orch_lib.OrchError):
            sent(H, h_out=H.clone(), **kw)
    with pytest.raises(orch_lib.OrchError):         # one stride for what is used
        sent(H, Y, None, Y.clone(), gate=CONTIGUOUS, shift=SLICE)
