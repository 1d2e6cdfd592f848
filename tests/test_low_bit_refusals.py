"""More refusals of the operators in few bits, before anything is launched: none of this needs a GPU.  What the binding asks of a tensor is
given by stand-ins, whose addresses are never followed."""
import pytest
import torch

from paper_2511_14450_b200 import hyperion as hyp
from tests import test_low_bit_args as args

E, CAP = args.E, args.CAP


class Stub:
    """What the binding asks of a CUDA tensor of this type and shape, without its memory."""
    device = "cuda:0"

    def __init__(self, dtype, *shape):
        self.dtype, self.shape, self._meta = dtype, torch.Size(shape), torch.empty(shape, dtype=dtype, device="meta")
        self.nbytes = self._meta.nbytes

    def get_device(self): return 0
    def is_contiguous(self): return True
    def dim(self): return len(self.shape)
    def stride(self): return self._meta.stride()
    def data_ptr(self): return args.P if self._meta.numel() else 0


def write_with(rope):
    i32 = torch.int32
    hyp.hyp_op_kv8_write((4, 2, 64), 0, Stub(torch.float32, 2, 512), Stub(torch.uint8, 3, 2, 2, 1088), Stub(i32, 2, 1), Stub(i32, 3), Stub(i32, 2), rope)


@pytest.mark.parametrize("shape", [(0, 32, 2), (), (5,), (0,), (5, 32), (5, 64, 2), (5, 32, 1)])
def test_rope_tables_of_no_or_other_positions(shape, monkeypatch):
    """An empty table is not the same as none: it must not leave the rows unrotated."""
    monkeypatch.setattr(hyp, "_launch", lambda *a: pytest.fail("launched"))
    args.refused(write_with, Stub(torch.float32, *shape))


def test_rope_tables_that_fit_reach_the_launch(monkeypatch):
    calls = []
    monkeypatch.setattr(hyp, "_launch", lambda *a: calls.append(a))
    write_with(Stub(torch.float32, 5, 32, 2))
    write_with(None)
    rope = [(a[11], a[12]) for a in calls]                       # the table's address and positions
    assert rope == [(args.P, 5), (None, 0)]


@pytest.mark.parametrize("hkv,pages,dpages", [(16, 1 << 26, 1 << 26), (32767, 32769, 1 << 26), (32767, 1 << 26, 32769), (64, 1 << 24, 1 << 24)])
def test_read_of_more_half_pages_than_31_bits_count(hkv, pages, dpages):
    """The warps' steps over a sequence's half pages would have wrapped around: refused by the sizes, whatever the lengths are."""
    assert args.call("hyp_op_kv8_read", shape=args.shape(hkv, hkv, 64), pages=pages, dpages=dpages) == CAP
    assert args.call("hyp_op_kv8_read", shape=args.shape(hkv, hkv, 64), pages=0, dpages=dpages) == E
