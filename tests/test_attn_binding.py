"""What the binding of the attention entry points passes on and refuses, on the
CPU: a stand-in tensor says that it is on the device, and no kernel runs."""
import pytest
import torch

from paper_2609_15030_amd import linattn as la


class OnDevice:
    """A host tensor that the binding takes for a device one."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def _rows(t, shape):
    return la._rows(OnDevice(t), t.dtype, shape)


@pytest.mark.parametrize("tokens,heads,dim", [(7, 2, 64), (2, 1, 128), (5, 8, 64)])
def test_tokens_expanded_from_one_are_refused(tokens, heads, dim):
    """Stride 0 would stand for packed rows, of which only the first is there."""
    one = torch.zeros((1, heads, dim), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        _rows(one.expand(tokens, heads, dim), (tokens, heads, dim))
    # heads expanded from one, and tokens that overlap by some of their heads
    if heads > 1:
        with pytest.raises(ValueError):
            _rows(one[:, :1].expand(1, heads, dim), (1, heads, dim))
        flat = torch.zeros(tokens * heads * dim, dtype=torch.bfloat16)
        with pytest.raises(ValueError):
            _rows(flat.as_strided((tokens, heads, dim), ((heads - 1) * dim, dim, 1)), (tokens, heads, dim))


def test_token_strides_that_are_passed_on():
    x = torch.zeros((6, 5, 64), dtype=torch.bfloat16)
    assert _rows(x, x.shape) == (x.data_ptr(), 0)
    part = x[:, 1:3]
    assert _rows(part, part.shape) == (part.data_ptr(), 320)
    every_other = x[::2]
    assert _rows(every_other, every_other.shape) == (x.data_ptr(), 640)
    one = x[:1, 1:3].expand(1, 2, 64)                 # one token: its stride is never used
    assert _rows(one, one.shape) == (part.data_ptr(), 0)
