"""What the binding of the token operators hands to the library, and what it refuses before (no device, no compute)."""
import pytest
import torch

from paper_2609_35115_b200 import binding


class OnDevice:
    """As much of a CUDA tensor as the binding looks at."""

    def __init__(self, *shape, dtype=torch.float32, index=0):
        self.shape, self.dtype, self.index, self.device, self.is_cuda = shape, dtype, index, f"cuda:{index}", True

    def get_device(self):
        return self.index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape[0] if len(self.shape) == 1 else self.shape[0] * self.shape[1]

    def stride(self, i):
        return self.shape[1] if i == 0 and len(self.shape) == 2 else 1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000


class Library:
    def __init__(self):
        self.calls = []

    def dc_sample_tokens(self, *args):
        self.calls.append(args)
        return 0


# the library launches on the current device: another device's addresses must not get there
@pytest.mark.parametrize("current", [0, 1, 2])
def test_logits_of_another_device_than_the_current_one_are_not_sampled(monkeypatch, current):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    logits, u, tokens = OnDevice(3, 100, index=1), OnDevice(3, index=1), OnDevice(3, dtype=torch.int32, index=1)
    if current == 1:
        assert binding.sample_tokens(logits, u, tokens=tokens, stream=0) is tokens and len(lib.calls) == 1
    else:
        with pytest.raises(ValueError, match="current device"):
            binding.sample_tokens(logits, u, tokens=tokens, stream=0)
        assert not lib.calls


class Rows(OnDevice):
    """A matrix whose rows are `apart` values apart."""

    def __init__(self, n, width, apart):
        super().__init__(n, width, dtype=torch.bfloat16)
        self.apart = apart

    def stride(self):
        return self.apart, 1


# the stride of a single row counts for nothing: it may be that of any matrix which the row was taken from
@pytest.mark.parametrize("n,apart,want", [(1, 260, 264), (1, 256, 256), (1, 3, 256), (1, 1000, 1000), (2, 260, 260), (2, 264, 264)])
def test_rows_of_a_single_token_lie_any_number_of_values_apart(n, apart, want):
    c = binding.TokenCache.__new__(binding.TokenCache)
    c.handle, c.dtype, c._index, c.head_dim, c.device = None, torch.bfloat16, 0, 64, "cuda:0"
    assert c._rows("q", Rows(n, 256, apart), 256, n) == (0x10000, want)
