"""The attention operators launch on the current device: tensors of another one are refused before anything is launched.  Without a GPU: the tensors say that
they are somewhere, and the library only counts its calls."""
from __future__ import annotations

import pytest

from paper_2412_17560_amd import binding

torch = pytest.importorskip("torch")


class On:
    """A contiguous tensor that says that it lies on a device."""

    is_cuda = True

    def __init__(self, device, dtype, *shape):
        self.number, self.dtype, self.shape = device, dtype, torch.Size(shape)
        self.device = torch.device("cuda", device)

    def get_device(self):
        return self.number

    def stride(self):
        return tuple(int(torch.tensor(self.shape[i + 1:]).prod()) for i in range(len(self.shape)))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append(name) or 0


HALF, INT, FLOAT = torch.float16, torch.int32, torch.float32


def calls(at):
    """Every operator with its tensors, each on the device that `at` names for its place."""
    def heads(i, n):
        return On(at(i), HALF, 3, n, 64)

    def ints(i, *shape):
        return On(at(i), INT, *shape)
    cache = binding.GqsaCache(0, 2, 64)
    yield 8, lambda: binding.gqsa_qk_norm_rotate(heads(0, 4), heads(1, 2), ints(2, 3), On(at(3), FLOAT, 9, 32, 2), On(at(4), HALF, 64), On(at(5), HALF, 64),
                                                 q_out=heads(6, 4), k_out=heads(7, 2))
    yield 5, lambda: binding.gqsa_cache_append(cache, heads(0, 2), heads(1, 2), ints(2, 2, 5), ints(3, 2), ints(4, 3))
    yield 5, lambda: binding.gqsa_cache_read(cache, ints(2, 2, 5), ints(3, 2), ints(4, 3), heads(0, 2), heads(1, 2))
    yield 5, lambda: binding.gqsa_cache_attend(cache, heads(0, 4), ints(1, 2, 5), ints(2, 2), ints(3, 3), out=heads(4, 4))
    yield 6, lambda: binding.gqsa_prompt_attend(heads(0, 4), heads(1, 2), heads(2, 2), ints(3, 3), ints(4, 3), out=heads(5, 4))


@pytest.mark.parametrize("current", [0, 1])
def test_tensors_of_another_device_are_refused(monkeypatch, current):
    library = Library()
    monkeypatch.setattr(binding, "_lib", lambda: library)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    other = 1 - current
    for n, (count, call) in enumerate(calls(lambda i: current)):
        call()
        assert len(library.calls) == n + 1
    library.calls.clear()
    for place in [None, *range(8)]:                    # all of them, or one
        for count, call in calls(lambda i: other if place in (None, i) else current):
            if place is None or place < count:
                with pytest.raises(ValueError):
                    call()
    assert library.calls == []
