"""The operators on drafted tokens launch on the current device: tensors of another one are refused before anything is launched, and so are those of another shape or type.
Without a GPU: the tensors say that they are somewhere, and the library only counts its calls."""
from __future__ import annotations

import pytest

from paper_2412_17560_amd import binding
from test_attention_devices import FLOAT, HALF, INT, Library, On

torch = pytest.importorskip("torch")


def calls(at, shape=lambda i, s: s, dtype=lambda i, t: t):
    """Every operator with its tensors, each on the device that `at` names for its place, of the shape and type that the others make of its own."""
    def on(i, t, *s):
        return On(at(i), dtype(i, t), *shape(i, s))
    cache, verifier = binding.GqsaCache(0, 2, 64), binding.GqsaVerifier(0)

    def where(i):
        return on(i, INT, 2, 5), on(i + 1, INT, 2), on(i + 2, INT, 3)
    yield 12, lambda: binding.gqsa_cache_append_rotated(cache, on(0, HALF, 3, 4, 64), on(1, HALF, 3, 2, 64), on(2, HALF, 3, 2, 64), on(3, INT, 3), on(4, FLOAT, 9, 32, 2),
                                                        *where(5), on(8, HALF, 64), on(9, HALF, 64), q_out=on(10, HALF, 3, 4, 64), k_out=on(11, HALF, 3, 2, 64))
    yield 6, lambda: binding.gqsa_cache_attend_tree(cache, on(0, HALF, 3, 4, 64), *where(1), on(4, INT, 3, 1), out=on(5, HALF, 3, 4, 64))
    yield 5, lambda: binding.gqsa_cache_keep(cache, *where(0), on(3, INT, 3), on(4, INT, 2))
    yield 9, lambda: binding.gqsa_verify(verifier, on(0, FLOAT, 3, 50), on(1, INT, 3), on(2, FLOAT, 3), on(3, FLOAT, 2), on(4, INT, 3), on(5, INT, 3),
                                         path=on(6, INT, 3), out=on(7, INT, 3), accepted=on(8, INT, 2))
    yield 9, lambda: binding.gqsa_verify(verifier, on(0, FLOAT, 3, 50), on(1, INT, 3), on(2, FLOAT, 3), on(3, FLOAT, 2), on(4, INT, 3), draft=on(5, FLOAT, 3, 50),
                                         path=on(6, INT, 3), out=on(7, INT, 3), accepted=on(8, INT, 2))


@pytest.fixture
def library(monkeypatch):
    library = Library()
    monkeypatch.setattr(binding, "_lib", lambda: library)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    return library


@pytest.mark.parametrize("current", [0, 1])
def test_tensors_of_another_device_are_refused(monkeypatch, library, current):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
    for n, (count, call) in enumerate(calls(lambda i: current)):
        call()
        assert len(library.calls) == n + 1
    library.calls.clear()
    for place in [None, *range(12)]:                   # all of them, or one
        for count, call in calls(lambda i: 1 - current if place in (None, i) else current):
            if place is None or place < count:
                with pytest.raises(ValueError):
                    call()
    assert library.calls == []


def test_tensors_of_another_shape_or_type_are_refused(monkeypatch, library):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    other = {HALF: FLOAT, FLOAT: HALF, INT: torch.int64}
    for place in range(12):
        for kw in (dict(shape=lambda i, s: s + (1,) if i == place else s), dict(dtype=lambda i, t: other[t] if i == place else t)):
            for count, call in calls(lambda i: 0, **kw):
                if place < count:
                    with pytest.raises(ValueError):
                        call()
    for place in range(12):        # one row, sequence or element more (but of positions in a table, and of the rows that keep is told of by `path` alone)
        for number, (count, call) in enumerate(calls(lambda i: 0, shape=lambda i, s: (s[0] + 1,) + s[1:] if i == place else s)):
            if place < count and (number, place) not in ((0, 4), (2, 3)):
                with pytest.raises(ValueError):
                    call()
    assert library.calls == []
