"""Tensors that are too small for what the eviction's calls write: refused before the library is called, by the native module and by ctypes alike."""
import pytest
import torch

from paper_2603_08453_amd import binding as lc
from tests.test_binding_args4 import B, H, M, T, Index, Stream, seen, t  # noqa: F401  (fixtures)


class Sized(Index):
    sizes = (B, H, M, T)                                     # sequences, KV heads, max_chunks, max_tokens


def _wide(b=B, h=H, rows=T, d=128):
    return torch.zeros(b, h, rows, d, dtype=torch.bfloat16)


def _narrow(b=B, h=H, rows=T + 1, stride=72):
    return torch.zeros(b, h, rows, stride, dtype=torch.uint8)[..., 2:70]


@pytest.mark.parametrize("index", [Index, Sized])
def test_a_destination_smaller_than_the_source(seen, t, index):  # noqa: F811
    keep = (t["keep"], t["bounds"], t["n"])
    rows = lambda *caches: lc.lc_evict_rows(index, *keep, *caches, stream=Stream)
    for short in (dict(rows=T - 1), dict(h=H - 1), dict(b=B - 1), dict(d=120)):
        with pytest.raises(AssertionError):
            rows(t["K"], t["V"], _wide(**short), _wide(**short))
    for short in (dict(rows=T - 1), dict(h=H - 1), dict(b=B - 1)):
        with pytest.raises(AssertionError):
            rows(t["K4"], t["V4"], _narrow(**short), _narrow(**short))
    assert seen == []
    rows(t["K"], t["V"], _wide(rows=T + 3), _wide(rows=T + 3))
    rows(t["K4"], t["V4"], _narrow(rows=T + 3), _narrow(rows=T + 3))
    assert [name for name, _ in seen] == ["evict_rows", "evict_rows4"]


def test_a_destination_smaller_than_the_index(seen, t):  # noqa: F811
    """Source and destination alike, both with fewer rows, heads or sequences than the index has room for."""
    keep = (t["keep"], t["bounds"], t["n"])
    for make in (_wide, _narrow):
        for short in (dict(rows=T - 1), dict(h=H - 1), dict(b=B - 1)):
            with pytest.raises(AssertionError):
                lc.lc_evict_rows(Sized, *keep, *(make(**short) for _ in range(4)), stream=Stream)
        # a source that has no rows behind the tokens there are is fine
        lc.lc_evict_rows(Sized, *keep, make(rows=T - 1), make(rows=T - 1), make(rows=T), make(rows=T), stream=Stream)
    assert [name for name, _ in seen] == ["evict_rows", "evict_rows4"]


def test_values_smaller_than_their_keys(seen, t):  # noqa: F811
    """The same strides, fewer rows: what the keys have room for would be read or written behind the values' end."""
    keep = (t["keep"], t["bounds"], t["n"])
    for K, V, K_to, V_to in ((t["K"], t["V"][:, :, :T - 1], t["Kb"], t["Vb"]), (t["K"], t["V"], t["Kb"], t["Vb"][:, :, :T - 1]), (t["K"], t["V"], t["Kb"], t["Vb"][:B - 1]),
                             (t["K4"], t["V4"][:, :, :T], t["K4b"], t["V4b"]), (t["K4"], t["V4"], t["K4b"], t["V4b"][:, :, :T])):
        with pytest.raises(AssertionError):
            lc.lc_evict_rows(Sized, *keep, K, V, K_to, V_to, stream=Stream)
    for call in (lambda: lc.lc_sparse_decode4(Sized, t["q"], t["K4"], t["V4"][:, :, :T], t["ids"], t["counts"], t["out"], t["ws"], stream=Stream),
                 lambda: lc.lc_append4(Sized, t["K4"], t["V4"][:, :, :T], t["row"], t["row"], stream=Stream)):
        with pytest.raises(AssertionError):
            call()
    assert seen == []
