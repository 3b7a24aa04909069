"""Tensors that are too small for what the eviction's calls write: refused before the library is called, by the native module and by ctypes alike."""
import pytest
import torch

from paper_2603_08453_amd import binding as lc
from tests.test_binding_args4 import B, G, H, M, T, Index, Stream, seen, t  # noqa: F401  (fixtures)


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


# ------------------------------------------------------------------ tables that go by the index's room for chunks

def test_lists_and_weights_sized_by_the_chunks_there_are(seen, t):  # noqa: F811
    """The index has room for M chunks; tensors made for fewer would be written behind their ends."""
    f, i32 = (lambda *n: torch.zeros(*n)), (lambda *n: torch.zeros(*n, dtype=torch.int32))
    select = lambda **kw: lc.lc_evict_select(Sized, *(kw.get(k, t[k]) for k in ("weights",)), 10, 0, *(kw.get(k, t[k]) for k in ("keep", "bounds", "n")), t["ws"],
                                             keep_lens=kw.get("lens", t["lens"]), stream=Stream)
    for bad in (dict(weights=f(B, H, M - 1)), dict(weights=f(B, H - 1, M)), dict(weights=f(B, H, M + 1)), dict(weights=f(B, H, M).half()), dict(weights=f(B, M, H).transpose(1, 2)),
                dict(keep=i32(B, M - 1)), dict(keep=i32(B - 1, M)), dict(keep=i32(B, M + 1)), dict(keep=i32(B, M).long()), dict(keep=i32(M, B).t()),
                dict(bounds=i32(B, M)), dict(bounds=i32(B - 1, M + 1)), dict(bounds=i32(B, M + 1).short()), dict(n=i32(B - 1)), dict(n=i32(2 * B)[::2]), dict(lens=i32(B - 1))):
        with pytest.raises(AssertionError):
            select(**bad)
    rows = lambda **kw: lc.lc_evict_rows(Sized, *(kw.get(k, t[k]) for k in ("keep", "bounds", "n")), t["K"], t["V"], t["Kb"], t["Vb"],
                                         **{k: kw.get(k, t[k]) for k in ("weights", "weights_to")}, stream=Stream)
    for bad in (dict(weights=f(B, H, M - 1)), dict(weights_to=f(B, H, M - 1)), dict(weights_to=f(B, H - 1, M)), dict(weights_to=f(B, M, H).transpose(1, 2)),
                dict(keep=i32(B, M - 1)), dict(bounds=i32(B, M)), dict(n=i32(B - 1))):
        with pytest.raises(AssertionError):
            rows(**bad)
    for call, K in ((lc.lc_weigh_chunks, t["K"]), (lc.lc_weigh_chunks4, t["K4"])):
        for bad in (dict(weights=f(B, H, M - 1)), dict(weights=f(B, H, M + 1)), dict(weights=f(B - 1, H, M)), dict(weights=f(B, H, M).double()), dict(lse=f(B, H * G - 1)),
                    dict(lse=f(H * G, B).t()), dict(counts=i32(B, H - 1)), dict(counts=i32(B, H).long()), dict(ids=i32(B, H - 1, M)), dict(ids=i32(B, H, 2 * M)[:, :, ::2])):
            with pytest.raises(AssertionError):
                call(Sized, t["q"], K, *(bad.get(k, t[k]) for k in ("ids", "counts", "lse", "weights")), stream=Stream)
    assert seen == []


def test_tables_that_have_the_room(seen, t):  # noqa: F811
    """Flat ones, and ones with room for more sequences, as before."""
    more = torch.zeros(B + 1, H, M)
    lc.lc_evict_select(Sized, more, 10, 0, t["keep"].reshape(-1), t["bounds"], t["n"].reshape(B, 1), t["ws"], stream=Stream)
    lc.lc_evict_rows(Sized, t["keep"], t["bounds"], t["n"], t["K"], t["V"], t["Kb"], t["Vb"], weights=more, weights_to=t["weights_to"].reshape(-1), stream=Stream)
    lc.lc_evict_rows(Sized, t["keep"], t["bounds"], t["n"], t["K"], t["V"], t["Kb"], t["Vb"], stream=Stream)
    lc.lc_weigh_chunks(Sized, t["q"], t["K"], t["ids"], t["counts"], t["lse"].reshape(-1), more, stream=Stream)
    # a list's table may have less or more room than the index
    lc.lc_weigh_chunks4(Sized, t["q"], t["K4"], torch.zeros(B, H, 2, dtype=torch.int32), t["counts"], t["lse"], t["weights"], stream=Stream)
    assert [name for name, _ in seen] == ["evict_select", "evict_rows", "evict_rows", "weigh_chunks", "weigh_chunks4"]


# ------------------------------------------------------------------ types

def test_other_types_than_bfloat16(seen, t):  # noqa: F811
    """float16 has as many bytes: its bits would be taken for bfloat16's."""
    half = {k: t[k].half() for k in ("q", "K", "V", "row")}
    wide = {k: t[k].float() for k in ("q", "row")}
    for call in (lambda: lc.lc_cache4_store(half["K"], half["V"], t["K4"], t["V4"], stream=Stream),
                 lambda: lc.lc_cache4_store(t["K"], half["V"], t["K4"], t["V4"], stream=Stream),
                 lambda: lc.lc_cache4_load(t["K4"], t["V4"], half["K"], half["V"], stream=Stream),
                 lambda: lc.lc_sparse_decode4(Index, half["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"], t["ws"], stream=Stream),
                 lambda: lc.lc_sparse_decode4(Index, wide["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"], t["ws"], stream=Stream),
                 lambda: lc.lc_append4(Index, t["K4"], t["V4"], half["row"], t["row"], stream=Stream),
                 lambda: lc.lc_append4(Index, t["K4"], t["V4"], t["row"], wide["row"], stream=Stream),
                 lambda: lc.lc_weigh_chunks(Index, t["q"], half["K"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream),
                 lambda: lc.lc_weigh_chunks(Index, half["q"], t["K"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream),
                 lambda: lc.lc_weigh_chunks4(Index, wide["q"], t["K4"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream)):
        with pytest.raises(AssertionError):
            call()
    assert seen == []
    # bfloat16 bits in another type's clothes are bfloat16 bits
    bits = {k: t[k].view(torch.int16) for k in ("q", "K", "V", "row")}
    lc.lc_cache4_store(bits["K"], bits["V"], t["K4"], t["V4"], stream=Stream)
    lc.lc_sparse_decode4(Index, bits["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"], t["ws"], stream=Stream)
    lc.lc_append4(Index, t["K4"], t["V4"], bits["row"], bits["row"], stream=Stream)
    lc.lc_weigh_chunks(Index, bits["q"], bits["K"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream)
    assert [name for name, _ in seen] == ["cache4_store", "sparse_decode4", "append4", "weigh_chunks"]


# ------------------------------------------------------------------ attention, lazy update

def test_attention_into_tensors_that_are_too_small(seen, t):  # noqa: F811
    f, i32, bf = (lambda *n: torch.zeros(*n)), (lambda *n: torch.zeros(*n, dtype=torch.int32)), (lambda *n: torch.zeros(*n, dtype=torch.bfloat16))
    attend = lambda **kw: lc.lc_sparse_decode4(Sized, *(kw.get(k, t[k]) for k in ("q", "K4", "V4", "ids", "counts", "out")), t["ws"], lse=kw.get("lse", t["lse"]), stream=Stream)
    for bad in (dict(out=f(B, H * G - 1, 128)), dict(out=f(B - 1, H * G, 128)), dict(out=f(B, H * G, 128).half()), dict(out=f(B, H * G, 256)[..., ::2]), dict(lse=f(B, H * G - 1)),
                dict(q=bf(B - 1, H * G, 128)), dict(q=bf(H * G, B, 128).transpose(0, 1)), dict(ids=i32(B, H - 1, M)), dict(ids=i32(B, H, 2 * M)[:, :, ::2]),
                dict(counts=i32(B, H - 1)), dict(K4=_narrow(b=B - 1), V4=_narrow(b=B - 1)), dict(K4=_narrow(h=H - 1), V4=_narrow(h=H - 1))):
        with pytest.raises(AssertionError):
            attend(**bad)
    for call, K in ((lc.lc_weigh_chunks, _wide), (lc.lc_weigh_chunks4, _narrow)):
        for bad in (dict(q=bf(B - 1, H * G, 128)), dict(K=K(b=B - 1)), dict(K=K(h=H - 1))):
            with pytest.raises(AssertionError):
                call(Sized, bad.get("q", t["q"]), bad.get("K", K()), t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream)
    assert seen == []
    attend(out=f(B, H * G * 128), lse=f(B * H * G), q=bf(B, H * G, 1, 128))
    attend(K4=_narrow(rows=2), V4=_narrow(rows=2))           # (rows behind the tokens there are need not be)
    assert [name for name, _ in seen] == ["sparse_decode4"] * 2


def test_appending_to_a_cache_that_is_too_small(seen, t):  # noqa: F811
    bf = lambda *n: torch.zeros(*n, dtype=torch.bfloat16)
    append = lambda K, V, k=t["row"], v=t["row"]: lc.lc_append4(Sized, K, V, k, v, stream=Stream)
    for short in (dict(rows=T - 1), dict(h=H - 1), dict(b=B - 1)):
        with pytest.raises(AssertionError):
            append(_narrow(**short), _narrow(**short))
    for k in (bf(B, H - 1, 128), bf(B - 1, H, 128), bf(H, B, 128).transpose(0, 1), bf(B, H, 256)[..., ::2]):
        for new in ((k, t["row"]), (t["row"], k)):
            with pytest.raises(AssertionError):
                append(t["K4"], t["V4"], *new)
    assert seen == []
    append(_narrow(rows=T), _narrow(rows=T), bf(B, 1, H, 128), bf(B, H, 1, 128))
    assert [name for name, _ in seen] == ["append4"]


# ------------------------------------------------------------------ nothing to do

@pytest.mark.parametrize("native", [True, False])
def test_no_rows_to_store_or_load(native, monkeypatch):
    """Tensors without rows, which have no address: nothing is launched, no error."""
    if not native:
        monkeypatch.setattr(lc, "_fast_mod", lc._Unmarshalled)
    K, K4 = _wide(rows=0), torch.full((B, H, T, 68), 3, dtype=torch.uint8)
    for args in (dict(), dict(counts=[0] * B), dict(first=[T, 0, 1], counts=[0] * B)):
        lc.lc_cache4_store(K, K, K4, K4.clone(), stream=Stream, **args)
        lc.lc_cache4_load(K4, K4.clone(), K, K, stream=Stream, **args)
    assert (K4 == 3).all()
    for bad, code in ((dict(first=[T + 1, 0, 0]), lc.LC_ERR_CAPACITY), (dict(first=[-1, 0, 0]), lc.LC_ERR_INVALID_ARG)):
        with pytest.raises(lc.LycheeError) as e:
            lc.lc_cache4_store(K, K, K4, K4.clone(), stream=Stream, **bad)
        assert e.value.code == code


# ------------------------------------------------------------------ numbers beyond C's int

@pytest.mark.parametrize("given,want", [(2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32, 2 ** 31 - 1), (2 ** 40 + 3, 2 ** 31 - 1), (2 ** 80, 2 ** 31 - 1),
                                        (-1, -1), (-2 ** 32, -2 ** 31), (torch.tensor(9), 9), (7.9, 7)])
def test_tokens_to_keep_beyond_an_int(seen, t, given, want):  # noqa: F811
    """To keep 2^32 tokens is to keep them all, not none."""
    lc.lc_evict_select(Sized, t["weights"], given, given, t["keep"], t["bounds"], t["n"], t["ws"], stream=Stream)
    assert seen[0][1][2:4] == [want, want]


# ------------------------------------------------------------------ close flags

@pytest.mark.parametrize("call", ["lc_append", "lc_append4"])
def test_fewer_close_flags_than_sequences(t, monkeypatch, call):  # noqa: F811
    """Without the native module too, the library finds a flag for every sequence it takes; those not given are off."""
    got = []

    class Library:
        pass
    library = Library()
    setattr(library, call, lambda *a: got.append(bytes(a[6])) or 0)
    monkeypatch.setattr(lc, "_fast_mod", lc._Unmarshalled)
    monkeypatch.setattr(lc, "lib", lambda: library)
    for flags, want in (([1], b"\1"), ([0, 2, True], b"\0\1\1"), ([], b"")):
        if call == "lc_append":
            lc.lc_append(Sized, t["K"], t["V"], t["row"], t["row"], flags, t["ws"], stream=Stream)
        else:
            lc.lc_append4(Sized, t["K4"], t["V4"], t["row"], t["row"], flags, stream=Stream)
        assert got.pop() == want + bytes(1024 - len(want))


# ------------------------------------------------------------------ the same numbers in other shapes

def test_tables_in_other_shapes(seen, t):  # noqa: F811
    """What lies in memory as the library reads it is taken: heads split into groups, a longer table of a single row."""
    lc.lc_weigh_chunks(Sized, t["q"], t["K"], t["ids"], t["counts"], t["lse"].reshape(B, H, G), t["weights"].reshape(B * H, M), stream=Stream)
    lc.lc_sparse_decode4(Sized, t["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"].reshape(B, H, G, 128), t["ws"], lse=t["lse"].reshape(B, H, G), stream=Stream)

    class One(Index):
        sizes = (1, 1, M, T)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    lc.lc_evict_select(One, torch.zeros(1, 1, 3 * M), 10, 0, i32(1, 2 * M), i32(1, 2 * M + 1), i32(4), t["ws"], stream=Stream)
    assert [name for name, _ in seen] == ["weigh_chunks", "sparse_decode4", "evict_select"]
    with pytest.raises(AssertionError):                      # (of several rows a longer one would be read at the wrong places)
        lc.lc_sparse_decode4(Sized, t["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"], t["ws"], lse=torch.zeros(B, H * G + 1), stream=Stream)


def test_a_destination_larger_than_the_source(seen, t):  # noqa: F811
    for index in (Index, Sized):
        for make in (_wide, _narrow):
            lc.lc_evict_rows(index, t["keep"], t["bounds"], t["n"], make(), make(), make(b=B + 1, h=H + 1), make(b=B + 1, h=H + 1), stream=Stream)
    assert [name for name, _ in seen] == ["evict_rows", "evict_rows4"] * 2
