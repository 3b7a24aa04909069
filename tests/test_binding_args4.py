"""How the calls of the 4-bit cache and of the eviction marshal their arguments, without a GPU: the native module bound to stand-ins that record
what they are called with, and ctypes where there is no native module, which has to hand over the same."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_08453_amd import binding as lc

VP, INT, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
MOVE = (VP, VP, VP, VP, VP, INT, INT, INT, VP, VP, VP, INT, VP)
LOAD = (VP, VP, VP, VP, VP, INT, INT, INT, VP, VP, VP, INT, VP)
WEIGH = (VP, VP, VP, VP, VP, VP, INT, INT, VP, VP, VP)
ROWS = (VP, VP, VP, VP, VP, VP, VP, VP, VP, VP, VP, VP, VP)
SIGNATURES = {"cache4_store": MOVE, "cache4_load": LOAD, "sparse_decode4": (VP, VP, VP, VP, VP, VP, VP, INT, INT, VP, VP, VP, SZ, VP),
              "append4": (VP, VP, VP, VP, VP, VP, VP, VP), "weigh_chunks": WEIGH, "weigh_chunks4": WEIGH,
              "evict_select": (VP, VP, INT, INT, VP, VP, VP, VP, VP, SZ, VP), "evict_rows": ROWS, "evict_rows4": ROWS}
ARRAYS = {"cache4_store": {2: (ctypes.c_int64, 3), 10: (ctypes.c_int64, 3)}, "cache4_load": {2: (ctypes.c_int64, 3), 10: (ctypes.c_int64, 3)},
          "sparse_decode4": {4: (ctypes.c_int64, 3)}, "append4": {3: (ctypes.c_int64, 3)}, "weigh_chunks": {3: (ctypes.c_int64, 3)}, "weigh_chunks4": {3: (ctypes.c_int64, 3)},
          "evict_rows": {6: (ctypes.c_int64, 3), 9: (ctypes.c_int64, 3)}, "evict_rows4": {6: (ctypes.c_int64, 3), 9: (ctypes.c_int64, 3)}}
B, H, G, T, M = 3, 2, 2, 8, 5


class Stream:
    cuda_stream = 0x77


class Index:
    handle = ctypes.c_void_p(0x1000)
    address = 0x1000


def _recorder(seen, name):
    def record(*a):
        a = list(a)
        for i, (kind, n) in ARRAYS.get(name, {}).items():
            a[i] = list((kind * n).from_address(a[i]))
        if name.startswith("cache4"):
            for i in (3, 4):
                a[i] = a[i] and list((ctypes.c_int32 * a[5]).from_address(a[i]))
        if name == "append4":
            a[6] = a[6] and ctypes.string_at(a[6], B)
        seen.append((name, a))
        return 0
    return record


@pytest.fixture(params=["native", "ctypes"])
def seen(request, monkeypatch):
    got, keep = [], {}
    for name, sig in SIGNATURES.items():
        keep[name] = ctypes.CFUNCTYPE(INT, *sig)(_recorder(got, name))
    if request.param == "native":
        lc._fast().bind4(*(ctypes.cast(f, VP).value for f in keep.values()))
    else:
        class Library:
            pass
        library = Library()
        for name, f in keep.items():
            p = ctypes.CFUNCTYPE(INT, *SIGNATURES[name])(ctypes.cast(f, VP).value)
            p.argtypes = getattr(lc.lib(), "lc_" + name).argtypes
            setattr(library, "lc_" + name, p)
        monkeypatch.setattr(lc, "_fast_mod", lc._Unmarshalled)
        monkeypatch.setattr(lc, "lib", lambda: library)
    yield got
    monkeypatch.undo()
    lc._fast_mod = None                                      # (the next call binds the library again)
    lc._fast()


@pytest.fixture
def t():
    wide = lambda: torch.zeros(B, H, T, 128, dtype=torch.bfloat16)
    narrow = lambda: torch.zeros(B, H, T + 1, 72, dtype=torch.uint8)[..., 2:70]
    return dict(q=torch.zeros(B, H * G, 128, dtype=torch.bfloat16), K=wide(), V=wide(), K4=narrow(), V4=narrow(), K4b=narrow(), V4b=narrow(), Kb=wide(), Vb=wide(),
                ids=torch.zeros(B, H, M, dtype=torch.int32), counts=torch.zeros(B, H, dtype=torch.int32), out=torch.zeros(B, H * G, 128), lse=torch.zeros(B, H * G),
                ws=torch.zeros(256, dtype=torch.uint8), weights=torch.zeros(B, H, M), weights_to=torch.zeros(B, H, M), row=torch.zeros(B, H, 128, dtype=torch.bfloat16),
                keep=torch.zeros(B, M, dtype=torch.int32), bounds=torch.zeros(B, M + 1, dtype=torch.int32), n=torch.zeros(B, dtype=torch.int32), lens=torch.zeros(B, dtype=torch.int32))


S, S4 = [H * T * 128, T * 128, 128], [H * (T + 1) * 72, (T + 1) * 72, 72]


def test_store_and_load(seen, t):
    p = {k: v.data_ptr() for k, v in t.items()}
    lc.lc_cache4_store(t["K"], t["V"], t["K4"], t["V4"], stream=Stream)
    lc.lc_cache4_store(t["K"], t["V"], t["K4"], t["V4"], first=[1, 0, np.int64(4)], counts=np.array([2, 8, 0]), stream=Stream)
    lc.lc_cache4_load(t["K4"], t["V4"], t["K"], t["V"], first=torch.tensor([1, 0, 4]), counts=(2, 3, 0), stream=Stream)
    assert seen == [("cache4_store", [p["K"], p["V"], S, None, [8, 8, 8], B, H, 128, p["K4"], p["V4"], S4, T + 1, 0x77]),
                    ("cache4_store", [p["K"], p["V"], S, [1, 0, 4], [2, 8, 0], B, H, 128, p["K4"], p["V4"], S4, T + 1, 0x77]),
                    ("cache4_load", [p["K4"], p["V4"], S4, [1, 0, 4], [2, 3, 0], B, H, 128, p["K"], p["V"], S, T + 1, 0x77])]
    for bad in (dict(counts=[9, 0, 0]), dict(counts=[1, 1]), dict(first=[0])):
        with pytest.raises(AssertionError):
            lc.lc_cache4_store(t["K"], t["V"], t["K4"], t["V4"], stream=Stream, **bad)
    assert len(seen) == 3


def test_attention_append_and_weights(seen, t):
    p = {k: v.data_ptr() for k, v in t.items()}
    lc.lc_sparse_decode4(Index, t["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"], t["ws"], lse=t["lse"], stream=Stream)
    lc.lc_sparse_decode4(Index, t["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"], t["ws"], stream=Stream)
    lc.lc_append4(Index, t["K4"], t["V4"], t["row"], t["row"], stream=Stream)
    lc.lc_append4(Index, t["K4"], t["V4"], t["row"], t["row"], [0, 3, True], stream=Stream)
    lc.lc_weigh_chunks(Index, t["q"], t["K"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream)
    lc.lc_weigh_chunks4(Index, t["q"], t["K4"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream)
    d = [0x1000, p["q"], p["K4"], p["V4"], S4, p["ids"], p["counts"], M, H * G, p["out"]]
    assert seen == [("sparse_decode4", d + [p["lse"], p["ws"], 256, 0x77]), ("sparse_decode4", d + [None, p["ws"], 256, 0x77]),
                    ("append4", [0x1000, p["K4"], p["V4"], S4, p["row"], p["row"], None, 0x77]),
                    ("append4", [0x1000, p["K4"], p["V4"], S4, p["row"], p["row"], b"\0\1\1", 0x77]),
                    ("weigh_chunks", [0x1000, p["q"], p["K"], S, p["ids"], p["counts"], M, H * G, p["lse"], p["weights"], 0x77]),
                    ("weigh_chunks4", [0x1000, p["q"], p["K4"], S4, p["ids"], p["counts"], M, H * G, p["lse"], p["weights"], 0x77])]
    other = torch.zeros(B, H, T + 1, 68, dtype=torch.uint8)
    for call in (lambda: lc.lc_sparse_decode4(Index, t["q"], t["K4"], other, t["ids"], t["counts"], t["out"], t["ws"], stream=Stream),
                 lambda: lc.lc_append4(Index, t["K"], t["V"], t["row"], t["row"], stream=Stream),
                 lambda: lc.lc_weigh_chunks4(Index, t["q"], t["K"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream)):
        with pytest.raises(AssertionError):
            call()


def test_eviction(seen, t):
    p = {k: v.data_ptr() for k, v in t.items()}
    lc.lc_evict_select(Index, t["weights"], 100, np.int64(7), t["keep"], t["bounds"], t["n"], t["ws"], keep_lens=t["lens"], stream=Stream)
    lc.lc_evict_select(Index, t["weights"], 100, 0, t["keep"], t["bounds"], t["n"], t["ws"], stream=Stream)
    lc.lc_evict_rows(Index, t["keep"], t["bounds"], t["n"], t["K"], t["V"], t["Kb"], t["Vb"], weights=t["weights"], weights_to=t["weights_to"], stream=Stream)
    lc.lc_evict_rows(Index, t["keep"], t["bounds"], t["n"], t["K4"], t["V4"], t["K4b"], t["V4b"], stream=Stream)
    assert seen == [("evict_select", [0x1000, p["weights"], 100, 7, p["keep"], p["bounds"], p["n"], p["lens"], p["ws"], 256, 0x77]),
                    ("evict_select", [0x1000, p["weights"], 100, 0, p["keep"], p["bounds"], p["n"], None, p["ws"], 256, 0x77]),
                    ("evict_rows", [0x1000, p["keep"], p["bounds"], p["n"], p["K"], p["V"], S, p["Kb"], p["Vb"], S, p["weights"], p["weights_to"], 0x77]),
                    ("evict_rows4", [0x1000, p["keep"], p["bounds"], p["n"], p["K4"], p["V4"], S4, p["K4b"], p["V4b"], S4, None, None, 0x77])]
    with pytest.raises(AssertionError):
        lc.lc_evict_rows(Index, t["keep"], t["bounds"], t["n"], t["K"], t["V"], t["K4b"], t["V4b"], stream=Stream)


def test_halves_of_a_cache_with_other_types(seen, t):
    """Shapes and strides alike, a smaller or larger element: rows would be read behind the tensor's end."""
    bytes_, floats = torch.zeros(B, H, T, 128, dtype=torch.uint8), torch.zeros(B, H, T, 128)
    shorts = torch.zeros(B, H, T + 1, 72, dtype=torch.int16)[..., 2:70]
    keep = (t["keep"], t["bounds"], t["n"])
    for call in (lambda: lc.lc_cache4_store(t["K"], bytes_, t["K4"], t["V4"], stream=Stream),
                 lambda: lc.lc_cache4_load(t["K4"], shorts, t["K"], t["V"], stream=Stream),
                 lambda: lc.lc_sparse_decode4(Index, t["q"], t["K4"], shorts, t["ids"], t["counts"], t["out"], t["ws"], stream=Stream),
                 lambda: lc.lc_append4(Index, t["K4"], shorts, t["row"], t["row"], stream=Stream),
                 lambda: lc.lc_evict_rows(Index, *keep, t["K"], bytes_, t["Kb"], t["Vb"], stream=Stream),
                 lambda: lc.lc_evict_rows(Index, *keep, t["K"], t["V"], t["Kb"], bytes_, stream=Stream),
                 lambda: lc.lc_evict_rows(Index, *keep, floats, floats, floats, floats, stream=Stream),
                 lambda: lc.lc_evict_rows(Index, *keep, t["K4"], t["V4"], t["K4b"], shorts, stream=Stream)):
        with pytest.raises(AssertionError):
            call()
    assert seen == []


def test_other_threads_run_while_the_library_works(t):
    """The entry points replaced by the C library's usleep, whose argument is the handle: 200 ms in which another thread has to get on."""
    import threading
    usleep = ctypes.cast(ctypes.CDLL(None).usleep, VP).value
    lc._fast().bind4(*[usleep] * 9)

    class Sleep:
        handle = None
        address = 200_000
    try:
        for call in (lambda: lc.lc_sparse_decode4(Sleep, t["q"], t["K4"], t["V4"], t["ids"], t["counts"], t["out"], t["ws"], stream=Stream),
                     lambda: lc.lc_append4(Sleep, t["K4"], t["V4"], t["row"], t["row"], [1, 0, 0], stream=Stream),
                     lambda: lc.lc_weigh_chunks4(Sleep, t["q"], t["K4"], t["ids"], t["counts"], t["lse"], t["weights"], stream=Stream),
                     lambda: lc.lc_evict_select(Sleep, t["weights"], 5, 0, t["keep"], t["bounds"], t["n"], t["ws"], stream=Stream),
                     lambda: lc.lc_evict_rows(Sleep, t["keep"], t["bounds"], t["n"], t["K"], t["V"], t["Kb"], t["Vb"], stream=Stream)):
            ticks, done = [0], threading.Event()

            def tick():
                while not done.wait(0.001):
                    ticks[0] += 1
            thread = threading.Thread(target=tick)
            thread.start()
            before = ticks[0]
            call()
            got = ticks[0] - before
            done.set()
            thread.join()
            assert got >= 5
    finally:
        lc._fast_mod = None
        lc._fast()
