"""The C ABI and the Python entry points of the operators of a quantised paged cache:
exported symbols, and every refusal, which happens on the host before a device is
touched (the addresses are never dereferenced)."""

import ctypes
import math
import os
import re
import warnings

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2608_26004_amd as asp
from paper_2608_26004_amd import step

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "asymspec_cache.h")
FAKE = 1 << 30
VP, I32, I64, SZ, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="host-only check")


class Cache(ctypes.Structure):
    """asymspec_cache."""
    _fields_ = [(n, VP) for n in ("keys", "key_scales", "values", "value_scales")] + \
               [(n, I32) for n in ("blocks", "heads", "block_size", "dim", "bits")]


class Heads(ctypes.Structure):
    """asymspec_heads."""
    _fields_ = [("at", VP)] + [(n, I64) for n in ("request", "row", "head")]


class Rotate(ctypes.Structure):
    """asymspec_rotate."""
    _fields_ = [(n, Heads) for n in ("q", "k", "q_out", "k_out")] + \
               [("positions", VP), ("frequencies", VP), ("magnitude", F32)] + \
               [(n, I32) for n in ("every_row", "interleaved", "dtype", "B", "R", "q_heads", "k_heads", "dim", "n")]


class Attend(ctypes.Structure):
    """asymspec_attend."""
    _fields_ = [("cache", Cache), ("q", Heads)] + \
               [(n, VP) for n in ("out", "lse", "block_table", "lengths", "new_tokens")] + [("scale", F32)] + \
               [(n, I32) for n in ("window", "dtype", "B", "R", "q_heads", "max_blocks")]


def library():
    lib = asp.load_library()
    lib.asymspec_rotate_heads.argtypes = [ctypes.POINTER(Rotate), VP]
    lib.asymspec_write_cache.argtypes = [ctypes.POINTER(Cache), ctypes.POINTER(Heads), ctypes.POINTER(Heads), I32, VP, I32,
                                         I32, VP]
    lib.asymspec_read_cache.argtypes = [ctypes.POINTER(Cache), VP, I32, VP, VP, I32, I32, I32, VP, VP, VP]
    lib.asymspec_attend_workspace_size.argtypes = [ctypes.POINTER(Attend)]
    lib.asymspec_attend_workspace_size.restype = SZ
    lib.asymspec_attend_cache.argtypes = [ctypes.POINTER(Attend), VP, SZ, VP]
    return lib


def test_library_exports_header_symbols():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(asymspec_[a-z_]+)\s*\(", src)))
    assert len(names) == 5
    for n in names:
        assert hasattr(library(), n), n


@pytest.mark.parametrize("name,struct", [("cache", Cache), ("heads", Heads), ("rotate", Rotate), ("attend", Attend)])
def test_struct_layouts_match_the_header(name, struct):
    """The ctypes structures have the header's fields in the header's order."""
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct asymspec_%s \{(.*?)\} asymspec_%s;" % (name, name), src, re.S).group(1)
    assert re.findall(r"\*?\s*(\w+)\s*[,;]", body) == [f[0] for f in struct._fields_]


# Three regions far apart, and what a valid call looks like.
def cache(**over):
    kw = dict(keys=FAKE * 10, key_scales=FAKE * 11, values=FAKE * 12, value_scales=FAKE * 13, blocks=8, heads=2, block_size=16,
              dim=64, bits=4)
    kw.update(over)
    return Cache(**kw)


def heads(at=FAKE, request=1200, row=300, head=100):
    return Heads(at, request, row, head)


CACHE_REFUSALS = [
    (dict(keys=None), asp.E_ARG), (dict(key_scales=None), asp.E_ARG), (dict(values=None), asp.E_ARG),
    (dict(value_scales=None), asp.E_ARG), (dict(blocks=0), asp.E_ARG), (dict(heads=0), asp.E_ARG),
    (dict(heads=4097), asp.E_ARG), (dict(block_size=0), asp.E_ARG), (dict(dim=0), asp.E_ARG), (dict(dim=48), asp.E_ARG),
    (dict(dim=288), asp.E_ARG), (dict(bits=16), asp.E_ARG), (dict(bits=3), asp.E_ARG), (dict(blocks=1 << 26), asp.E_ARG),
    (dict(keys=FAKE * 10 + 8), asp.E_ALIGN), (dict(key_scales=FAKE * 11 + 4), asp.E_ALIGN),
    (dict(values=FAKE * 12 + 1), asp.E_ALIGN), (dict(value_scales=FAKE * 13 + 2), asp.E_ALIGN),
]


def rotate_call(**over):
    kw = dict(q=heads(FAKE), k=heads(FAKE * 2), q_out=heads(FAKE * 3), k_out=heads(FAKE * 4), positions=FAKE * 5,
              frequencies=FAKE * 6, magnitude=1.0, every_row=0, interleaved=0, dtype=asp.BF16, B=4, R=4, q_heads=3, k_heads=2,
              dim=64, n=32)
    kw.update(over)
    return library().asymspec_rotate_heads(ctypes.byref(Rotate(**kw)), None)


@pytest.mark.parametrize("over,code", [
    (dict(q=heads(None)), asp.E_ARG), (dict(k=heads(None)), asp.E_ARG), (dict(q_out=heads(None)), asp.E_ARG),
    (dict(k_out=heads(None)), asp.E_ARG), (dict(positions=None), asp.E_ARG), (dict(frequencies=None), asp.E_ARG),
    (dict(dtype=2), asp.E_ARG), (dict(B=0), asp.E_ARG), (dict(R=0), asp.E_ARG), (dict(q_heads=0), asp.E_ARG),
    (dict(k_heads=-1), asp.E_ARG), (dict(q_heads=4095), asp.E_ARG), (dict(dim=1, n=1), asp.E_ARG), (dict(n=0), asp.E_ARG),
    (dict(n=33), asp.E_ARG), (dict(dim=1026), asp.E_ARG), (dict(B=1 << 30, R=2), asp.E_ARG),
    (dict(q=heads(request=-1)), asp.E_ARG), (dict(k=heads(FAKE * 2, row=-1)), asp.E_ARG),
    (dict(q=heads(head=1 << 41)), asp.E_ARG),
    # heads of an output that share channels
    (dict(q_out=heads(FAKE * 3, head=63)), asp.E_ARG), (dict(q_out=heads(FAKE * 3, row=200)), asp.E_ARG),
    (dict(k_out=heads(FAKE * 4, request=0)), asp.E_ARG),
    # in place with other strides, and not quite in place
    (dict(q_out=heads(FAKE, row=301)), asp.E_ARG), (dict(q_out=heads(FAKE + 128)), asp.E_ARG),
    # an output over the other's tensors, or over the tables
    (dict(q_out=heads(FAKE * 2)), asp.E_ARG), (dict(k_out=heads(FAKE * 3)), asp.E_ARG), (dict(k_out=heads(FAKE)), asp.E_ARG),
    (dict(q_out=heads(FAKE * 5)), asp.E_ARG), (dict(k_out=heads(FAKE * 6 - 64)), asp.E_ARG),
    # one projection: keys that begin in the queries' last head, or end in the next row's first
    (dict(q=heads(row=300), q_out=heads(row=300), k=heads(FAKE + 2 * 263, row=300), k_out=heads(FAKE + 2 * 263, row=300)), asp.E_ARG),
    (dict(q=heads(), q_out=heads(), k=heads(FAKE + 2 * 264, head=10), k_out=heads(FAKE * 4)), asp.E_ARG),
    (dict(q=heads(FAKE + 1)), asp.E_ALIGN), (dict(dtype=asp.FP32, k=heads(FAKE * 2 + 2)), asp.E_ALIGN),
    (dict(positions=FAKE * 5 + 2), asp.E_ALIGN), (dict(frequencies=FAKE * 6 + 4), asp.E_ALIGN),
])
def test_rotate_refusals(over, code):
    assert rotate_call(**over) == code


@no_gpu
@pytest.mark.parametrize("over", [
    dict(), dict(k=heads(None), k_out=heads(None), k_heads=0), dict(q_out=heads(FAKE), k_out=heads(FAKE * 2)),
    dict(every_row=1, interleaved=1, n=7), dict(q=heads(FAKE + 2), q_out=heads(FAKE * 3 + 2)),
    dict(B=1, q_out=heads(FAKE * 3, request=-5)), dict(q=heads(request=0, row=0, head=0)),
    # parts of one projection, in place: rows of [q | k], of requests; rows outside requests
    dict(q=heads(row=500, request=2000), q_out=heads(row=500, request=2000),
         k=heads(FAKE + 2 * 264, row=500, request=2000), k_out=heads(FAKE + 2 * 264, row=500, request=2000)),
    dict(k=heads(row=500, request=2000), k_out=heads(row=500, request=2000),
         q=heads(FAKE + 2 * 164, row=500, request=2000), q_out=heads(FAKE + 2 * 164, row=500, request=2000)),
    dict(q=heads(row=2000, request=500), q_out=heads(row=2000, request=500),
         k=heads(FAKE + 2 * 264, row=2000, request=500), k_out=heads(FAKE + 2 * 264, row=2000, request=500)),
    # heads outside rows
    dict(q=heads(request=2000, row=64, head=256), q_out=heads(request=2000, row=64, head=256),
         k=heads(FAKE + 2 * 768, request=2000, row=64, head=256), k_out=heads(FAKE + 2 * 768, request=2000, row=64, head=256)),
])
def test_rotate_accepts(over):
    """Valid calls pass the checks; with no GPU they end at the device."""
    assert rotate_call(**over) == asp.E_DEVICE


def write_call(c=None, **over):
    kw = dict(k=heads(FAKE), v=heads(FAKE * 2), dtype=asp.BF16, slots=FAKE * 3, B=4, R=4)
    kw.update(over)
    return library().asymspec_write_cache(ctypes.byref(cache(**(c or {}))), ctypes.byref(kw["k"]), ctypes.byref(kw["v"]),
                                          kw["dtype"], kw["slots"], kw["B"], kw["R"], None)


@pytest.mark.parametrize("over,code", CACHE_REFUSALS)
def test_write_refuses_the_cache(over, code):
    assert write_call(over) == code


@pytest.mark.parametrize("over,code", [
    (dict(k=heads(None)), asp.E_ARG), (dict(v=heads(None)), asp.E_ARG), (dict(slots=None), asp.E_ARG), (dict(dtype=5), asp.E_ARG),
    (dict(B=0), asp.E_ARG), (dict(R=0), asp.E_ARG), (dict(B=1 << 30, R=2), asp.E_ARG), (dict(k=heads(head=-1)), asp.E_ARG),
    (dict(v=heads(FAKE * 2, row=1 << 41)), asp.E_ARG),
    # over the cache
    (dict(k=heads(FAKE * 10)), asp.E_ARG), (dict(v=heads(FAKE * 13 + 32)), asp.E_ARG), (dict(slots=FAKE * 12 + 8), asp.E_ARG),
    (dict(k=heads(FAKE + 1)), asp.E_ALIGN), (dict(dtype=asp.FP32, v=heads(FAKE * 2 + 2)), asp.E_ALIGN),
    (dict(slots=FAKE * 3 + 4), asp.E_ALIGN),
])
def test_write_refusals(over, code):
    assert write_call(**over) == code


def test_write_refuses_parts_of_a_cache_that_overlap():
    assert write_call(dict(values=FAKE * 10)) == asp.E_ARG
    assert write_call(dict(key_scales=FAKE * 10 + 16)) == asp.E_ARG


@no_gpu
def test_write_accepts():
    for over in (dict(), dict(k=heads(FAKE + 2)), dict(v=heads(FAKE)), dict(B=1, k=heads(request=-1)), dict(R=1, B=1 << 20)):
        assert write_call(**over) == asp.E_DEVICE
    for c in (dict(dim=32), dict(dim=256), dict(bits=8, dim=160), dict(block_size=1), dict(blocks=1 << 25, heads=1, block_size=63,
              keys=1 << 50, key_scales=1 << 51, values=1 << 52, value_scales=1 << 53)):
        assert write_call(c) == asp.E_DEVICE


def read_call(c=None, **over):
    kw = dict(table=FAKE, top=10, lengths=FAKE * 2, first=FAKE * 3, dtype=asp.BF16, B=3, width=40, k=FAKE * 4, v=FAKE * 5)
    kw.update(over)
    return library().asymspec_read_cache(ctypes.byref(cache(**(c or {}))), *kw.values(), None)


@pytest.mark.parametrize("over,code", CACHE_REFUSALS)
def test_read_refuses_the_cache(over, code):
    assert read_call(over) == code


@pytest.mark.parametrize("over,code", [
    (dict(table=None), asp.E_ARG), (dict(lengths=None), asp.E_ARG), (dict(k=None, v=None), asp.E_ARG), (dict(dtype=2), asp.E_ARG),
    (dict(B=0), asp.E_ARG), (dict(top=0), asp.E_ARG), (dict(width=0), asp.E_ARG), (dict(B=1 << 26), asp.E_ARG),
    (dict(width=2 ** 31 - 1), asp.E_ARG),
    (dict(k=FAKE * 5), asp.E_ARG), (dict(k=FAKE * 10), asp.E_ARG), (dict(v=FAKE * 13 - 16), asp.E_ARG), (dict(k=FAKE), asp.E_ARG),
    (dict(v=FAKE * 2), asp.E_ARG), (dict(v=FAKE * 3), asp.E_ARG),
    (dict(k=FAKE * 4 + 8), asp.E_ALIGN), (dict(v=FAKE * 5 + 2), asp.E_ALIGN), (dict(table=FAKE + 2), asp.E_ALIGN),
    (dict(lengths=FAKE * 2 + 1), asp.E_ALIGN), (dict(first=FAKE * 3 + 2), asp.E_ALIGN),
])
def test_read_refusals(over, code):
    assert read_call(**over) == code


@no_gpu
@pytest.mark.parametrize("over", [dict(), dict(first=None), dict(k=None), dict(v=None), dict(dtype=asp.FP32, width=1)])
def test_read_accepts(over):
    assert read_call(**over) == asp.E_DEVICE


def attend(c=None, **over):
    kw = dict(q=heads(FAKE), out=FAKE * 2, lse=FAKE * 3, block_table=FAKE * 4, lengths=FAKE * 5, new_tokens=FAKE * 6, scale=0.1,
              window=0, dtype=asp.BF16, B=4, R=3, q_heads=8, max_blocks=20)
    kw.update(over)
    return Attend(cache=cache(**(c or {})), **kw)


def attend_call(c=None, ws=FAKE * 7, wsb=1 << 29, **over):
    return library().asymspec_attend_cache(ctypes.byref(attend(c, **over)), ws, wsb, None)


@pytest.mark.parametrize("over,code", CACHE_REFUSALS + [(dict(dim=32), asp.E_ARG), (dict(dim=160), asp.E_ARG)])
def test_attend_refuses_the_cache(over, code):
    assert attend_call(over) == code


@pytest.mark.parametrize("over,code", [
    (dict(q=heads(None)), asp.E_ARG), (dict(out=None), asp.E_ARG), (dict(block_table=None), asp.E_ARG), (dict(lengths=None), asp.E_ARG),
    (dict(ws=None), asp.E_ARG), (dict(dtype=3), asp.E_ARG), (dict(B=0), asp.E_ARG), (dict(B=4097), asp.E_ARG), (dict(R=0), asp.E_ARG),
    (dict(R=65), asp.E_ARG), (dict(q_heads=7), asp.E_ARG), (dict(q_heads=0), asp.E_ARG), (dict(q_heads=130), asp.E_ARG),
    (dict(max_blocks=0), asp.E_ARG), (dict(max_blocks=(1 << 27) - 16), asp.E_ARG), (dict(max_blocks=1 << 26, B=4096), asp.E_ARG),
    (dict(window=-1), asp.E_ARG), (dict(q=heads(row=-1)), asp.E_ARG),
    (dict(out=FAKE), asp.E_ARG), (dict(lse=FAKE * 2 + 64), asp.E_ARG), (dict(ws=FAKE * 10), asp.E_ARG), (dict(ws=FAKE), asp.E_ARG),
    (dict(out=FAKE * 5), asp.E_ARG), (dict(lse=FAKE * 6), asp.E_ARG), (dict(out=FAKE * 4), asp.E_ARG), (dict(lse=FAKE * 13), asp.E_ARG),
    (dict(q=heads(FAKE + 1)), asp.E_ALIGN), (dict(out=FAKE * 2 + 8), asp.E_ALIGN), (dict(lse=FAKE * 3 + 2), asp.E_ALIGN),
    (dict(block_table=FAKE * 4 + 2), asp.E_ALIGN), (dict(new_tokens=FAKE * 6 + 2), asp.E_ALIGN), (dict(ws=FAKE * 7 + 8), asp.E_ALIGN),
    (dict(wsb=100), asp.E_WORKSPACE),
])
def test_attend_refusals(over, code):
    assert attend_call(**over) == code


@no_gpu
@pytest.mark.parametrize("over", [dict(), dict(lse=None, new_tokens=None), dict(window=2 ** 31 - 1), dict(q_heads=128, R=64),
                                  dict(q=heads(FAKE + 2)), dict(dtype=asp.FP32, c=dict(bits=8, dim=256)), dict(B=4096)])
def test_attend_accepts(over):
    assert attend_call(**over) == asp.E_DEVICE


def test_attend_workspace_size():
    def size(c=None, **over):
        return library().asymspec_attend_workspace_size(ctypes.byref(attend(c, q=heads(None), out=None, lse=None, block_table=None,
                                                                            lengths=None, new_tokens=None, **over)))
    assert 0 < size(B=1, max_blocks=1) < size() <= size(max_blocks=20000)
    assert library().asymspec_attend_workspace_size(None) == 0
    for bad in (dict(B=0), dict(R=65), dict(q_heads=3), dict(max_blocks=0)):
        assert size(**bad) == 0


def test_attend_workspace_has_room_for_whole_lines():
    """Workgroups' parts are read through caches whose lines hold 128 bytes, and must share none.
    They begin on a line, wherever a workspace begins (at a multiple of 16): 112 bytes ahead
    of them at most, and nothing but whole lines otherwise."""
    def size(c=None, **over):
        return library().asymspec_attend_workspace_size(ctypes.byref(attend(c, **over)))
    for c in (dict(), dict(dim=96, bits=8), dict(dim=128), dict(dim=192, bits=8), dict(dim=256)):
        for over in (dict(), dict(B=1, R=1, max_blocks=1), dict(R=64), dict(dtype=asp.FP32, max_blocks=1000)):
            assert size(c, **over) > 524288 + 112 and (size(c, **over) - 524288 - 112) % 128 == 0


def test_null_structures_are_refused():
    lib = library()
    assert lib.asymspec_rotate_heads(None, None) == asp.E_ARG
    assert lib.asymspec_attend_cache(None, FAKE, 1 << 20, None) == asp.E_ARG
    h = ctypes.byref(heads())
    assert lib.asymspec_write_cache(None, h, h, 0, FAKE * 3, 1, 1, None) == asp.E_ARG
    assert lib.asymspec_write_cache(ctypes.byref(cache()), None, h, 0, FAKE * 3, 1, 1, None) == asp.E_ARG
    assert lib.asymspec_read_cache(None, FAKE, 1, FAKE, None, 0, 1, 1, FAKE, FAKE, None) == asp.E_ARG


# ------------------------------------------------------------------ binding --
@pytest.fixture
def no_stream(monkeypatch):
    """(without a GPU there is no current stream to ask for)"""
    monkeypatch.setattr(step, "_raw_stream", lambda device: 0)


def fakes(device="cuda"):
    """Valid arguments of each call on a GPU that is not there."""
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with FakeTensorMode():
            def e(*s, dtype=torch.bfloat16):
                return torch.empty(*s, dtype=dtype, device=device)
            i = lambda *s: e(*s, dtype=torch.int32)     # noqa: E731
            u = lambda *s: e(*s, dtype=torch.uint8)     # noqa: E731
            c = (u(9, 2, 16, 32), u(9, 2, 16, 2), u(9, 2, 16, 32), u(9, 2, 16, 2))
            return dict(rotate_heads=[e(4, 3, 8, 64), e(4, 3, 2, 64), i(4), e(32, dtype=torch.float64)],
                        write_cache=[e(4, 3, 2, 64), e(4, 3, 2, 64), e(4, 3, dtype=torch.int64), c],
                        read_cache=[c, i(4, 7), i(4), 50], attend_cache=[e(4, 3, 8, 64), c, i(4, 7), i(4), i(4)])


NAMES = ["attend_cache", "read_cache", "rotate_heads", "write_cache"]


@no_gpu
@pytest.mark.parametrize("name", NAMES)
def test_valid_calls_pass_the_binding(name, no_stream):
    """They end behind it, at addresses that are not there or at the missing device."""
    with pytest.raises((asp.AsymSpecError, RuntimeError)) as e:
        getattr(asp, name)(*fakes()[name])
    assert getattr(e.value, "status", asp.E_DEVICE) in (asp.E_ARG, asp.E_DEVICE)


@no_gpu
@pytest.mark.parametrize("name", NAMES)
def test_what_is_no_tensor_is_refused(name, no_stream):
    args = fakes()[name]
    for k, a in enumerate(args):
        for bad in (None, [1, 2], 3.5):
            if (name, k, bad) in (("rotate_heads", 1, None), ("attend_cache", 4, None)):
                continue                                   # (may be left out)
            with pytest.raises(TypeError):
                getattr(asp, name)(*args[:k], bad, *args[k + 1:])
        if isinstance(a, tuple):
            for bad in (a[:3], a[:3] + (None,)):
                with pytest.raises(TypeError):
                    getattr(asp, name)(*args[:k], bad, *args[k + 1:])


@no_gpu
def test_wrong_tensors_are_refused(no_stream):
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        a = fakes()
        with FakeTensorMode():
            def e(*s, dtype=torch.bfloat16):
                return torch.empty(*s, dtype=dtype, device="cuda")
            i = lambda *s: e(*s, dtype=torch.int32)     # noqa: E731
            u = lambda *s: e(*s, dtype=torch.uint8)     # noqa: E731
            c = a["read_cache"][0]
            bad = {
                "rotate_heads": [(0, e(4, 3, 64)), (0, e(4, 3, 8, 64, dtype=torch.float16)), (0, e(4, 3, 8, 128)[..., ::2]),
                                 (1, e(4, 2, 2, 64)), (1, e(4, 3, 2, 32)), (1, e(4, 3, 2, 64, dtype=torch.float32)),
                                 (2, i(3)), (2, i(4, 2)), (2, e(4, dtype=torch.int64)), (2, i(8)[::2]),
                                 (3, e(32, dtype=torch.float32)), (3, e(33, dtype=torch.float64)),
                                 (3, e(4, 8, dtype=torch.float64)), (2, torch.empty(4, dtype=torch.int32))],
                "write_cache": [(0, e(4, 3, 3, 64)), (0, e(4, 3, 2, 32)), (0, e(12, 2, 64)), (0, e(4, 3, 2, 64, dtype=torch.float16)),
                                (1, e(4, 3, 2, 64, dtype=torch.float32)), (1, e(4, 3, 2, 128)[..., ::2]), (2, i(4, 3)),
                                (2, e(4, dtype=torch.int64)), (2, e(4, 3, 1, dtype=torch.int64)),
                                (3, (c[0], c[1], c[2], u(9, 2, 16, 1))), (3, (u(9, 2, 16, 48), c[1], u(9, 2, 16, 48), c[1])),
                                (3, (u(9, 2, 32, 32)[:, :, ::2],) + c[1:]), (3, c[:3] + (i(9, 2, 16, 2),)),
                                (3, c[:2] + (u(8, 2, 16, 32), c[3])), (3, (u(9, 2, 16, 0), u(9, 2, 16, 0)) * 2)],
                "read_cache": [(1, i(4)), (1, e(4, 7, dtype=torch.int64)), (2, i(3)), (3, 0), (3, -5), (1, i(4, 14)[:, ::2])],
                "attend_cache": [(0, e(4, 3, 7, 64)), (0, e(4, 3, 8, 32)), (0, e(12, 8, 64)), (0, e(4, 3, 8, 64, dtype=torch.float16)),
                                 (2, i(3, 7)), (3, i(3)), (4, i(5)), (4, e(4, dtype=torch.int64)), (0, e(4, 3, 8, 128)[..., ::2])],
            }
    for name, each in bad.items():
        for k, x in each:
            with pytest.raises((ValueError, TypeError)):
                getattr(asp, name)(*a[name][:k], x, *a[name][k + 1:])
    for kw in (dict(window=-1), dict(out=(1, 2)), dict(out=3), dict(return_lse=True, out=a["attend_cache"][0])):
        with pytest.raises((ValueError, TypeError)):
            asp.attend_cache(*a["attend_cache"], **kw)
    with pytest.raises(TypeError):
        asp.read_cache(*a["read_cache"], dtype=torch.float16)


@no_gpu
def test_empty_batches_are_refused(no_stream):
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        c = fakes()["read_cache"][0]
        with FakeTensorMode():
            def e(*s, dtype=torch.bfloat16):
                return torch.empty(*s, dtype=dtype, device="cuda")
            i = lambda *s: e(*s, dtype=torch.int32)     # noqa: E731
            none = tuple(torch.empty(0, 2, 16, n, dtype=torch.uint8, device="cuda") for n in (32, 2) * 2)
            calls = [("rotate_heads", [e(0, 3, 8, 64), None, i(0), e(32, dtype=torch.float64)]),
                     ("rotate_heads", [e(4, 3, 8, 64), e(4, 3, 0, 64), i(4), e(32, dtype=torch.float64)]),
                     ("rotate_heads", [e(4, 3, 8, 64), None, i(4), e(0, dtype=torch.float64)]),
                     ("write_cache", [e(0, 2, 64), e(0, 2, 64), e(0, dtype=torch.int64), c]),
                     ("write_cache", [e(4, 2, 64), e(4, 2, 64), e(4, dtype=torch.int64), none]),
                     ("read_cache", [c, i(0, 7), i(0), 5]), ("read_cache", [c, i(4, 0), i(4), 5]),
                     ("attend_cache", [e(0, 3, 8, 64), c, i(0, 7), i(0)]), ("attend_cache", [e(4, 0, 8, 64), c, i(4, 7), i(4)]),
                     ("attend_cache", [e(4, 3, 8, 64), c, i(4, 0), i(4)]), ("attend_cache", [e(4, 3, 0, 64), c, i(4, 7), i(4)])]
    for name, args in calls:
        with pytest.raises((asp.AsymSpecError, ValueError)) as err:
            getattr(asp, name)(*args)
        assert getattr(err.value, "status", asp.E_ARG) == asp.E_ARG, (name, err.value)


@no_gpu
def test_gradients_and_lazy_tensors_are_refused():
    x = torch.zeros(1, 1, 1, 64)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)     # noqa: E731
    f = asp.rotary_frequencies(64, device="cpu")
    w = x.clone().requires_grad_()
    c = asp.new_cache(1, 1, 1, 64, 8, device="cpu")
    with pytest.raises(ValueError, match="gradient"):
        asp.rotate_heads(x, None, i(1), f, out=w)
    with pytest.raises(ValueError, match="gradient"):
        asp.attend_cache(x, c, i(1, 1), i(1), out=w)
    for call in (lambda: asp.rotate_heads(torch._neg_view(x), None, i(1), f),
                 lambda: asp.write_cache(x, torch._neg_view(x), torch.zeros(1, 1, dtype=torch.int64), c),
                 lambda: asp.attend_cache(torch._neg_view(x), c, i(1, 1), i(1))):
        with pytest.raises(ValueError, match="negated"):
            call()
    with pytest.raises(ValueError, match="must be on the GPU"):
        asp.rotate_heads(x, None, i(1), f)
    with pytest.raises(ValueError, match="must be on the GPU"):
        asp.attend_cache(x, c, i(1, 1), i(1))


@no_gpu
@pytest.mark.parametrize("heads,dim", [(1, 32), (3, 64), (5, 256), (7, 96), (4096, 128)])
def test_read_limit_is_the_documented_one(heads, dim):
    """requests * ceil(width / floor(2048 / dim)) * heads below 2^24, also for heads that do not
    divide 2^24.  (Tensors on the CPU, which are refused behind the check.)"""
    c = asp.new_cache(1, heads, 1, dim, 8, device="cpu")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)     # noqa: E731
    for B in (1, 3):
        tiles = ((1 << 24) - 1) // heads // B
        width = tiles * (2048 // dim)
        with pytest.raises(ValueError, match="must be on the GPU"):
            asp.read_cache(c, i(B, 1), i(B), width)
        with pytest.raises(asp.AsymSpecError) as e:
            asp.read_cache(c, i(B, 1), i(B), width + 1)
        assert e.value.status == asp.E_ARG
    with pytest.raises(asp.AsymSpecError):
        asp.read_cache(c, i(B, 1), i(B), 2 ** 31 - 1)


# ------------------------------------------------------------------ helpers --
def test_new_cache():
    c = asp.new_cache(3, 2, 5, 96, 4, device="cpu")
    assert [tuple(t.shape) for t in c] == [(3, 2, 5, 48), (3, 2, 5, 3)] * 2
    assert [tuple(t.shape) for t in asp.new_cache(3, 2, 5, 96, 8, device="cpu")] == [(3, 2, 5, 96), (3, 2, 5, 3)] * 2
    for bad in (dict(bits=2), dict(dim=100), dict(dim=288), dict(dim=0), dict(blocks=0), dict(heads=0), dict(block_size=0),
                dict(blocks=1 << 30)):
        with pytest.raises(ValueError):
            asp.new_cache(**{**dict(blocks=3, heads=2, block_size=5, dim=96, bits=4, device="cpu"), **bad})


def test_rotary_frequencies():
    f = asp.rotary_frequencies(8, base=100.0, device="cpu")
    assert f.dtype == torch.float64
    for i in range(4):
        assert abs(f[i] - 100.0 ** (-i / 4)) < 1e-15
    assert torch.equal(asp.rotary_frequencies(8, base=100.0, stretch=4.0, device="cpu"), f / 4)
    g = asp.rotary_frequencies(8, base=100.0, stretch=4.0, kind="base", device="cpu")
    assert g[0] == 1 and abs(g[3] * 4 - f[3]) < 1e-15 and (g <= f).all()
    f = asp.rotary_frequencies(128, device="cpu")
    r = asp.rotary_frequencies(128, stretch=8.0, kind="ramp", context=4096, device="cpu")
    turns = f * 4096 / (2 * math.pi)
    # a whole index of rounding at either end of the ramp
    step_ = 10000.0 ** (2 / 128)
    assert torch.equal(r[turns > 32 * step_], f[turns > 32 * step_])
    assert torch.allclose(r[turns < 1 / step_], f[turns < 1 / step_] / 8, rtol=1e-15)
    assert (r.diff() < 0).all() and (r <= f).all() and (r >= f / 8 * (1 - 1e-15)).all()
    for bad in (dict(channels=7), dict(channels=0), dict(base=1.0), dict(stretch=0.0), dict(kind="other"),
                dict(channels=2, kind="base"), dict(kind="ramp", fast=1.0, slow=1.0)):
        with pytest.raises(ValueError):
            asp.rotary_frequencies(**{**dict(channels=64, device="cpu"), **bad})


@pytest.mark.parametrize("channels,base,stretch,context,fast,slow", [
    (128, 10000.0, 4.0, 65536, 32.0, 1.0), (128, 10000.0, 4.0, 131072, 32.0, 1.0), (128, 10000.0, 32.0, 1 << 20, 32.0, 1.0),
    (64, 10000.0, 8.0, 4096, 32.0, 1.0), (64, 500.0, 8.0, 1 << 22, 32.0, 1.0), (96, 10000.0, 4.0, 100, 32.0, 1.0),
    (128, 10000.0, 4.0, 6, 32.0, 1.0), (128, 10000.0, 4.0, 1, 32.0, 1.0), (32, 1000.0, 2.0, 4096, 1.001, 1.0)])
def test_a_ramp_of_any_context(channels, base, stretch, context, fast, slow):
    """Pairs that turn `fast` times and more stay, those that turn `slow` times and less are
    stretched, and the share falls by the same from index to index in between: also where the
    slowest pair still turns more than `slow` times, or none does so often."""
    f = [base ** (-2 * i / channels) for i in range(channels // 2)]
    got = asp.rotary_frequencies(channels, base=base, stretch=stretch, kind="ramp", context=context, fast=fast, slow=slow,
                                 device="cpu").tolist()
    turns = [x * context / (2 * math.pi) for x in f]
    # the ramp's ends as whole indices, of pairs that there need not be
    ratio = base ** (2 / channels)
    lo = max(0, math.floor(math.log(turns[0] / fast) / math.log(ratio)))
    hi = min(channels - 1, math.ceil(math.log(turns[0] / slow) / math.log(ratio)))
    for i, (x, y, t) in enumerate(zip(f, got, turns)):
        share = 0.0 if t <= slow else 1.0 if i <= lo else (hi - i) / (hi - lo)
        want = x * share + x / stretch * (1 - share)
        # a quotient, a difference, two products and a sum: 8 roundings of 2^-53, and the power's
        assert abs(y - want) <= 16 * 2.0 ** -53 * x, (i, y, want)
    for i, t in enumerate(turns):
        assert got[i] == f[i] or abs(got[i] - f[i]) <= 4 * 2.0 ** -53 * f[i] or t < fast
        assert abs(got[i] - f[i] / stretch) <= 4 * 2.0 ** -53 * f[i] or t > slow
