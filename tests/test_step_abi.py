"""The C ABI and the Python entry points of the operators around the decision
step: exported symbols, and every refusal, which happens on the host before a
device is touched (the addresses are never dereferenced)."""

import ctypes
import os
import re

import pytest
import torch

import paper_2608_26004_amd as asp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "asymspec_step.h")
FAKE = 1 << 20
ODD = FAKE + 2
VP, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t


class Shape(ctypes.Structure):
    """asymspec_shape."""
    _fields_ = ([(n, VP) for n in ("logits", "out")]
                + [(n, I64) for n in ("request_stride", "row_stride", "out_request_stride", "out_row_stride")]
                + [(n, VP) for n in ("history", "lengths", "prompt_lengths", "draft_tokens")] + [("draft_stride", I64)]
                + [(n, VP) for n in ("id_map", "repetition", "frequency", "presence", "bias_ids", "bias_values",
                                     "mask", "mask_index")]
                + [(n, ctypes.c_int32) for n in ("dtype", "B", "R", "V", "max_history", "D", "n_ids", "n_bias",
                                                 "n_masks")])


def library():
    lib = asp.load_library()
    lib.asymspec_shape_logits.argtypes = [ctypes.POINTER(Shape), VP]
    lib.asymspec_draw_workspace_size.argtypes = [I32, I32, I32]
    lib.asymspec_draw_workspace_size.restype = SZ
    lib.asymspec_draw_tokens.argtypes = [VP, I32, I32, I32, I64, VP, VP, I64, VP, I64, VP, I64, VP, SZ, VP]
    lib.asymspec_commit_tokens.argtypes = [VP, VP, VP, I64, VP, I32, VP, VP, VP, I32, VP, I32, I32, VP, VP, VP, VP, VP]
    lib.asymspec_plan_slots.argtypes = [VP, VP, VP, VP, I32, VP, VP, I32, VP, I32, I32, I32, I32, VP, VP, VP, VP, VP, VP]
    return lib


def test_library_exports_header_symbols():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(asymspec_[a-z_]+)\s*\(", src)))
    assert len(names) == 5
    for n in names:
        assert hasattr(library(), n), n


def test_struct_layout_matches_header():
    """The ctypes structure has the header's fields in the header's order."""
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct asymspec_shape \{(.*?)\} asymspec_shape;", src, re.S).group(1)
    names = re.findall(r"\*?\s*(\w+)\s*[,;]", body)
    assert names == [f[0] for f in Shape._fields_]


def shape_call(**over):
    kw = dict(logits=FAKE, out=FAKE, request_stride=300, row_stride=100, out_request_stride=300, out_row_stride=100,
              history=FAKE, lengths=FAKE, prompt_lengths=FAKE, draft_tokens=FAKE, draft_stride=2, id_map=None,
              repetition=FAKE, frequency=FAKE, presence=FAKE, bias_ids=FAKE, bias_values=FAKE, mask=FAKE,
              mask_index=FAKE, dtype=asp.FP32, B=4, R=3, V=100, max_history=50, D=2, n_ids=0, n_bias=5, n_masks=7)
    kw.update(over)
    return library().asymspec_shape_logits(ctypes.byref(Shape(**kw)), None)


@pytest.mark.parametrize("over,code", [
    (dict(logits=None), asp.E_ARG), (dict(out=None), asp.E_ARG), (dict(dtype=2), asp.E_ARG),
    (dict(B=0), asp.E_ARG), (dict(R=0), asp.E_ARG), (dict(R=65), asp.E_ARG), (dict(V=0), asp.E_ARG),
    (dict(V=1 << 30, R=1, B=1, D=0), asp.E_ARG), (dict(request_stride=1 << 55, out_request_stride=1 << 55), asp.E_ARG),
    # out of place, but not apart: a part of it, and the next rows
    (dict(out=FAKE + 400), asp.E_ARG), (dict(out=FAKE + 4 * 1199), asp.E_ARG), (dict(logits=FAKE + 4 * 1199), asp.E_ARG),
    (dict(lengths=None), asp.E_ARG), (dict(max_history=0), asp.E_ARG), (dict(max_history=1 << 20), asp.E_ARG),
    (dict(D=-1), asp.E_ARG), (dict(D=1), asp.E_ARG), (dict(D=65), asp.E_ARG), (dict(draft_stride=-1), asp.E_ARG),
    (dict(bias_values=None), asp.E_ARG), (dict(n_bias=1024), asp.E_ARG), (dict(n_bias=-1), asp.E_ARG),
    (dict(mask_index=None), asp.E_ARG), (dict(mask=None), asp.E_ARG), (dict(n_masks=-1), asp.E_ARG),
    (dict(id_map=FAKE, n_ids=-1), asp.E_ARG),
    # more threads than a launch has
    (dict(B=1 << 23, R=1, D=0), asp.E_ARG), (dict(B=1 << 10, R=1, D=0, V=1 << 26, request_stride=1 << 26,
                                                  out_request_stride=1 << 26), asp.E_ARG),
    # in place with other strides; rows of one tensor that overlap
    (dict(out_row_stride=101, out_request_stride=303), asp.E_ARG),
    (dict(row_stride=99, out_row_stride=99), asp.E_ARG),
    (dict(request_stride=200, out_request_stride=200), asp.E_ARG),
    (dict(request_stride=0, out_request_stride=0), asp.E_ARG),
    (dict(request_stride=-300, out_request_stride=-300), asp.E_ARG),
    (dict(out=FAKE * 2, row_stride=-1), asp.E_ARG),
    (dict(logits=ODD, out=ODD), asp.E_ALIGN), (dict(dtype=asp.BF16, logits=FAKE + 1, out=FAKE + 1), asp.E_ALIGN),
    (dict(history=ODD), asp.E_ALIGN), (dict(mask=ODD), asp.E_ALIGN), (dict(presence=ODD), asp.E_ALIGN),
    (dict(bias_values=ODD), asp.E_ALIGN), (dict(draft_tokens=ODD), asp.E_ALIGN),
])
def test_shape_refusals(over, code):
    assert shape_call(**over) == code


@pytest.mark.parametrize("over", [
    dict(), dict(dtype=asp.BF16, logits=ODD, out=ODD), dict(history=None, lengths=None, max_history=0),
    dict(draft_tokens=None, D=7), dict(D=64), dict(bias_ids=None, bias_values=None, n_bias=9),
    dict(mask=None, mask_index=None, n_masks=0), dict(B=1, request_stride=-5, out_request_stride=0),
    dict(R=1, D=0, row_stride=-9, out_row_stride=1),
    # rows outside requests: [R][B][V]
    dict(request_stride=100, row_stride=400, out_request_stride=100, out_row_stride=400),
    # right behind, and right ahead
    dict(out=FAKE + 4 * 1200), dict(logits=FAKE + 4 * 1200),
    # a repeated input row is fine out of place
    dict(out=FAKE * 2, request_stride=0, row_stride=0)])
def test_shape_accepts(over):
    """Valid calls pass the checks; with no GPU they end at the device."""
    if torch.cuda.is_available():
        pytest.skip("host-only check")
    assert shape_call(**over) == asp.E_DEVICE


def draw_call(**over):
    kw = dict(logits=FAKE, dtype=asp.BF16, N=3, V=5000, stride=5000, tau=FAKE, u=FAKE, us=1, token=FAKE, ts=1,
              prob=FAKE, ps=1, ws=FAKE, wsb=1 << 20)
    kw.update(over)
    return library().asymspec_draw_tokens(*kw.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(logits=None), asp.E_ARG), (dict(tau=None), asp.E_ARG), (dict(token=None), asp.E_ARG),
    (dict(ws=None), asp.E_ARG), (dict(dtype=9), asp.E_ARG), (dict(N=0), asp.E_ARG), (dict(V=0), asp.E_ARG),
    (dict(V=1 << 30), asp.E_ARG), (dict(N=1 << 30), asp.E_ARG),
    (dict(N=1 << 26, V=1, wsb=1 << 40), asp.E_ARG), (dict(stride=-1), asp.E_ARG),
    (dict(ts=0), asp.E_ARG), (dict(ps=0), asp.E_ARG), (dict(us=-1), asp.E_ARG),
    (dict(logits=FAKE + 1), asp.E_ALIGN), (dict(dtype=asp.FP32, logits=ODD), asp.E_ALIGN),
    (dict(prob=ODD), asp.E_ALIGN), (dict(ws=FAKE + 8), asp.E_ALIGN), (dict(wsb=32), asp.E_WORKSPACE),
])
def test_draw_refusals(over, code):
    assert draw_call(**over) == code


def test_draw_workspace_size():
    size = library().asymspec_draw_workspace_size
    assert size(1, 1, asp.FP32) > 0 and size(4, 100000, asp.BF16) == 4 * size(1, 100000, asp.BF16)
    assert size((1 << 26) - 5, 1024, 0) == ((1 << 26) - 5) * size(1, 1, 0)
    for bad in ((1 << 26, 5, 0), ((1 << 25), 1025, 0), (0, 5, 0), (1, 0, 0), (1, 1 << 30, 0), (1, 5, 2), (-1, 5, 0)):
        assert size(*bad) == 0


def commit_call(**over):
    kw = dict(acc=FAKE, nxt=FAKE, d=FAKE, ds=2, hist=FAKE, L=100, lens=FAKE, fin=FAKE, stops=FAKE, n_stop=2,
              maxl=FAKE, B=3, K=2, lo=FAKE, fo=FAKE, to=FAKE, co=FAKE)
    kw.update(over)
    return library().asymspec_commit_tokens(*kw.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(acc=None), asp.E_ARG), (dict(nxt=None), asp.E_ARG), (dict(d=None), asp.E_ARG), (dict(hist=None), asp.E_ARG),
    (dict(lens=None), asp.E_ARG), (dict(lo=None), asp.E_ARG), (dict(fo=None), asp.E_ARG), (dict(to=None), asp.E_ARG),
    (dict(co=None), asp.E_ARG), (dict(stops=None), asp.E_ARG), (dict(n_stop=-1), asp.E_ARG), (dict(B=0), asp.E_ARG),
    (dict(B=1 << 26), asp.E_ARG), (dict(K=-1), asp.E_ARG), (dict(K=64), asp.E_ARG), (dict(L=0), asp.E_ARG), (dict(ds=-1), asp.E_ARG),
    (dict(hist=ODD), asp.E_ALIGN), (dict(co=ODD), asp.E_ALIGN),
])
def test_commit_refusals(over, code):
    assert commit_call(**over) == code


def slots_call(**over):
    kw = dict(lens=FAKE, new=FAKE, rel=FAKE, table=FAKE, top=10, held=FAKE, ring=FAKE, N=100, state=FAKE, bs=16, B=3,
              width=2, total=0, slots=FAKE, starts=FAKE, short=FAKE, held_out=FAKE * 2, state_out=FAKE * 2)
    kw.update(over)
    return library().asymspec_plan_slots(*kw.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(lens=None), asp.E_ARG), (dict(table=None), asp.E_ARG), (dict(held=None), asp.E_ARG),
    (dict(ring=None), asp.E_ARG), (dict(state=None), asp.E_ARG), (dict(slots=None), asp.E_ARG),
    (dict(short=None), asp.E_ARG), (dict(held_out=None), asp.E_ARG), (dict(state_out=None), asp.E_ARG),
    (dict(B=0), asp.E_ARG), (dict(B=4097), asp.E_ARG), (dict(bs=0), asp.E_ARG), (dict(top=0), asp.E_ARG),
    (dict(N=0), asp.E_ARG), (dict(width=-1), asp.E_ARG), (dict(width=0), asp.E_ARG),
    (dict(width=0, total=5, new=None), asp.E_ARG), (dict(B=4096, top=1 << 19), asp.E_ARG),
    (dict(B=4096, width=1 << 19), asp.E_ARG), (dict(held_out=FAKE), asp.E_ARG), (dict(state_out=FAKE), asp.E_ARG),
    (dict(slots=FAKE + 4), asp.E_ALIGN), (dict(ring=ODD), asp.E_ALIGN), (dict(starts=ODD), asp.E_ALIGN),
])
def test_slots_refusals(over, code):
    assert slots_call(**over) == code


def test_valid_calls_end_at_the_device():
    if torch.cuda.is_available():
        pytest.skip("host-only check")
    assert draw_call() == draw_call(u=None, prob=None, ps=0) == asp.E_DEVICE
    assert draw_call(N=1, stride=-5, ts=0, ps=0, us=-1) == asp.E_DEVICE
    assert commit_call() == commit_call(K=0, d=None) == commit_call(stops=None, n_stop=0) == asp.E_DEVICE
    assert slots_call() == slots_call(new=None, rel=None, starts=None) == slots_call(width=0, total=7) == asp.E_DEVICE


def test_python_refusals():
    """Wrong shapes, types and pairings, and tensors that are not on a GPU."""
    x = torch.zeros(2, 3, 64)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)     # noqa: E731
    bad = [
        dict(logits=x.half()), dict(logits=x[0]), dict(logits=x.transpose(1, 2)), dict(logits=x, lengths=i(2)),
        dict(logits=x, history=i(2, 5)), dict(logits=x, history=i(2, 5), lengths=i(3)),
        dict(logits=x, history=i(2, 5).long(), lengths=i(2)), dict(logits=x, draft_tokens=i(2, 1)),
        dict(logits=x, bias_ids=i(2, 4)), dict(logits=x, bias_ids=i(2, 4), bias_values=torch.zeros(2, 5)),
        dict(logits=x, mask=i(4, 2)), dict(logits=x, mask=i(4, 3), mask_index=i(2, 3)),
        dict(logits=x, mask=i(4, 2), mask_index=i(2, 2)), dict(logits=x, repetition=torch.ones(3)),
        dict(logits=x, out=torch.zeros(2, 3, 63)), dict(logits=x, out=x.bfloat16()),
        dict(logits=x, history=i(5, 2).t(), lengths=i(2)), dict(logits=x)]
    for kw in bad:
        with pytest.raises((ValueError, TypeError)):
            asp.shape_logits(**kw)
    for args in ((x[0], torch.ones(3), torch.ones(3)), (x, torch.ones(2), torch.ones(2)),
                 (x[0].t(), torch.ones(64), torch.ones(64)), (x[0].double(), torch.ones(3), torch.ones(3))):
        with pytest.raises((ValueError, TypeError)):
            asp.draw_tokens(*args)
    with pytest.raises(ValueError):
        asp.commit_tokens(i(2), i(2), i(2, 3), i(2, 9), i(2))
    ok = dict(lengths=i(2), new_tokens=None, block_table=i(2, 4), n_blocks=i(2), free_ring=i(8), free_state=i(2),
              block_size=16)
    for kw in (dict(width=1), dict(), dict(width=1, total=2), dict(total=4), dict(width=0)):
        with pytest.raises(ValueError):
            asp.plan_slots(**ok, **kw)


def test_kernels_do_not_spill():
    path = os.path.join(ROOT, "paper_2608_26004_amd", "libasymspec.resources.txt")
    if not os.path.exists(path):
        pytest.skip("no build report")
    rows = [l.split() for l in open(path) if "asym_step" in l]
    assert len(rows) >= 10
    for r in rows:
        assert dict(x.split("=") for x in r[1:])["scratch"] == "0", r
