"""The Python binding of the operators around the decision step, on the CPU:
what it refuses, which the C entry points do not see, and what it leaves to
them.  Tensors that claim a device without having memory there (fake tensors)
go through its checks as those of a GPU do."""

import warnings

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2608_26004_amd as asp
from paper_2608_26004_amd import step

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-only check")


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    """(without a GPU there is no current stream to ask for)"""
    monkeypatch.setattr(step, "_raw_stream", lambda device: 0)


def fake(make):
    """The tensors that `make` makes, on a GPU that is not there."""
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with FakeTensorMode():
            return make(lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda"),
                        lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda"))


EMPTY = {
    "shape_logits": lambda i, f: (f(0, 3, 64),),
    "draw_tokens": lambda i, f: (f(0, 64), f(0), f(0)),
    "commit_tokens": lambda i, f: (i(0), i(0), i(0, 2), i(0, 9), i(0)),
    "plan_slots": lambda i, f: (i(0), None, i(0, 4), i(0), i(8), i(2), 16, 3),
}


@pytest.mark.parametrize("name", sorted(EMPTY))
def test_an_empty_batch_is_refused(name):
    with pytest.raises(asp.AsymSpecError) as e:
        getattr(asp, name)(*fake(EMPTY[name]))
    assert e.value.status == asp.E_ARG


@pytest.mark.parametrize("offset", [2, 3])
def test_an_empty_id_map_beside_logits_of_any_alignment(offset):
    """It maps nothing, wherever the bf16 rows begin: the call is valid and ends at
    the device, which is missing here."""
    x, ids = fake(lambda i, f: (f(2, 3, 80, dtype=torch.bfloat16)[..., offset:offset + 64], i(0)))
    with pytest.raises(asp.AsymSpecError) as e:
        asp.shape_logits(x, id_map=ids)
    assert e.value.status == asp.E_DEVICE


def test_what_is_no_tensor_is_refused():
    """TypeError, wherever it stands among the arguments."""
    i, f = (lambda *s: torch.zeros(*s, dtype=torch.int32)), torch.zeros
    commit, slots = [i(2), i(2), i(2, 3), i(2, 9), i(2)], [i(2), i(2), i(2, 4), i(2), i(8), i(2)]
    for bad in (None, [1, 2], 3.0):
        with pytest.raises(TypeError):
            asp.shape_logits(bad)
        with pytest.raises(TypeError):
            asp.draw_tokens(bad, f(2), f(2))
        for k in range(len(commit)):
            with pytest.raises(TypeError):
                asp.commit_tokens(*commit[:k], bad, *commit[k + 1:])
        for k in (0, 2, 3, 4, 5):
            with pytest.raises(TypeError):
                asp.plan_slots(*slots[:k], bad, *slots[k + 1:], 16, width=1)


def test_writing_to_a_tensor_that_requires_a_gradient_is_refused():
    """A gradient through it would be wrong without a word; without gradients, or
    on a detached one, the call goes on (here to the missing GPU)."""
    x, y = torch.zeros(2, 3, 64, requires_grad=True), torch.zeros(2, 3, 64)
    q = torch.zeros(6, requires_grad=True)
    t = torch.zeros(6, dtype=torch.int32)
    draw = (y.view(6, 64), torch.ones(6), torch.ones(6))
    for call in (lambda: asp.shape_logits(x), lambda: asp.shape_logits(x * 2), lambda: asp.shape_logits(y, out=x),
                 lambda: asp.draw_tokens(*draw, out=(t, q))):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="must be on the GPU"):
            call()
    for call in (lambda: asp.shape_logits(x.detach()), lambda: asp.shape_logits(x, out=y),
                 lambda: asp.draw_tokens(x[0], torch.ones(3), torch.ones(3))):
        with pytest.raises(ValueError, match="must be on the GPU"):
            call()


def test_lazily_negated_tensors_are_refused():
    """Their memory holds the values without the sign."""
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)     # noqa: E731
    x, one, neg = torch.zeros(2, 1, 64), torch.ones(2), torch._neg_view
    for call in (lambda: asp.shape_logits(neg(x)), lambda: asp.shape_logits(x, out=neg(x.clone())),
                 lambda: asp.shape_logits(x, presence=neg(one)), lambda: asp.draw_tokens(neg(x[:, 0]), one, one),
                 lambda: asp.draw_tokens(x[:, 0], neg(one), one), lambda: asp.draw_tokens(x[:, 0], one, neg(one)),
                 lambda: asp.draw_tokens(x[:, 0], one, one, out=(i(2), neg(one))),
                 lambda: asp.shape_logits(x, presence=torch._efficientzerotensor(2))):
        with pytest.raises(ValueError, match="negated"):
            call()


def test_slots_that_overlap_are_refused():
    """Every workgroup of plan_slots reads all requests while others already write:
    nothing that is written may overlap another tensor."""
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)     # noqa: E731
    B, top, N, W = 4, 4, 20, 2
    names = ["lengths", "new_tokens", "block_table", "n_blocks", "free_ring", "free_state", "release"]
    outs = ["slots", "short", "held", "state", "starts"]

    def call(packed, **over):
        a = dict(lengths=i(B), new_tokens=i(B), block_table=i(B, top), n_blocks=i(B), free_ring=i(N), free_state=i(2),
                 release=i(B), slots=torch.zeros(9 if packed else (B, W), dtype=torch.int64), short=i(B), held=i(B),
                 state=i(2), starts=i(B + 1))
        a.update(over)
        kw = {k: a[k] for k in names}
        own = {k: v for k, v in over.items() if k in outs}
        out = [a[k] for k in outs[:5 if packed else 4]] if own else None
        return lambda: asp.plan_slots(**kw, block_size=16, out=out, **({"total": 9} if packed else {"width": W}))

    room = i(400)
    at = lambda k, *s: room[k:k + int(np.prod(s))].view(*s)     # noqa: E731
    big = room.view(torch.int64)
    for packed in (False, True):
        bad = [dict(short=at(0, B), release=at(0, B)), dict(short=at(3, B), lengths=at(0, B)),
               dict(held=at(0, B), n_blocks=at(3, B)), dict(held=at(0, B), new_tokens=at(2, B)),
               dict(state=at(0, 2), free_state=at(1, 2)), dict(state=at(3, 2), lengths=at(0, B)),
               dict(block_table=at(0, B, top), free_ring=at(15, N)), dict(block_table=at(0, B, top), n_blocks=at(12, B)),
               dict(free_ring=at(0, N), free_state=at(18, 2)), dict(short=at(0, B), held=at(1, B)),
               dict(short=at(0, B), block_table=at(2, B, top)),
               dict(slots=big[:9] if packed else big[:8].view(B, W), lengths=at(15, B))]
        if packed:
            bad += [dict(starts=at(0, B + 1), lengths=at(4, B)), dict(starts=at(0, B + 1), short=at(4, B))]
        for over in bad:
            with pytest.raises(ValueError, match="overlap"):
                call(packed, **over)()
        # side by side, and inputs that are one tensor
        for over in (dict(short=at(0, B), held=at(B, B), state=at(2 * B, 2), starts=at(2 * B + 2, B + 1),
                          lengths=at(4 * B, B), n_blocks=at(5 * B, B)),
                     dict(lengths=at(0, B), new_tokens=at(0, B), release=at(0, B), n_blocks=at(0, B)),
                     dict(block_table=at(0, B, top), free_ring=at(B * top, N))):
            with pytest.raises(ValueError, match="must be on the GPU"):
                call(packed, **over)()
