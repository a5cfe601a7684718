"""GPU tests of nsc_adapter_project and nsc_adapter_backward by every kernel that
their plan picks (layer_forms.py), against fp64."""
import pytest
import torch

from layer_forms import ADAPTER_FORMS
from test_gpu_adapter import SENTINEL, Rows, check_backward, check_forward, untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ADAPTER_FORMS, ids=str)
def test_every_form(form):
    r = Rows(*form[:5], dtype=form[5], pad=form[6], seed=sum(form[:5]))
    r.forward()
    check_forward(r)
    r.backward()
    check_backward(r)
    if form[6]:
        untouched(r, r.y, r.d)
        untouched(r, r.dx, r.k)


def test_more_adapters_than_listing_workgroups():
    """3,000 adapters (2,047 workgroups and one for the rest list their rows)."""
    r = Rows(700, 40, 24, 3, 3000, dtype="f32", order="mixed", seed=2)
    r.forward()
    check_forward(r)
    r.backward()
    check_backward(r)


@pytest.mark.parametrize("form", [(40, 640, 128, 16, 5), (700, 256, 320, 16, 5)], ids=str)
def test_overlapping_calls_write_everything(form):
    """Two calls on two streams, each with its own workspace, into outputs that
    were cleared before."""
    rs = [Rows(*form, seed=s) for s in (1, 2)]
    outs = [(r.y, r.dx, r.da, r.db) for r in rs]
    for r in rs:
        r.forward()
        r.backward()
    want = [[t.clone() for t in o] for o in outs]
    streams = [torch.cuda.Stream() for _ in rs]
    for _ in range(3):
        for o in outs:
            for t in o:
                t.fill_(SENTINEL)
        torch.cuda.synchronize()
        for r, s in zip(rs, streams):
            r.forward(stream=s)
            r.backward(stream=s)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(t, v) for t, v in zip(o, w))
