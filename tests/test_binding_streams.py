"""The stream that the binding hands to a call is the current one of the context's device, whatever device is current."""
import inspect
from types import SimpleNamespace

import pytest
import torch

import paper_2604_03425_amd.binding as binding

ONE = object()   # in a tensor's place


class _Library:
    """Takes any call and keeps its last argument, the stream."""

    def __getattr__(self, name):
        def call(*args):
            self.stream = args[-1].value
            return 0
        return call


LISTS = dict(limb_ids=[0], galois_elts=[1], evks=[ONE], evk_baby=[], evk_giant=[], evk_value=[], new_lens=[1], lens=[1], k_pages=[ONE], v_pages=[ONE],
             factors=[1])
NUMBERS = ("npoly", "galois_elt", "eval_domain", "B", "nlimbs", "dnum", "n1", "n2", "stride", "npt", "tokens", "in_limbs", "page_tokens", "k_limbs", "v_limbs",
           "window", "sinks", "bias", "squarings", "square", "eps", "start")
CALLS = [f for name, f in sorted(vars(binding).items()) if name.startswith("ckks_") and inspect.isfunction(f) and "_stream(" in inspect.getsource(f)]


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
def test_the_stream_is_of_the_contexts_device(call, monkeypatch):
    library = _Library()
    monkeypatch.setattr(binding, "_lib", library)
    monkeypatch.setattr(binding, "_ptr", lambda *a: SimpleNamespace(value=1))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: SimpleNamespace(cuda_stream=100 + (0 if device is None else device)))
    ctx = SimpleNamespace(handle=None, device=3, N=1024, nq=2, np_=1, params=SimpleNamespace(dnum=1))
    tensor = SimpleNamespace(numel=lambda: 1, element_size=lambda: 8)
    args = {}
    for name, p in inspect.signature(call).parameters.items():
        if p.default is not p.empty:
            continue
        args[name] = ctx if name == "ctx" else LISTS[name] if name in LISTS else 1 if name in NUMBERS else tensor
    call(**args)
    assert library.stream == 103


def test_every_call_that_enqueues_is_looked_at():
    assert len(CALLS) == 24
