"""Every call that takes a context runs on the context's device and, without a stream, on that device's current one, whichever device is current."""
import inspect
import types

import pytest
import torch

from paper_2508_12801_b200 import binding as ms

# calls on a context's buffers whose tensors may be left out here
CALLS = ["route_fwd", "dispatch", "combine", "route_bwd", "gate", "softtopk_fwd", "softtopk_bwd", "softtopk_bwd_aux", "aux_loss", "assign", "assign_iterative",
         "assign_top2_sinkhorn", "index_build", "combine_bwd", "gate_bwd", "check_internal", "test_raise_internal", "route_dispatch_host"]


@pytest.fixture
def seen(monkeypatch):
    """Two pretended devices, 0 the current one; what the C entry would have seen: (device, stream)."""
    state = types.SimpleNamespace(device=0, calls=[])

    class Switch:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.old, state.device = state.device, self.dev

        def __exit__(self, *exc):
            state.device = self.old
    monkeypatch.setattr(torch.cuda, "device", Switch)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: types.SimpleNamespace(cuda_stream=1000 + (state.device if dev is None else dev)))
    monkeypatch.setattr(ms, "_current_device", lambda: state.device)
    monkeypatch.setattr(ms, "_current_raw_stream", lambda dev: 1000 + dev)
    for name in CALLS:
        def entry(*args):
            state.calls.append((state.device, getattr(args[-1], "value", args[-1])))
            return 0
        monkeypatch.setattr(ms._lib, "maxscore_" + name, entry)
    return state


def call(name, dev, **kw):
    ctx = types.SimpleNamespace(handle=None, device_index=dev)
    fn = getattr(ms, name)
    args = []
    for p in list(inspect.signature(fn).parameters.values())[1:]:
        if p.default is inspect.Parameter.empty:
            args.append({"lam": 0.1, "sinkhorn_eps": 0.1, "sinkhorn_iters": 3, "dev": ms.DeviceBuffers()}.get(p.name))
    fn(ctx, *args, **kw)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("dev", [0, 1])
def test_device_and_stream(seen, name, dev):
    call(name, dev)
    assert seen.calls == [(dev, 1000 + dev)] and seen.device == 0


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_that_is_given(seen, name):
    call(name, 1, stream=types.SimpleNamespace(cuda_stream=77))
    call(name, 1, stream=78)
    assert seen.calls == [(1, 77), (1, 78)] and seen.device == 0


def test_no_call_is_left_out():
    """Whoever takes a context and a stream is here, or checks its tensors' device as well and is tested with them."""
    takes = {n for n, f in inspect.getmembers(ms, inspect.isfunction) if not n.startswith("_") and {"ctx", "stream"} <= set(inspect.signature(f).parameters)}
    checked = {n for n in takes if "_need(" in inspect.getsource(getattr(ms, n))}
    assert takes - checked == set(CALLS)
