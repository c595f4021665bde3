"""The torch stream that the binding prepares a workspace on."""
import pytest
import torch

import paper_2606_07684_amd as scd
from synth import workloads as W
from tests import parity_util as U


@pytest.mark.parametrize("given", [0, "default", 4096, "other"])
def test_stream_of_a_handle(monkeypatch, given):
    """Handle 0 is the default stream itself; any other is taken as it is."""
    class Made:
        def __init__(self, raw, device=None):
            self.cuda_stream, self.device = raw or 77, device  # torch makes a new stream of handle 0

    class Default:
        cuda_stream = 0

    monkeypatch.setattr(torch.cuda, "ExternalStream", Made)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Default())
    stream = Default() if given == "default" else Made(512) if given == "other" else given
    want = 0 if given in (0, "default") else 512 if given == "other" else given
    assert scd._torch_stream(stream, torch.device("cuda", 0)).cuda_stream == want


@pytest.mark.gpu
@pytest.mark.parametrize("as_handle", [False, True])
def test_workspace_is_cleared_on_the_default_stream(monkeypatch, as_handle):
    """A call that belongs to the default stream, made while another one is current."""
    cache = scd.PagedCache(*[torch.zeros(64, 2, 64, 64, dtype=torch.int8, device="cuda") for _ in "kv"],
                           *[torch.ones(64, 2, device="cuda") for _ in "kv"],
                           torch.arange(64, dtype=torch.int32, device="cuda").view(1, 64))
    batch = scd.Batch(1, None, torch.tensor([4000], dtype=torch.int32, device="cuda"))
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    out = torch.full_like(q, float("nan"))
    torch.cuda.synchronize()
    entered = []
    enter = torch.cuda.stream
    monkeypatch.setattr(torch.cuda, "stream", lambda s: entered.append(s.cuda_stream) or enter(s))
    default = torch.cuda.default_stream()
    side = torch.cuda.Stream()
    with enter(side):
        scd.scd_cache_attend(cache, batch, q, out, stream=0 if as_handle else default)
    default.synchronize()
    assert entered == [0]
    assert bool((out == 0).all())


@pytest.mark.gpu
def test_tensors_belong_to_the_stream_that_fills_them(monkeypatch):
    """Entry points that make their outputs or a workspace make them on the stream they are given: the allocator
    neither hands them memory that the current stream still uses, nor the workspace back to it too early."""
    from tests.test_gpu_fit import BRANCHES, _lam, _setup

    wl, dev = W.FIT_POS0_KEYS, torch.device("cuda")
    model, batch = U.model_of(wl), U.batch_of(wl, dev)
    _, a_in, b_in, rope = _setup(wl, "k", dev)
    calls = [lambda s: scd.scd_rope_table(model, 50, stream=s).buffer, lambda s: scd.scd_positions(batch, stream=s),
             lambda s: scd.scd_rotary_table(scd.Rotary(64, 1e4), 50, stream=s).buffer,
             lambda s: scd.fit_reuse(model, batch, rope, BRANCHES["k"], a_in, b_in, _lam(wl), stream=s)[0]]
    want = [call(None) for call in calls]
    torch.cuda.synchronize()
    side, made, empty = torch.cuda.Stream(), [], torch.empty

    def recorded(*args, **kwargs):
        made.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kwargs)

    monkeypatch.setattr(torch, "empty", recorded)
    for call, expected in zip(calls, want):
        made.clear()
        got = call(side)
        assert made and set(made) == {side.cuda_stream}
        side.synchronize()
        for x, y in zip(*((v if isinstance(v, list) else [v]) for v in (got, expected))):
            assert (x is None and y is None) or torch.equal(x, y)
