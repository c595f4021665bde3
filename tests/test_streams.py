"""The torch stream that the binding prepares a workspace on."""
import pytest
import torch

import paper_2606_07684_amd as scd


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
