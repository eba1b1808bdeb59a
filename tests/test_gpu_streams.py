"""The probe's calls on a stream of the caller's, without outputs given."""
import pytest

from gpu_helpers import to_device
from paper_2608_05780_gb300 import workloads as wl

pytestmark = pytest.mark.gpu


def _calls(ev, probe, qkv, stream):
    """Every call that makes its own outputs; the workspaces are returned to live until the caller has waited."""
    cfg = probe.cfg
    q, k, v = qkv
    shape = (probe.cu_seqlens, probe.n_vis, cfg.tokens_per_frame, cfg.tile)
    args = (q, k, v, *shape, probe.row_ptr, probe.col_idx)
    o, lse, ws = ev.evisel_probe_attention(*args, stream=stream, cross_frame=True)
    maps = ev.evisel_evidence_reduce(ws, cfg.hq, probe.n_vis, cfg.tokens_per_frame, len(probe.n_vis), accumulate=True,
                                     stream=stream)
    aif = ev.evisel_intra_frame_evidence(*args, o, lse, ws, accumulate=True, stream=stream)
    aff, eff = ev.evisel_cross_frame_evidence(*args, o, lse, ws, stream=stream)
    keep, uni, ws2 = ev.evisel_topp_mask(q, k, *shape, 16, 0.9, stream=stream)
    coarse = ev.evisel_coarse_evidence(q, k, *shape, 16, keep, ws2, stream=stream)
    return [o, lse, *maps, aif, aff, eff, keep, uni, *coarse], (ws, ws2)


def test_new_outputs_are_made_on_the_stream_of_the_call(cuda_lib):
    import torch
    probe = wl.make_probe(wl.CONFIGS["tiny"])
    qkv = to_device(probe)
    want, _ = _calls(cuda_lib, probe, qkv, None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)               # the current stream is busy for about 0.1 s
    got, held = _calls(cuda_lib, probe, qkv, side)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(want, got)):
        assert torch.equal(a, b), i
    for ws in held:
        assert cuda_lib.evisel_status(ws) == 0


@pytest.mark.parametrize("default", [False, True])
def test_streams_of_other_libraries_by_their_handle(cuda_lib, default):
    """An object with a ``cuda_stream`` only, the default stream's 0 among them, while the current stream is busy."""
    import torch

    class Handle:
        def __init__(self, cuda_stream):
            self.cuda_stream = cuda_stream

    probe = wl.make_probe(wl.CONFIGS["tiny"])
    qkv = to_device(probe)
    want, _ = _calls(cuda_lib, probe, qkv, None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    current = side if default else torch.cuda.current_stream()
    with torch.cuda.stream(current):
        torch.cuda._sleep(200_000_000)
        got, held = _calls(cuda_lib, probe, qkv, Handle(0 if default else side.cuda_stream))
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(want, got)):
        assert torch.equal(a, b), i
    for ws in held:
        assert cuda_lib.evisel_status(ws) == 0


def test_the_stream_that_tensors_are_made_on(cuda_lib):
    """What is current while a new tensor is made: the stream given, whatever kind of object it comes as."""
    import torch
    from paper_2608_05780_gb300._binding import _maker
    side = torch.cuda.Stream()

    def make(device):
        return torch.cuda.current_stream(device).cuda_stream

    for handle in (0, side.cuda_stream):
        given = type("Handle", (), {"cuda_stream": handle})()
        for current in (side, torch.cuda.Stream(), torch.cuda.default_stream()):
            with torch.cuda.stream(current):
                assert _maker(make, given)(device="cuda") == handle
                assert _maker(make, side)(device="cuda") == side.cuda_stream
                assert _maker(make, None)(device="cuda") == current.cuda_stream
