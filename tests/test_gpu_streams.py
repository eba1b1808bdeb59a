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
