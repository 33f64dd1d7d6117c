"""Sinks and windows that change nothing: the same bits as the launch without them, in every output."""
import ctypes

import pytest
import torch

from test_gpu_sinks import DEV, _inputs, plx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,Tkv", [(500, 500), (130, 700)])
@pytest.mark.parametrize("d", [64, 128])
def test_nothing_is_hidden(plx, dtype, T, Tkv, d):
    y = _inputs(2, 4, 2, T, Tkv, d, seed=9, dtype=dtype)
    tensors = [y[n] for n in "qrkv"]
    lib, outs = plx.load_library(), []

    def forward(window, sinks):
        """Without key ranges, which only the plain call may take."""
        o, vbar = torch.empty_like(y["q"]), torch.empty_like(y["q"])
        stats = torch.empty(2, 4, T, 2, dtype=torch.float32, device=DEV)
        a = plx.prefill_args(*tensors, o, y["scale"], window=window)
        a.vbar, a.row_stats = vbar.data_ptr(), stats.data_ptr()
        stream = torch.cuda.current_stream().cuda_stream
        call = lib.parallax_prefill(ctypes.byref(a), stream) if sinks is None else lib.parallax_prefill_sinks(ctypes.byref(a), sinks, stream)
        assert call == plx.PLX_OK
        return [o, vbar, stats]

    for window, sinks in ((0, None), (100, Tkv - 100), (100, Tkv), (Tkv, 3), (Tkv + 7, Tkv), (2**31 - 1, 1), (1, 2**31 - 1)):
        saved = forward(window, sinks)
        grads = plx.parallax_prefill_backward(*tensors, *saved, y["g"], y["scale"], window=window, sinks=sinks or 0)
        outs.append([*saved, *grads])
    for case, other in enumerate(outs[1:]):
        for name, a, b in zip(("o", "vbar", "row_stats", "dq", "dr", "dk", "dv"), outs[0], other):
            assert torch.equal(a, b), (case, name)
