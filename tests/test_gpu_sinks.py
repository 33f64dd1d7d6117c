"""GPU parity of causal attention with a sliding window and sinks, forward and backward (parallax_prefill /
parallax_prefill_backward with sinks=, through the C ABI), against the masked CPU oracle."""
import numpy as np
import pytest
import torch

from oracle import masked, rows
from parity import BF16_REL_L2, F32_MAX_REL, assert_gradient_close, host, max_rel, rel_l2

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def plx():
    from paper_2605_29157_amd import binding

    binding.load_library()
    assert torch.cuda.is_available()
    return binding


def _normal(shape, seed, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def _inputs(B, Hq, Hkv, T, Tkv, d, seed, dtype=torch.bfloat16):
    return dict(q=_normal((B, Hq, T, d), seed, dtype), r=_normal((B, Hq, T, d), seed + 1, dtype),
                k=_normal((B, Hkv, Tkv, d), seed + 2, dtype), v=_normal((B, Hkv, Tkv, d), seed + 3, dtype),
                g=_normal((B, Hq, T, d), seed + 4, dtype), scale=d ** -0.5)


def _see(T, Tkv, window, sinks):
    pos = np.arange(T)[:, None] + (Tkv - T)
    j = np.arange(Tkv)[None, :]
    return (j <= pos) & ((j > pos - window) | (j < sinks))


def _check(plx, y, window, sinks, info=(), backward=True):
    T, Tkv = y["q"].shape[2], y["k"].shape[2]
    see = _see(T, Tkv, window, sinks)
    ins = [host(y[n]) for n in "qrkv"]
    f32 = y["q"].dtype == torch.float32
    want, vbar, ubar, lse = masked.masked_forward_with_cache(*ins, y["scale"], see)
    tensors = [y[n] for n in "qrkv"]
    got = plx.parallax_prefill(*tensors, y["scale"], window=window, sinks=sinks)
    o, vb, stats = plx.parallax_prefill(*tensors, y["scale"], window=window, sinks=sinks, save_for_backward=True)
    for x, name in ((got, "o"), (o, "o with the row cache")):
        x = host(x).astype(np.float64)
        assert np.isfinite(x).all(), info
        if f32:
            assert max_rel(x, want) <= F32_MAX_REL, info + (name,)
        else:
            assert rel_l2(x, want) <= BF16_REL_L2, info + (name,)
            bound = rows.bf16_bound(*ins, y["scale"], see)
            assert (np.abs(x - want) <= bound).all(), info + (name, float((np.abs(x - want) / bound).max()))
    tol = F32_MAX_REL if f32 else BF16_REL_L2
    assert rel_l2(host(vb), vbar) <= tol, info
    # (scores of N(0, 1) vectors, fp32 sums of bf16 products: 2^-24 of sums of up to 256 products of size ~1, and exp2, log2)
    np.testing.assert_allclose(host(stats)[..., 0] * np.log(2), lse, rtol=0, atol=1e-4, err_msg=str(info))
    np.testing.assert_allclose(host(stats)[..., 1], ubar, rtol=0, atol=1e-3, err_msg=str(info))
    if not backward:
        return
    grads = plx.parallax_prefill_backward(*tensors, o, vb, stats, y["g"], y["scale"], window=window, sinks=sinks)
    ref = masked.masked_backward(*ins, host(y["g"]), y["scale"], see)
    # (rows of very few keys: o in bf16 moves tau, and dQ, dR are differences that may cancel, so there is no bound
    # relative to the gradient)
    bounds = rows.bf16_backward_bound(*ins, host(y["g"]), y["scale"], see, *([64 * 2.0 ** -24] if f32 else []))
    for name, a, b, bound in zip(("dq", "dr", "dk", "dv"), grads, ref, bounds):
        err = np.abs(host(a).astype(np.float64) - b)
        assert (err <= bound).all(), info + (name, float((err / np.maximum(bound, 1e-300)).max()))


# window, sinks: sinks inside a tile, at its edge, over several; windows shorter than a tile, that meet the sinks, of one key
WS = [(1, 1), (16, 4), (33, 64), (64, 1), (100, 33), (128, 128), (129, 70), (257, 200), (300, 65), (500, 4), (20, 300),
      (5000, 4), (90, 5000)]


@pytest.mark.parametrize("window,sinks", WS)
@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 130, 300, 700])
def test_square(plx, T, window, sinks):
    _check(plx, _inputs(1, 4, 2, T, T, 128, seed=T + window), window, sinks, (T, window, sinks))


@pytest.mark.parametrize("window,sinks", WS)
@pytest.mark.parametrize("T,Hq,Hkv", [(65, 4, 4), (300, 6, 2), (515, 4, 2), (900, 8, 8)])
def test_square_d64(plx, T, Hq, Hkv, window, sinks):
    _check(plx, _inputs(2, Hq, Hkv, T, T, 64, seed=T + window), window, sinks, (T, window, sinks))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,Tkv", [(1, 500), (5, 900), (128, 1000), (200, 777), (384, 2048)])
@pytest.mark.parametrize("window,sinks", [(64, 4), (300, 130), (129, 64), (2000, 10)])
def test_chunk_behind_a_cache(plx, T, Tkv, window, sinks, d):
    _check(plx, _inputs(1, 4, 2, T, Tkv, d, seed=T + Tkv), window, sinks, (T, Tkv, window, sinks))


@pytest.mark.parametrize("B,Hq,Hkv,T,d,window,sinks", [
    (1, 16, 8, 2300, 128, 200, 20), (2, 16, 4, 1111, 128, 512, 4), (1, 32, 16, 3000, 64, 300, 70), (3, 8, 8, 1500, 64, 1000, 130)])
def test_larger(plx, B, Hq, Hkv, T, d, window, sinks):
    """Many workgroups: whole and halved chains, sinks' key blocks in several parts; one sequence and head of them checked, and
    the gradients of its key head."""
    y = _inputs(B, Hq, Hkv, T, T, d, seed=T)
    G, b, hk = Hq // Hkv, B - 1, Hkv // 2
    heads = slice(hk * G, hk * G + G)
    tensors = [y[n] for n in "qrkv"]
    o, vb, stats = plx.parallax_prefill(*tensors, y["scale"], window=window, sinks=sinks, save_for_backward=True)
    grads = plx.parallax_prefill_backward(*tensors, o, vb, stats, y["g"], y["scale"], window=window, sinks=sinks)
    part = [host(x[b:b + 1, heads]) for x in (y["q"], y["r"])] + [host(x[b:b + 1, hk:hk + 1]) for x in (y["k"], y["v"])]
    see = _see(T, T, window, sinks)
    want = masked.masked_forward(*part, y["scale"], see)
    assert rel_l2(host(o[b:b + 1, heads]), want) <= BF16_REL_L2
    ref = masked.masked_backward(*part, host(y["g"][b:b + 1, heads]), y["scale"], see)
    for name, a, c in zip(("dq", "dr"), grads[:2], ref[:2]):
        assert_gradient_close(name, host(a[b:b + 1, heads]), c, BF16_REL_L2)
    for name, a, c in zip(("dk", "dv"), grads[2:], ref[2:]):
        assert_gradient_close(name, host(a[b:b + 1, hk:hk + 1]), c, BF16_REL_L2)
        # the sinks' own rows, which are sums over all rows and over parts of them
        assert_gradient_close(name + " of the sinks", host(a[b:b + 1, hk:hk + 1, :sinks]), c[:, :, :sinks], 1.5 * BF16_REL_L2)


@pytest.mark.parametrize("d", [36, 64, 128, 200])
@pytest.mark.parametrize("T,Tkv,window,sinks", [(1, 1, 1, 1), (17, 17, 3, 2), (100, 100, 20, 4), (300, 300, 64, 33),
                                                (130, 400, 37, 70), (260, 260, 16, 200), (600, 600, 100, 4), (50, 50, 60, 2)])
def test_f32(plx, T, Tkv, window, sinks, d):
    _check(plx, _inputs(1, 4, 2, T, Tkv, d, seed=T + d, dtype=torch.float32), window, sinks, (T, Tkv, window, sinks, d))


def test_gradients_against_differences(plx):
    """fp32 gradients against central differences of the forward in 64 bits along random directions."""
    T, window, sinks = 90, 12, 5
    y = _inputs(1, 2, 1, T, T, 64, seed=5, dtype=torch.float32)
    tensors = [y[n] for n in "qrkv"]
    o, vb, stats = plx.parallax_prefill(*tensors, y["scale"], window=window, sinks=sinks, save_for_backward=True)
    grads = plx.parallax_prefill_backward(*tensors, o, vb, stats, y["g"], y["scale"], window=window, sinks=sinks)
    ins, g, see = [host(x).astype(np.float64) for x in tensors], host(y["g"]).astype(np.float64), _see(T, T, window, sinks)
    rng = np.random.default_rng(1)
    for i, grad in enumerate(grads):
        step = rng.standard_normal(ins[i].shape)
        eps = 1e-5
        up, down = ([x + (sign * eps * step if j == i else 0) for j, x in enumerate(ins)] for sign in (1, -1))
        want = ((masked.masked_forward(*up, y["scale"], see) - masked.masked_forward(*down, y["scale"], see)) * g).sum() / (2 * eps)
        got = (host(grad).astype(np.float64) * step).sum()
        size = np.linalg.norm(host(grad)) * np.linalg.norm(step) / np.sqrt(step.size)
        assert abs(got - want) <= 1e-4 * max(abs(want), size), i


def test_twin_strides_and_no_sinks(plx):
    """The softmax-only twin; views with gaps; sinks that change nothing give the launch without them, bit for bit."""
    T, window, sinks = 500, 100, 20
    for d in (64, 128):
        y = _inputs(2, 4, 2, T, T, d, seed=9)
        twin = plx.parallax_prefill(y["q"], None, y["k"], y["v"], y["scale"], use_r=False, window=window, sinks=sinks)
        want = masked.masked_forward(host(y["q"]), 0 * host(y["r"]), host(y["k"]), host(y["v"]), y["scale"],
                                     _see(T, T, window, sinks))
        assert rel_l2(host(twin), want) <= BF16_REL_L2
        views = {n: _normal((2, T, y[n].shape[1], d + 16), 20 + i)[..., 8:d + 8].transpose(1, 2) for i, n in enumerate("qrkv")}
        _check(plx, dict(y, **views), window, sinks, ("views", d))
        for opts, plain in ((dict(window=window, sinks=T - window), dict()), (dict(window=T, sinks=3), dict()),
                            (dict(window=T + 7, sinks=T), dict())):
            a = plx.parallax_prefill(*(y[n] for n in "qrkv"), y["scale"], save_for_backward=True, **opts)
            b = plx.parallax_prefill(*(y[n] for n in "qrkv"), y["scale"], save_for_backward=True, **plain)
            assert rel_l2(host(a[0]), host(b[0]).astype(np.float64)) <= BF16_REL_L2
            assert torch.equal(plx.parallax_prefill_backward(*(y[n] for n in "qrkv"), *b, y["g"], y["scale"], **opts)[2],
                               plx.parallax_prefill_backward(*(y[n] for n in "qrkv"), *b, y["g"], y["scale"], **plain)[2])


@pytest.mark.parametrize("d", [64, 128])
def test_peaked_scores(plx, d):
    """Scores far above and below those of the sinks: the fixed reference does not hold, the online update takes over."""
    T, window, sinks = 300, 70, 5
    y = _inputs(1, 4, 2, T, T, d, seed=33)
    for factor in (30.0, -30.0):
        z = dict(y, q=(y["q"].float() * abs(factor)).to(torch.bfloat16), k=y["k"].clone())
        z["k"][:, :, :sinks] = (z["k"][:, :, :sinks].float() * (factor / 15)).to(torch.bfloat16)
        see = _see(T, T, window, sinks)
        ins = [host(z[n]) for n in "qrkv"]
        want = masked.masked_forward(*ins, z["scale"], see)
        got = host(plx.parallax_prefill(*(z[n] for n in "qrkv"), z["scale"], window=window, sinks=sinks)).astype(np.float64)
        assert np.isfinite(got).all()
        # (one key has nearly all the weight: 1 + ubar - u is a difference of numbers of size |u|, see the bound)
        assert (np.abs(got - want) <= 2 * rows.bf16_bound(*ins, z["scale"], see)).all()


def test_graph_and_bits(plx):
    """A training step captured, replayed with new inputs between eager work; the same bits every time, on another stream too."""
    T, window, sinks = 700, 150, 70
    y = _inputs(2, 8, 4, T, T, 64, seed=44)

    def step():
        o, vb, st = plx.parallax_prefill(*(y[n] for n in "qrkv"), y["scale"], window=window, sinks=sinks, save_for_backward=True)
        return (o, *plx.parallax_prefill_backward(*(y[n] for n in "qrkv"), o, vb, st, y["g"], y["scale"], window=window, sinks=sinks))

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for seed in range(3):
        for i, n in enumerate("qrkvg"):
            y[n].copy_(_normal(y[n].shape, 100 * seed + i))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), seed
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    for a, b in zip(outs, other):
        assert torch.equal(a, b)
