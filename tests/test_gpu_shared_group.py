"""A camera group of one shared fp32 network with low-rank adapters of its dense
layer, against the oracle's cascade of each camera with the adapter's product
added to its dense weights."""
import ctypes
import dataclasses

import numpy as np
import pytest
import torch

import oracle
import paper_1703_02529_amd as nsc
import synth
from paper_1703_02529_amd.runner import GroupRunner
from synth import workloads as W

from helpers import compare_cascade

DEV = "cuda"
SIDE, CH = 12, 32          # the last map of the 100x100 workload's network
FLAT, DENSE = SIDE * SIDE * CH, 32


def _blob():
    wl = W.TINY
    return synth.weight_blob(wl.cnn, synth.cnn_weights(wl.cnn, wl.weight_seed)).astype(np.float32)


def _adapters(n, rank, seed=3):
    rng = np.random.default_rng(seed)
    a = rng.normal(0, FLAT ** -0.5, (n, rank, FLAT)).astype(np.float32)   # (y, x, c) features
    b = rng.normal(0, 2 * rank ** -0.5, (n, DENSE, rank)).astype(np.float32)
    return a, b, (0.5 + rng.random(n)).astype(np.float32)


def _merged(blob, a, b, scale):
    """The blob with scale * b a added to its dense weights, which it holds in
    (c, y, x) order."""
    out = blob.copy()
    at = len(blob) - (DENSE * FLAT + 2 * DENSE + 1)
    add = (float(scale) * b.astype(np.float64) @ a.astype(np.float64)).reshape(DENSE, SIDE, SIDE,
                                                                             CH)
    w = out[at:at + DENSE * FLAT].reshape(DENSE, FLAT)
    w[:] = (w + add.transpose(0, 3, 1, 2).reshape(DENSE, FLAT)).astype(np.float32)
    return out


def _cameras(k):
    return [W.TINY.replace(video=dataclasses.replace(W.TINY.video, seed=31 + c), delta=1 + c % 3,
                           delta_diff=(20.0, 12.0, 30.0)[c % 3], c_low=0.2 + 0.05 * c)
            for c in range(k)]


def _run(cams, of_camera, ads, sizes):
    a, b, scale = (torch.from_numpy(v).to(DEV) for v in ads)
    of = torch.tensor(of_camera, dtype=torch.int32, device=DEV)
    run = GroupRunner(cams, [_blob()] * len(cams), max(sizes),
                      adapters=(a.shape[1], a, b, scale, of))
    videos = [synth.Video(c.video) for c in cams]
    keys = ("score", "fire", "logit", "label", "defer")
    outs, t = [{k: [] for k in keys} for _ in cams], 0
    for n in sizes:
        batch = np.concatenate([v.frames(t, t + n) for v in videos])
        run.run(torch.from_numpy(batch.reshape(-1)).to(DEV), n, t0=t)
        for k in keys:
            got = getattr(run, k)[:len(cams) * n].cpu().numpy().reshape(len(cams), n)
            for c in range(len(cams)):
                outs[c][k].append(got[c].copy())
        t += n
    run.close()
    return [{k: np.concatenate(o[k]) for k in keys} for o in outs], videos


@pytest.mark.gpu
@pytest.mark.parametrize("rank", [1, 8, 20])
def test_each_camera_is_its_own_cascade(rank):
    cams, of_camera, sizes = _cameras(5), [0, 2, -1, 1, 0], [300, 1, 299]
    ads = _adapters(3, rank)
    gpu, videos = _run(cams, of_camera, ads, sizes)
    fired = 0
    for c, (wl, p) in enumerate(zip(cams, of_camera)):
        blob = _blob() if p < 0 else _merged(_blob(), ads[0][p], ads[1][p], ads[2][p])
        cfg, keep = oracle.make_cfg(wl)
        ref, _ = oracle.cascade(cfg, wl.cnn, blob, videos[c].frames(0, sum(sizes)), t0=0)
        fired += compare_cascade(wl, gpu[c], ref, t0=0)["fired"]
    assert fired > 50


@pytest.mark.gpu
def test_cameras_without_adapters_share_the_network():
    """Adapters change their own cameras' logits and nobody else's."""
    cams, sizes = _cameras(4), [50]
    ads = _adapters(2, 4)
    plain, _ = _run(cams, [-1, -1, 99, -7], ads, sizes)
    some, _ = _run(cams, [-1, 1, -1, 0], ads, sizes)
    for c in (0, 2):
        assert np.array_equal(plain[c]["logit"], some[c]["logit"], equal_nan=True)
    for c in (1, 3):
        assert not np.array_equal(plain[c]["logit"], some[c]["logit"], equal_nan=True)


def test_refusals_on_the_host():
    cfg = nsc.make_cfg(in_h=100, in_w=100, dd_h=50, dd_w=50, cnn_h=50, cnn_w=50)
    cfgs = (nsc.CascadeCfg * 1)(cfg)
    h = ctypes.c_void_p()
    ad = nsc.GroupAdapters(4, 2, 4096, 4096, 4096, 4096)
    make = lambda cnn, a, n=1: nsc.lib().nsc_group_create_shared(
        cfgs, cnn, ctypes.byref(a) if a is not None else None, n, ctypes.byref(h))
    assert make(None, ad) == nsc.NSC_E_INVAL and "handle" in nsc.last_error()
    assert make(None, None) == nsc.NSC_E_INVAL
    assert make(None, ad, 0) == nsc.NSC_E_INVAL
    for field in ("a", "b", "scale", "of_camera"):
        for bad in (None, 4098):
            broken = nsc.GroupAdapters(4, 2, 4096, 4096, 4096, 4096)
            setattr(broken, field, bad)
            assert make(None, broken) == nsc.NSC_E_INVAL, field
            assert "adapter buffer" in nsc.last_error()


@pytest.mark.gpu
def test_refusals_with_a_network():
    wl = W.TINY
    of = torch.zeros(1, dtype=torch.int32, device=DEV)
    a, b, scale = (torch.from_numpy(v).to(DEV) for v in _adapters(2, 4))
    cfg = nsc.make_cfg(in_h=100, in_w=100, dd_h=50, dd_w=50, cnn_h=50, cnn_w=50)
    narrow = nsc.Cnn(nsc.make_desc(wl.cnn.conv, wl.cnn.pool, 32, 50, 50, True), _blob())
    with pytest.raises(nsc.NscError, match="NSC_E_DTYPE"):
        nsc.SharedGroup([cfg], narrow, 4, a, b, scale, of)
    cnn = nsc.Cnn(nsc.make_desc(wl.cnn.conv, wl.cnn.pool, 32, 50, 50, False), _blob())
    with pytest.raises(ValueError, match="a:"):
        nsc.SharedGroup([cfg], cnn, 5, a, b, scale, of)
    with pytest.raises(ValueError, match="of_camera:"):
        nsc.SharedGroup([cfg, cfg], cnn, 4, a, b, scale, of)
    narrow.close()
    cnn.close()
