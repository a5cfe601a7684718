"""Host-side checks of the single layers (nsc_group_norm, nsc_adapter_project
and their gradients): descriptions, sizes and refusals, without GPU calls."""
import ctypes
import math

import pytest

import paper_1703_02529_amd as nsc

P = 4096  # a non-null, aligned address that no refused call reads


def _norm(**kw):
    base = dict(h=25, w=25, c=64, groups=8, act=nsc.NSC_ACT_RELU, dtype=nsc.NSC_T_BF16)
    base.update(kw)
    return nsc.make_norm_desc(**base)


@pytest.mark.parametrize("kw", [dict(), dict(h=1, w=1, c=1, groups=1), dict(groups=64),
                                dict(c=45, groups=5), dict(x_stride=25 * 25 * 64 + 3),
                                dict(c=1024, groups=1), dict(c=65536, groups=64),
                                dict(h=4096, w=4096, c=8, groups=1)])
def test_norm_descriptions_that_hold(kw):
    assert nsc.nsc_norm_check(_norm(**kw)) == 0, nsc.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(h=0), nsc.NSC_E_SHAPE), (dict(w=-1), nsc.NSC_E_SHAPE), (dict(c=0), nsc.NSC_E_SHAPE),
    (dict(h=4097, w=4096), nsc.NSC_E_SHAPE), (dict(c=65537, groups=65537), nsc.NSC_E_SHAPE),
    (dict(groups=0), nsc.NSC_E_SHAPE), (dict(groups=7), nsc.NSC_E_SHAPE),
    (dict(groups=128), nsc.NSC_E_SHAPE), (dict(c=2048, groups=1), nsc.NSC_E_SHAPE),
    (dict(act=3), nsc.NSC_E_INVAL), (dict(act=-1), nsc.NSC_E_INVAL),
    (dict(dtype=3), nsc.NSC_E_DTYPE), (dict(dtype=-1), nsc.NSC_E_DTYPE),
    (dict(eps=0.0), nsc.NSC_E_INVAL), (dict(eps=-1.0), nsc.NSC_E_INVAL),
    (dict(eps=math.nan), nsc.NSC_E_INVAL), (dict(eps=math.inf), nsc.NSC_E_INVAL),
    (dict(x_stride=25 * 25 * 64 - 1), nsc.NSC_E_INVAL),
    (dict(y_stride=0), nsc.NSC_E_INVAL), (dict(x_stride=2 ** 41), nsc.NSC_E_INVAL),
])
def test_norm_descriptions_that_are_refused(kw, code):
    assert nsc.nsc_norm_check(_norm(**kw)) == code
    assert nsc.last_error() != ""


def _norm_fwd(d, x=P, gamma=P, beta=P, count=None, n=4, y=P, stats=None, ws=P, ws_bytes=1 << 40):
    return nsc.lib().nsc_group_norm(ctypes.byref(d), x, gamma, beta, count, n, y, stats, ws,
                                    ws_bytes, None)


def _norm_bwd(d, x=P, dy=P, gamma=P, beta=P, stats=P, n=4, dx=P, dgamma=P, dbeta=P, ws=P,
              ws_bytes=1 << 40):
    return nsc.lib().nsc_group_norm_backward(ctypes.byref(d), x, dy, gamma, beta, stats, None, n,
                                             dx, dgamma, dbeta, ws, ws_bytes, None)


def test_norm_calls_are_refused_on_the_host():
    d = _norm()
    for kw in (dict(x=None), dict(gamma=None), dict(beta=None), dict(y=None), dict(n=-1),
               dict(n=2 ** 31), dict(x=P + 1), dict(y=P + 1), dict(gamma=P + 2),
               dict(beta=P + 1), dict(stats=P + 4), dict(count=P + 2)):
        assert _norm_fwd(d, **kw) == nsc.NSC_E_INVAL, kw
    # in place only with equal strides
    assert _norm_fwd(_norm(y_stride=2 * 25 * 25 * 64)) == nsc.NSC_E_INVAL
    assert _norm_fwd(d, n=0, x=None, gamma=None, beta=None, y=None) == 0
    for kw in (dict(x=None), dict(dy=None), dict(gamma=None), dict(beta=None), dict(stats=None),
               dict(dx=None), dict(dgamma=None), dict(dbeta=None), dict(n=-1), dict(dy=P + 1),
               dict(stats=P + 4), dict(dgamma=P + 2)):
        assert _norm_bwd(d, **kw) == nsc.NSC_E_INVAL, kw
    need = nsc.nsc_group_norm_workspace_bytes(d, 4, backward=True)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=P + 128), dict(ws_bytes=need - 1)):
        assert _norm_bwd(d, **kw) == nsc.NSC_E_WORKSPACE, kw
    assert nsc.lib().nsc_group_norm(None, P, P, P, None, 1, P, None, P, 0, None) == nsc.NSC_E_INVAL


def test_norm_workspace_sizes():
    d = _norm()
    sizes = [nsc.nsc_group_norm_workspace_bytes(d, n, backward=True) for n in (0, 1, 100, 10000)]
    assert sizes == sorted(sizes)
    for bad in (-1, 2 ** 31):
        with pytest.raises(nsc.NscError):
            nsc.nsc_group_norm_workspace_bytes(d, bad)
    with pytest.raises(nsc.NscError):
        nsc.nsc_group_norm_workspace_bytes(_norm(groups=7), 1)
    assert nsc.lib().nsc_group_norm_workspace_bytes(ctypes.byref(d), 1, 0, None) == nsc.NSC_E_INVAL
    b = ctypes.c_size_t()
    assert nsc.lib().nsc_group_norm_workspace_bytes(ctypes.byref(d), 1, 2,
                                                    ctypes.byref(b)) == nsc.NSC_E_INVAL


@pytest.mark.parametrize("dtype", [nsc.NSC_T_F32, nsc.NSC_T_BF16])
@pytest.mark.parametrize("side", [(1, 1), (3, 5), (40, 40), (300, 200)])
def test_norm_workspaces_of_every_form(side, dtype):
    """A workspace is found for all channel counts, groups and strides."""
    for c, groups in ((1, 1), (17, 1), (45, 5), (64, 8), (513, 1), (700, 1), (1021, 1021),
                      (1024, 1), (2046, 2), (2040, 2040), (4096, 64), (65536, 64)):
        for pad in (0, 1, 2, 8):
            d = _norm(h=side[0], w=side[1], c=c, groups=groups, dtype=dtype,
                      x_stride=side[0] * side[1] * c + pad)
            for n in (1, 3, 300, 5000):
                for backward in (False, True):
                    got = nsc.nsc_group_norm_workspace_bytes(d, n, backward=backward)
                    assert got >= (8 * n * c if backward else 0)


def _adapter(**kw):
    base = dict(k=4608, d=128, rank=8, n_adapters=24, dtype=nsc.NSC_T_BF16)
    base.update(kw)
    return nsc.make_adapter_desc(**base)


@pytest.mark.parametrize("kw", [dict(), dict(k=1, d=1, rank=1, n_adapters=1), dict(rank=128),
                                dict(n_adapters=65535), dict(x_stride=5000, y_stride=129)])
def test_adapter_descriptions_that_hold(kw):
    assert nsc.nsc_adapter_check(_adapter(**kw)) == 0, nsc.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(k=0), nsc.NSC_E_SHAPE), (dict(d=0), nsc.NSC_E_SHAPE), (dict(k=2 ** 24 + 1), nsc.NSC_E_SHAPE),
    (dict(d=2 ** 24 + 1), nsc.NSC_E_SHAPE), (dict(rank=0), nsc.NSC_E_SHAPE),
    (dict(rank=129), nsc.NSC_E_SHAPE), (dict(n_adapters=0), nsc.NSC_E_INVAL),
    (dict(n_adapters=65536), nsc.NSC_E_INVAL), (dict(dtype=3), nsc.NSC_E_DTYPE),
    (dict(x_stride=4607), nsc.NSC_E_INVAL), (dict(y_stride=127), nsc.NSC_E_INVAL),
    (dict(x_stride=2 ** 32), nsc.NSC_E_INVAL),
])
def test_adapter_descriptions_that_are_refused(kw, code):
    assert nsc.nsc_adapter_check(_adapter(**kw)) == code
    assert nsc.last_error() != ""


def _project(d, x=P, w=P, bias=None, a=P, b=P, scale=P, ids=P, n=4, y=P, ws=P, ws_bytes=1 << 40):
    return nsc.lib().nsc_adapter_project(ctypes.byref(d), x, w, bias, a, b, scale, ids, None, n, y,
                                         ws, ws_bytes, None)


def _project_bwd(d, x=P, dy=P, w=P, a=P, b=P, scale=P, ids=P, n=4, dx=None, da=P, db=P, ws=P,
                 ws_bytes=1 << 40):
    return nsc.lib().nsc_adapter_backward(ctypes.byref(d), x, dy, w, a, b, scale, ids, None, n, dx,
                                          da, db, ws, ws_bytes, None)


def test_adapter_calls_are_refused_on_the_host():
    d = _adapter()
    for kw in (dict(x=None), dict(w=None), dict(a=None), dict(b=None), dict(scale=None),
               dict(ids=None), dict(y=None), dict(n=-1), dict(n=2 ** 31), dict(x=P + 1),
               dict(bias=P + 2), dict(scale=P + 1), dict(ids=P + 2), dict(y=P + 1)):
        assert _project(d, **kw) == nsc.NSC_E_INVAL, kw
    need = nsc.nsc_adapter_workspace_bytes(d, 4)
    for kw in (dict(ws=None), dict(ws=P + 16), dict(ws_bytes=need - 1)):
        assert _project(d, **kw) == nsc.NSC_E_WORKSPACE, kw
    assert _project(d, n=0, x=None, ws=None, ws_bytes=0) == 0
    for kw in (dict(x=None), dict(dy=None), dict(w=None), dict(a=None), dict(b=None),
               dict(scale=None), dict(ids=None), dict(da=None), dict(db=None), dict(n=-1),
               dict(dy=P + 1), dict(da=P + 2)):
        assert _project_bwd(d, **kw) == nsc.NSC_E_INVAL, kw
    need = nsc.nsc_adapter_workspace_bytes(d, 4, backward=True)
    for kw in (dict(ws=None), dict(ws=P + 16), dict(ws_bytes=need - 1)):
        assert _project_bwd(d, **kw) == nsc.NSC_E_WORKSPACE, kw
    with pytest.raises(nsc.NscError):
        nsc.nsc_adapter_workspace_bytes(d, -1)


def test_the_binding_refuses_host_tensors_and_short_buffers():
    torch = pytest.importorskip("torch")
    d = _adapter()
    x = torch.zeros(4 * 4608, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="x:"):
        nsc.nsc_adapter_project(d, x[:-1], x, None, x, x, x, x, x, x, 4)
    with pytest.raises(ValueError, match="x:"):
        nsc.nsc_adapter_project(d, x.float(), x, None, x, x, x, x, x, x, 4)
    with pytest.raises(nsc.NscError):
        nsc.nsc_adapter_project(_adapter(rank=0), x, x, None, x, x, x, x, x, x, 4)
    n = _norm()
    m = torch.zeros(25 * 25 * 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="x:"):
        nsc.nsc_group_norm(n, m, m, m, m, None, 2)
    with pytest.raises(ValueError, match="gamma:"):
        nsc.nsc_group_norm(n, m, m, m, m, None, 1)


def test_the_gradients_take_fewer_rows_than_32_bits_count():
    """Positions are looked up past the last row, in 32 bits: 2^31 - 256 rows are
    the most that nsc_adapter_backward takes."""
    d = _adapter(k=1, d=1, rank=1, n_adapters=1)
    most = 2 ** 31 - 256
    assert nsc.nsc_adapter_workspace_bytes(d, most, backward=True) > 2 * 64 * most
    assert nsc.nsc_adapter_workspace_bytes(d, 2 ** 31 - 1) > 64 * most
    for n in (most + 1, 2 ** 31 - 1):
        assert _project_bwd(d, n=n, ws_bytes=1 << 60) == nsc.NSC_E_INVAL
        with pytest.raises(nsc.NscError):
            nsc.nsc_adapter_workspace_bytes(d, n, backward=True)


COUNTS = (1, 2, 3, 5, 16, 17, 40, 64, 100, 255, 256, 300, 500, 511, 512, 900, 1100, 2047, 4096,
          8000, 8192, 8193, 20000)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw", [
    dict(h=112, w=112, c=320, groups=32), dict(h=200, w=300, c=8, groups=1),
    dict(h=60, w=60, c=320, groups=320, dtype=nsc.NSC_T_F32), dict(h=100, w=100, c=17, groups=1),
    dict(h=37, w=41, c=45, groups=5), dict(h=25, w=25, c=64, groups=8),
    dict(h=40, w=40, c=700, groups=1), dict(h=1, w=1, c=16, groups=4),
    dict(h=30, w=30, c=4096, groups=64), dict(h=9, w=9, c=16384, groups=16384)])
def test_a_norm_workspace_holds_smaller_calls(kw, backward):
    """The workspace "for up to max_count images" is enough for every smaller
    call (a call without x is refused for that, once its workspace is checked)."""
    d, call = _norm(**kw), (_norm_bwd if backward else _norm_fwd)
    sizes = [nsc.nsc_group_norm_workspace_bytes(d, n, backward=backward) for n in COUNTS]
    for i, n in enumerate(COUNTS):
        for size in sizes[i:]:
            assert call(d, x=None, n=n, ws_bytes=size) == nsc.NSC_E_INVAL, (n, size)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw", [
    dict(), dict(k=4096, d=4096, rank=16), dict(k=9216, d=128, rank=16, dtype=nsc.NSC_T_F32),
    dict(k=4608, d=32, rank=1, n_adapters=1, dtype=nsc.NSC_T_F32), dict(k=64, d=9216, rank=128),
    dict(k=2 ** 20, d=1, rank=3), dict(k=1, d=1, rank=1), dict(k=2304, d=2304, rank=64)])
def test_an_adapter_workspace_holds_smaller_calls(kw, backward):
    d, call = _adapter(**kw), (_project_bwd if backward else _project)
    sizes = [nsc.nsc_adapter_workspace_bytes(d, n, backward=backward) for n in COUNTS]
    for i, n in enumerate(COUNTS):
        for size in sizes[i:]:
            assert call(d, x=None, n=n, ws_bytes=size) == nsc.NSC_E_INVAL, (n, size)


def test_outputs_over_the_adapters_inputs_are_refused():
    """x and dy are read after dx is written, and rows of x after rows of y."""
    d, Q = _adapter(k=128, d=128), 1 << 20
    assert _project(d, x=P, y=P, w=Q, a=Q, b=Q, scale=Q, ids=Q) == nsc.NSC_E_INVAL
    assert "overlaps" in nsc.last_error()
    for other in (dict(x=P, dy=Q), dict(x=Q, dy=P)):
        assert _project_bwd(d, dx=P, w=Q, a=Q, b=Q, scale=Q, ids=Q, **other) == nsc.NSC_E_INVAL
        assert "overlaps" in nsc.last_error()


def test_cameras_with_adapters_have_one_network(monkeypatch):
    """A runner of a shared network packs it once, and refuses networks or weights
    that differ from camera to camera."""
    np = pytest.importorskip("numpy")
    import dataclasses

    from paper_1703_02529_amd import runner
    from synth import workloads as W

    class Made(Exception):
        pass

    made = []

    def shared(cfgs, cnn, *adapters):
        raise Made(len(cfgs), cnn, adapters)

    monkeypatch.setattr(runner, "Cnn", lambda desc, blob: made.append(blob) or len(made))
    monkeypatch.setattr(runner, "SharedGroup", shared)
    ads, blob = (4, "a", "b", "scale", "of"), np.arange(5, dtype=np.float32)
    wls = [W.TINY.replace(c_low=0.2 + 0.1 * c) for c in range(3)]
    for blobs in ([blob], [blob] * 3, [blob, blob.copy(), blob.copy()]):
        made.clear()
        with pytest.raises(Made) as e:
            runner.GroupRunner(wls, blobs, 10, adapters=ads)
        assert e.value.args == (3, 1, ads) and len(made) == 1 and made[0] is blob
    made.clear()
    other = wls[2].replace(cnn=dataclasses.replace(W.TINY.cnn, dense=64))
    for bad, blobs in ((wls, [blob, blob, blob + 1]), (wls, [blob, blob]), (wls, []),
                       (wls[:2] + [other], [blob])):
        with pytest.raises(ValueError, match="share one network"):
            runner.GroupRunner(bad, blobs, 10, adapters=ads)
    assert not made


class _Elsewhere:
    """What the binding asks of a tensor, on a device of the test's choice."""

    def __init__(self, dtype, numel, device):
        self.dtype, self._n, self._d, self.is_cuda = dtype, numel, device, True

    def numel(self):
        return self._n

    def get_device(self):
        return self._d

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P


def test_a_shared_group_takes_adapters_of_the_current_device(monkeypatch):
    torch = pytest.importorskip("torch")
    import types
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cnn = types.SimpleNamespace(desc=nsc.make_desc([16], [0], 16, 8, 8, False), handle=None)
    cfg = nsc.make_cfg(in_h=16, in_w=16, dd_h=8, dd_w=8, cnn_h=8, cnn_w=8)
    need = dict(a=(torch.float32, 2 * 3 * 16 * 64), b=(torch.float32, 2 * 3 * 16),
                scale=(torch.float32, 2), of_camera=(torch.int32, 1))
    for away in (None, *need):
        at = [_Elsewhere(t, n, int(k == away)) for k, (t, n) in need.items()]
        # on the current device: on to the library, which refuses the missing network
        with pytest.raises(ValueError if away else nsc.NscError,
                           match="device 1" if away else "network handle"):
            nsc.SharedGroup([cfg], cnn, 3, *at)
