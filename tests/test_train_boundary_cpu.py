"""Refusals of the training operators' entry points.  No kernel is launched: every call is refused on
the host, or has nothing to do.  Pointers are addresses that nothing reads."""
import ctypes as C
import os

import pytest

wn = pytest.importorskip("paper_2004_11077_amd")
from paper_2004_11077_amd import binding  # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists(wn.lib_path()),
                                reason="libwino.so not built (python -m paper_2004_11077_amd.build)")

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -4
A = 4096          # an aligned address
NAN, INF = float("nan"), float("inf")


def ref(d):
    return None if d is None else C.byref(d)


def norm(d, x=A, gamma=A, beta=A, y=A, mean=A, rstd=A):
    return binding._load().wino_layer_norm(ref(d), x, gamma, beta, y, mean, rstd, None)


def norm_backward(d, dy=A, x=A, gamma=A, mean=A, rstd=A, dx=A, dgamma=A, dbeta=A, ws=A, room=1 << 40):
    return binding._load().wino_layer_norm_backward(ref(d), dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, room, None)


def loss(d, h=A, w=A, bias=A, targets=A, loss=A, lse=A, ws=A, room=1 << 60):
    return binding._load().wino_linear_cross_entropy(ref(d), h, w, bias, targets, loss, lse, ws, room, None)


def loss_backward(d, h=A, w=A, bias=A, targets=A, lse=A, dloss=A, dh=A, dw=A, dbias=A, ws=A, room=1 << 60):
    return binding._load().wino_linear_cross_entropy_backward(ref(d), h, w, bias, targets, lse, dloss, dh, dw, dbias, ws, room, None)


def update(d, g=A, o=A, ws=A, room=1 << 60):
    return binding._load().wino_orthogonalise(ref(d), g, o, ws, room, None)


NORM = [(None, EINVAL), (wn.NormDesc(-1, 4), EINVAL), (wn.NormDesc(2, 0), EINVAL), (wn.NormDesc(2, (1 << 24) + 1), EINVAL),
        (wn.NormDesc(2, 4, x_type=wn.TYPE_I8), EUNSUPPORTED), (wn.NormDesc(2, 4, y_type=3), EUNSUPPORTED),
        (wn.NormDesc(2, 4, g_type=wn.TYPE_I8), EUNSUPPORTED), (wn.NormDesc(2, 4, eps=-1), EINVAL),
        (wn.NormDesc(2, 4, eps=NAN), EINVAL), (wn.NormDesc(2, 4, y_type=wn.TYPE_I8, s_y=0), EINVAL),
        (wn.NormDesc(2, 4, y_type=wn.TYPE_I8, s_y=INF), EINVAL), (wn.NormDesc(2, 4, x_stride=3), EINVAL),
        (wn.NormDesc(2, 4, y_stride=-4), EINVAL), (wn.NormDesc(2, 4, dy_stride=1), EINVAL), (wn.NormDesc(2, 4, dx_stride=1), EINVAL)]


@pytest.mark.parametrize("i", range(len(NORM)))
def test_norm_descriptors(i):
    d, code = NORM[i]
    size = C.c_size_t()
    assert norm(d) == norm_backward(d) == code
    assert binding._load().wino_layer_norm_backward_workspace_bytes(ref(d), C.byref(size)) == code


def test_norm_workspace_stays_small():
    """512 rows of partial sums up to 16384 channels, and no more bytes for longer rows until one row of
    them is that long."""
    for channels in (16, 16384, 16385, 100001, 1 << 20, 1 << 23, 1 << 24):
        size = wn.wino_layer_norm_backward_workspace_bytes(wn.NormDesc(1 << 20, channels))
        assert 8 * channels <= size <= max(8 * channels, 1 << 26)


def test_norm_pointers():
    d = wn.NormDesc(3, 8, x_type=wn.TYPE_BF16, y_type=wn.TYPE_F32, g_type=wn.TYPE_F32)
    for kw in (dict(x=None), dict(y=None), dict(x=A + 1), dict(y=A + 2), dict(gamma=A + 2), dict(beta=A + 1), dict(mean=A + 2), dict(rstd=A + 3)):
        assert norm(d, **kw) == EINVAL, kw
    for kw in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dy=A + 2), dict(dx=A + 1), dict(x=A + 1),
               dict(gamma=A + 2), dict(dgamma=A + 2), dict(dbeta=A + 1), dict(ws=None)):
        assert norm_backward(d, **kw) == EINVAL, kw
    need = wn.wino_layer_norm_backward_workspace_bytes(d)
    assert norm_backward(d, room=need - 1) == EWORKSPACE and norm_backward(d, ws=A + 128) == EWORKSPACE
    assert norm_backward(d, dx=None, dgamma=None, dbeta=None) == 0
    assert norm(wn.NormDesc(0, 8), x=None, y=None) == 0
    assert norm_backward(wn.NormDesc(0, 8), dgamma=None, dbeta=None) == 0
    assert binding._load().wino_layer_norm_backward_workspace_bytes(C.byref(d), None) == EINVAL


BIG = 1 << 21
LOSS = [(None, EINVAL), (wn.LossDesc(-1, 4, 4), EINVAL), (wn.LossDesc(BIG + 1, 4, 4), EINVAL), (wn.LossDesc(1, 0, 4), EINVAL),
        (wn.LossDesc(1, (1 << 20) + 1, 4), EINVAL), (wn.LossDesc(1, 4, 0), EINVAL), (wn.LossDesc(1, 4, (1 << 27) + 1), EINVAL),
        (wn.LossDesc(1, 4, 4, type=wn.TYPE_I8), EUNSUPPORTED), (wn.LossDesc(1, 4, 4, h_stride=3), EINVAL),
        (wn.LossDesc(1, 4, 4, w_stride=-1), EINVAL), (wn.LossDesc(1, 4, 4, piece=-1), EINVAL), (wn.LossDesc(1, 4, 4, piece=BIG + 1), EINVAL)]


@pytest.mark.parametrize("i", range(len(LOSS)))
def test_loss_descriptors(i):
    d, code = LOSS[i]
    size = C.c_size_t()
    assert loss(d) == loss_backward(d) == code
    assert binding._load().wino_linear_cross_entropy_workspace_bytes(ref(d), C.byref(size)) == code
    assert binding._load().wino_linear_cross_entropy_backward_workspace_bytes(ref(d), C.byref(size)) == code


@pytest.mark.parametrize("type,off", [(wn.TYPE_F32, 2), (wn.TYPE_BF16, 1)])
def test_loss_pointers(type, off):
    d = wn.LossDesc(3, 8, 5, type=type)
    for kw in (dict(h=None), dict(w=None), dict(targets=None), dict(loss=None), dict(lse=None), dict(ws=None), dict(h=A + off),
               dict(w=A + off), dict(bias=A + 2), dict(targets=A + 4), dict(loss=A + 2), dict(lse=A + 1)):
        assert loss(d, **kw) == EINVAL, kw
    for kw in (dict(h=None), dict(w=None), dict(targets=None), dict(lse=None), dict(dloss=None), dict(ws=None), dict(h=A + off),
               dict(dh=A + off), dict(dw=A + off), dict(dbias=A + 2), dict(dloss=A + 1), dict(targets=A + 2)):
        assert loss_backward(d, **kw) == EINVAL, kw
    need = wn.wino_linear_cross_entropy_workspace_bytes(d)
    assert loss(d, room=need - 1) == EWORKSPACE and loss(d, ws=A + 16) == EWORKSPACE
    need = wn.wino_linear_cross_entropy_backward_workspace_bytes(d)
    assert loss_backward(d, room=need - 1) == EWORKSPACE and loss_backward(d, ws=A + 16) == EWORKSPACE
    assert loss_backward(d, dh=None, dw=None, dbias=None) == 0
    assert loss(wn.LossDesc(0, 8, 5), h=None, w=None) == 0
    assert binding._load().wino_linear_cross_entropy_workspace_bytes(C.byref(d), None) == EINVAL


def test_loss_piece_bounds_the_workspace():
    sizes = [wn.wino_linear_cross_entropy_backward_workspace_bytes(wn.LossDesc(4096, 1024, 1 << 17, type=wn.TYPE_BF16, piece=p))
             for p in (1024, 8192, 65536)]
    assert sizes[0] < sizes[1] < sizes[2]
    # nowhere near the logits, 4096 x 2^17 of fp32
    assert wn.wino_linear_cross_entropy_backward_workspace_bytes(wn.LossDesc(4096, 1024, 1 << 17, type=wn.TYPE_BF16)) < 1 << 30


UPDATE = [(None, EINVAL), (wn.OrthogonaliseDesc(-1, 4, 4), EINVAL), (wn.OrthogonaliseDesc(65536, 4, 4), EINVAL),
          (wn.OrthogonaliseDesc(1, -4, 4), EINVAL), (wn.OrthogonaliseDesc(1, 4, (1 << 20) + 1), EINVAL),
          (wn.OrthogonaliseDesc(1, 4, 4, g_type=wn.TYPE_I8), EUNSUPPORTED), (wn.OrthogonaliseDesc(1, 4, 4, o_type=7), EUNSUPPORTED),
          (wn.OrthogonaliseDesc(1, 4, 4, steps=0), EINVAL), (wn.OrthogonaliseDesc(1, 4, 4, steps=101), EINVAL),
          (wn.OrthogonaliseDesc(1, 4, 4, a=NAN), EINVAL), (wn.OrthogonaliseDesc(1, 4, 4, c=INF), EINVAL),
          (wn.OrthogonaliseDesc(1, 4, 4, scale=NAN), EINVAL), (wn.OrthogonaliseDesc(1, 4, 4, eps=0), EINVAL),
          (wn.OrthogonaliseDesc(1, 4, 4, g_stride=3), EINVAL), (wn.OrthogonaliseDesc(1, 4, 4, o_stride=3), EINVAL),
          (wn.OrthogonaliseDesc(2, 4, 4, g_batch=15), EINVAL), (wn.OrthogonaliseDesc(2, 4, 4, o_stride=6, o_batch=21), EINVAL),
          (wn.OrthogonaliseDesc(30000, 1, 1 << 20), EINVAL), (wn.OrthogonaliseDesc(1, 1 << 20, 1 << 20), EINVAL),
          (wn.OrthogonaliseDesc(513, 1, 1 << 20), EINVAL)]


@pytest.mark.parametrize("i", range(len(UPDATE)))
def test_update_descriptors(i):
    d, code = UPDATE[i]
    size = C.c_size_t()
    assert update(d) == code
    assert binding._load().wino_orthogonalise_workspace_bytes(ref(d), C.byref(size)) == code


def test_update_pointers():
    d = wn.OrthogonaliseDesc(2, 5, 9, g_type=wn.TYPE_BF16)
    for kw in (dict(g=None), dict(o=None), dict(ws=None), dict(g=A + 1), dict(o=A + 2)):
        assert update(d, **kw) == EINVAL, kw
    need = wn.wino_orthogonalise_workspace_bytes(d)
    assert update(d, room=need - 1) == EWORKSPACE and update(d, ws=A + 8) == EWORKSPACE
    assert update(wn.OrthogonaliseDesc(0, 5, 9), g=None, o=None) == 0
    assert binding._load().wino_orthogonalise_workspace_bytes(C.byref(d), None) == EINVAL


def test_errors_name_the_argument():
    with pytest.raises(wn.WinoError, match="steps"):
        wn.wino_orthogonalise_workspace_bytes(wn.OrthogonaliseDesc(1, 4, 4, steps=0))
    with pytest.raises(wn.WinoError, match="classes"):
        wn.wino_linear_cross_entropy_workspace_bytes(wn.LossDesc(1, 4, 0))


def test_strides_reach_within_the_tensor():
    torch = pytest.importorskip("torch")
    whole = torch.zeros(100)
    binding._reach(("x", whole[10:], 9, 10, 9), ("y", None, 100, 10, 9), ("z", whole, 0, 1000, 1000),
                   ("none", whole, 50, 0, 50), ("view", whole.view(10, 10)[:, :3], 10, 10, 3),
                   ("g", whole, 10, 2, 7, 41, 3), ("dense rows", whole, 0, 5, 4, 40, 3), ("one", whole, 0, 4, 5, 0, 3))
    for bad in (("x", whole[11:], 9, 10, 9), ("view", whole.view(10, 10)[:, 3:], 10, 10, 8),
                ("g", whole, 10, 2, 7, 42, 3), ("rows", whole, 0, 5, 4, 41, 3), ("stride", whole, 10, 4, 7, 0, 3)):
        with pytest.raises(wn.WinoError) as e:
            binding._reach(bad)
        assert e.value.code == EINVAL and bad[0] in str(e.value)
