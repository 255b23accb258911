"""Linear cross entropy and its gradients: the library against the formulas in 64 bits.

Tolerances, with u = 2^-24.  fp32 factors are held by two planes of fp16: to 2^-22 of themselves, values below
2^-18 of the tensor's largest to 2^-40 of that (half of fp16's smallest step, 2^-25, under a power of two that
brings the largest to 2^14 at least: 2^-39), and the product of two lower planes, below 2^-22 of the term, is left out: 12 u of a term.
A logit is a sum of D such products in fp32: partial sums of at most |h_t| |w_v| and roundings that behave like
a random walk, so it is off by e = u (12 + 2 sqrt(D)) max|h| max|w| (+ u |bias|).  lse is off by e, by 64 u relative
of the sum of exponentials, and by u |lse|; a loss by twice that.  dl is off by (2 e + 64 u) |p| and 2 u |dl|; its
products add u (12 + 2 sqrt(n)) of their magnitudes, n terms, with fp32 operands 2^-40 of the largest |dloss|
(dl's planes hold it times 2^15 relative to that) times the other factor and 2^-39 of the other tensor's largest times dl;
with bf16 operands half a step, 2^-8, of every |dl|; and a bf16 result half a step more.  Below 2^-126 fp32 and bf16
hold no full significand, and such values may count as zero: 4 x 2^-126 times the other factor.
"""
import numpy as np
import pytest

from oracle import training as tr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": 0, "bf16": 1}


def tensors(T, D, V, type, seed, bias, ignored, extra=0, offset=0):
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[type]
    rng = np.random.default_rng(seed)

    def strided(a):
        rows, cols = a.shape
        whole = torch.zeros(offset + rows * (cols + extra) + 8, dtype=dt, device="cuda")
        t = whole[offset:offset + rows * (cols + extra)].view(rows, cols + extra)[:, :cols]
        t.copy_(torch.from_numpy(a))
        return t

    w = rng.standard_normal((V, D)) / np.sqrt(D)
    target = rng.integers(0, V, T)
    h = rng.standard_normal((T, D)) + 2 * w[target]
    out = rng.random(T) < ignored
    target[out] = rng.choice([-100, -1, V, V + 5], out.sum())
    b = (0.3 * rng.standard_normal(V)).astype(np.float32) if bias else None
    dloss = (rng.random(T) + 0.5).astype(np.float32) / T
    return strided(h), strided(w), b, target, dloss


def run(T, D, V, type, seed=0, bias=True, ignored=0.2, extra=0, offset=0, piece=0, change=None, ignore_index=-100):
    import torch
    import paper_2004_11077_amd as wn
    h, w, b, target, dloss = tensors(T, D, V, type, seed, bias, ignored, extra, offset)
    if change:
        change(h, w, b, target, dloss)
    cuda = lambda a: None if a is None else torch.from_numpy(a).cuda()
    tb, tt, td = cuda(b), cuda(target), cuda(dloss)
    desc = wn.LossDesc(T, D, V, type=TYPES[type], h_stride=D + extra, w_stride=D + extra, piece=piece, ignore_index=ignore_index)
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    loss, lse, dbias = nan(T), nan(T), nan(V) if bias else None
    dh, dw = nan(T, D).to(h.dtype), nan(V, D).to(h.dtype)
    room = lambda f: torch.full((f(desc),), 255, dtype=torch.uint8, device="cuda")
    ws = room(wn.wino_linear_cross_entropy_workspace_bytes)
    wn.wino_linear_cross_entropy(desc, h, w, tb, tt, loss, lse, ws)
    ws = room(wn.wino_linear_cross_entropy_backward_workspace_bytes)
    wn.wino_linear_cross_entropy_backward(desc, h, w, tb, tt, lse, td, dh, dw, dbias, ws)
    torch.cuda.synchronize()
    back = lambda t: None if t is None else t.double().cpu().numpy()
    return dict(h=back(h), w=back(w), b=b, target=target, dloss=dloss.astype(np.float64), loss=back(loss), lse=back(lse),
                dh=back(dh), dw=back(dw), dbias=back(dbias))


def check(r, type, ignore_index=-100):
    h, w, b, target, dloss = (r[k] for k in ("h", "w", "b", "target", "dloss"))
    T, D = h.shape
    V = w.shape[0]
    bf = type == "bf16"
    b64 = None if b is None else b.astype(np.float64)
    loss, lse = tr.cross_entropy(h, w, b64, target, ignore_index)
    e = U * (12 + 2 * np.sqrt(D)) * np.linalg.norm(h, axis=1).max() * np.linalg.norm(w, axis=1).max()
    e += 0 if b is None else U * np.abs(b[np.isfinite(b)]).max(initial=0)
    with np.errstate(invalid="ignore"):
        tol = e + 64 * U + 2 * U * np.abs(lse)
        same = (r["lse"] == lse) | (np.abs(r["lse"] - lse) <= tol)
        assert same.all()
        same = (r["loss"] == loss) | (np.abs(r["loss"] - loss) <= 2 * tol + U * np.abs(loss))
        assert same.all()
    dh, dw, db, dl = tr.cross_entropy_backward(h, w, b64, target, dloss, ignore_index)
    k = tr.kept(target, V, ignore_index)
    p = np.abs(dl)
    p[np.arange(T)[k], target[k]] += dloss[k]          # exp(l - lse) and the one, before their difference
    err = (2 * e + 66 * U) * p
    rounded = err + (2.0 ** -8 * np.abs(dl) if bf else 0)

    def near(got, ref, a, m, n):
        # products of dl (with its error) and the other operand
        tol = rounded_of(a) @ m + U * (12 + 2 * np.sqrt(n)) * (np.abs(a) @ m) + 2 * U * np.abs(ref)
        if not bf:
            tol += 2.0 ** -40 * np.abs(dloss[k]).max(initial=0) * m.sum(0) + 2.0 ** -39 * m.max(initial=0) * np.abs(a).sum(1, keepdims=True)
        tol += 2.0 ** -8 * np.abs(ref) if bf else 0
        tol += 4 * 2.0 ** -126 * (1 + np.abs(m).sum(0))
        assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()

    rounded_of = lambda a: rounded if a is dl else rounded.T
    near(r["dh"], dh, dl, np.abs(w), V)
    hk = np.where(k[:, None], np.abs(h), 0)
    near(r["dw"], dw, dl.T, hk, T)
    if b is not None:
        assert (np.abs(r["dbias"] - db) <= err.sum(0) + U * (8 + 2 * np.sqrt(T)) * np.abs(dl).sum(0) + U * np.abs(db) + 2.0 ** -126 * T).all()
    assert not r["dh"][~k].any() and not r["loss"][~k].any()


SHAPES = [(1, 1, 1), (1, 16, 2), (2, 3, 5), (7, 33, 10), (16, 64, 64), (64, 128, 130), (65, 127, 129), (130, 64, 1000),
          (256, 512, 10), (100, 256, 257), (33, 520, 1031), (300, 72, 515), (1, 256, 5000), (129, 200, 2051)]


@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("T,D,V", SHAPES)
def test_shapes(T, D, V, type):
    check(run(T, D, V, type, seed=T + D + V), type)


@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("T,D,V,piece", [(40, 96, 1000, 256), (200, 64, 1025, 512), (3, 128, 4000, 1024), (129, 192, 700, 256)])
def test_pieces(T, D, V, piece, type):
    """Small pieces: dh is summed over them, every class belongs to one."""
    check(run(T, D, V, type, piece=piece), type)


@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("D,extra,offset", [(64, 8, 0), (64, 3, 0), (64, 0, 1), (65, 0, 0), (192, 64, 8)])
def test_strides_and_alignment(D, extra, offset, type):
    check(run(50, D, 300, type, extra=extra, offset=offset), type)


@pytest.mark.parametrize("D,extra,offset,V,piece", [(64, 0, 0, 66000, 0), (925, 0, 0, 4700, 0), (515, 5, 3, 8200, 0), (1030, 0, 1, 4100, 1024), (33, 0, 0, 131072, 0)])
@pytest.mark.parametrize("T", [1, 5, 64])
def test_few_rows_and_large_weights(T, D, extra, offset, V, piece):
    """fp32 operands are taken as they stand here, whatever their strides and however many features are left
    over behind whole blocks of 32."""
    check(run(T, D, V, "f32", extra=extra, offset=offset, piece=piece, ignored=0.1), "f32")


def test_few_rows_beside_rows_left_out():
    """Large weights, and NaN and infinities in a padding row."""
    def change(h, w, b, target, dloss):
        target[[1, 5]] = -100
        h[1], h[5] = float("nan"), float("inf")
        dloss[1] = np.nan
    r = run(9, 130, 33000, "f32", ignored=0, change=change)
    assert np.isfinite(r["dw"]).all() and np.isfinite(r["dbias"]).all()
    r["h"][[1, 5]] = 0
    r["lse"][[1, 5]] = tr.cross_entropy(r["h"], r["w"], r["b"].astype(np.float64), r["target"])[1][[1, 5]]
    r["dloss"][1] = 0
    check(r, "f32")


@pytest.mark.parametrize("T", [2, 16, 17, 33, 48, 65, 100, 192, 193])
@pytest.mark.parametrize("D,V", [(67, 1000), (256, 257), (512, 1040)])
def test_rows_up_to_where_weights_are_copied(T, D, V):
    """Rows that leave out some of a tile's blocks and waves, and the first number of rows that takes planes."""
    check(run(T, D, V, "f32", extra=1), "f32")


@pytest.mark.parametrize("T,D,V", [(1000, 67, 3), (300, 520, 10), (4099, 300, 64), (8300, 257, 1), (17000, 260, 32), (16400, 256, 33), (1030, 64, 65)])
def test_few_classes_and_many_rows(T, D, V):
    check(run(T, D, V, "f32", extra=3), "f32")


@pytest.mark.parametrize("T,D,V", [(4097, 256, 200), (8000, 256, 66), (2, 300, 16000), (40, 256, 8100)])
def test_products_of_few_tiles(T, D, V):
    """About as many tiles as k is shared between a work group's waves for."""
    check(run(T, D, V, "f32"), "f32")


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_split_classes(type):
    """Few tiles of dh and many classes: ranges of classes are summed apart."""
    check(run(20, 96, 9000, type, bias=False), type)


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_ignore_index_may_be_a_class(type):
    def change(h, w, b, target, dloss):
        target[::3] = 4
    r = run(40, 64, 50, type, change=change, ignore_index=4)
    check(r, type, ignore_index=4)


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_nothing_from_rows_left_out(type):
    """Whatever stands in a padding row: NaN and infinities among it."""
    import torch

    def change(h, w, b, target, dloss):
        target[[1, 5, 6]] = -100
        h[1], h[5], h[6, 3] = float("nan"), float("inf"), float("-inf")
        dloss[[1, 5]] = np.nan, np.inf
    r = run(70, 128, 90, type, ignored=0, change=change)
    assert np.isfinite(r["dw"]).all() and np.isfinite(r["dbias"]).all()
    assert not r["dh"][[1, 5, 6]].any() and not r["loss"][[1, 5, 6]].any()
    for name in ("h",):
        r[name][[1, 5, 6]] = 0
    r["lse"][[1, 5, 6]] = tr.cross_entropy(r["h"], r["w"], r["b"].astype(np.float64), r["target"])[1][[1, 5, 6]]
    r["dloss"][[1, 5]] = 0
    check(r, type)


@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("all_of_them", [False, True])
def test_masked_classes(all_of_them, type):
    def change(h, w, b, target, dloss):
        b[::2] = -np.inf
        if all_of_them:
            b[:] = -np.inf
    r = run(30, 64, 200, type, ignored=0, change=change)
    check(r, type)
    assert np.isposinf(r["loss"]).any()


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_lowest_value_as_a_mask(type):
    """A bias of the type's lowest value masks like -infinity where other classes are left."""
    def change(h, w, b, target, dloss):
        b[10:] = np.finfo(np.float32).min
        target[:] = target % 10
    r = run(30, 64, 200, type, ignored=0, change=change)
    assert np.isfinite(r["loss"]).all() and not r["dbias"][10:].any() and not r["dw"][10:].any()


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_large_logits(type):
    """Logits of some hundreds: exponentials over- and underflow unless the maximum is taken off."""
    def change(h, w, b, target, dloss):
        h.mul_(100)
    check(run(40, 64, 300, type, change=change), type)


def test_one_weight_for_all_rows_rounds_nothing_alike():
    """bf16, dloss = 1 / 3891 in every row, every row a sure hit of a wrong class: the gradient of a
    target's class is -dloss h, free of a rounding of 1 / 3891 to bf16 (2^-8 of it at most)."""
    import torch
    import paper_2004_11077_amd as wn
    T, D, V = 64, 64, 64
    h = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
    h[torch.arange(T), torch.arange(T)] = 1
    w = 60 * torch.eye(V, D, device="cuda", dtype=torch.bfloat16).roll(1, 0)
    target = torch.arange(T, device="cuda")
    dloss = torch.full((T,), 1 / 3891, device="cuda")
    desc = wn.LossDesc(T, D, V, type=wn.TYPE_BF16)
    ws = torch.empty(wn.wino_linear_cross_entropy_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(2, T, device="cuda")
    wn.wino_linear_cross_entropy(desc, h, w, None, target, loss, lse, ws)
    dw = torch.empty_like(w)
    wn.wino_linear_cross_entropy_backward(desc, h, w, None, target, lse, dloss, None, dw, None, ws)
    assert torch.equal(torch.diagonal(dw), (-dloss).to(torch.bfloat16))


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_outputs_one_at_a_time_and_again(type):
    import torch
    import paper_2004_11077_amd as wn
    h, w, b, target, dloss = tensors(90, 128, 700, type, 3, True, 0.1)
    t = lambda a: torch.from_numpy(a).cuda()
    b, target, dloss = t(b), t(target), t(dloss)
    desc = wn.LossDesc(90, 128, 700, type=TYPES[type])
    ws = torch.empty(wn.wino_linear_cross_entropy_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(2, 90, device="cuda")
    wn.wino_linear_cross_entropy(desc, h, w, b, target, loss, lse, ws)
    new = lambda: (torch.zeros(90, 128, device="cuda", dtype=h.dtype), torch.zeros(700, 128, device="cuda", dtype=h.dtype), torch.zeros(700, device="cuda"))
    all3, alone = new(), new()
    wn.wino_linear_cross_entropy_backward(desc, h, w, b, target, lse, dloss, *all3, ws)
    for i in range(3):
        out = [alone[k] if k == i else None for k in range(3)]
        wn.wino_linear_cross_entropy_backward(desc, h, w, b, target, lse, dloss, *out, ws)
    assert all(torch.equal(x, y) for x, y in zip(all3, alone))


def test_no_rows_and_no_weight():
    import torch
    import paper_2004_11077_amd as wn
    for type, dt in ((0, torch.float32), (1, torch.bfloat16)):
        desc = wn.LossDesc(0, 5, 7, type=type)
        wn.wino_linear_cross_entropy(desc, None, None, None, None, None, None, None)
        dw, dbias = torch.ones(7, 5, dtype=dt, device="cuda"), torch.ones(7, device="cuda")
        wn.wino_linear_cross_entropy_backward(desc, None, None, None, None, None, None, None, dw, dbias, None)
        assert not dw.any() and not dbias.any()

    def change(h, w, b, target, dloss):
        dloss[:] = 0
    r = run(9, 40, 30, "f32", change=change)
    assert not r["dh"].any() and not r["dw"].any() and not r["dbias"].any()
