"""Orthogonalised updates: the library against the formula in 64 bits.

Tolerance.  With f(s) = a s + b s^3 + c s^5 on the singular values, |f'| <= 4 on [0, 1.2], the range
that the usual coefficients keep them in, so an error of the matrix before a step leaves it at most four
times as large in the Frobenius norm.  A step adds three products, q = 3 x 2^-22 each (both factors held
to 2^-22 of themselves by two planes of fp16, and the product of their lower planes left out) and fp32 sums that behave like random
walks of their length n, u (8 + 2 sqrt(n)), each relative to |X| times the size of the polynomial's terms, at most a + |b| +
|c| = 10.3 for singular values up to one.  So the result's error is at most the sum over the steps of
4^(steps - k) 10.3 (3 q + u (8 + 2 sqrt(n))) max(|X_k|, |X_(k+1)|), and half a step of a bf16 result.
"""
import numpy as np
import pytest

from oracle import training as tr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": 0, "bf16": 1}


def gradients(batch, rows, cols, seed, scale=1e-3, kind="noisy"):
    rng = np.random.default_rng(seed)
    k = min(8, rows, cols)
    strong = (rng.standard_normal((batch, rows, k)) * 0.5 ** np.arange(k)) @ rng.standard_normal((batch, k, cols))
    return (strong + (0.3 if kind == "noisy" else 0) * rng.standard_normal((batch, rows, cols))) * scale


def room(wn, desc):
    import torch
    return torch.full((wn.wino_orthogonalise_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")


def dtype_of(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def compare(got, g, o_type, steps=5, scale=1.0):
    q = 3 * 2.0 ** -22
    for i in range(len(g)):
        ref, norms = tr.orthogonalise(g[i], steps=steps, scale=scale)
        norms = norms + [np.linalg.norm(ref) / abs(scale)]
        n = max(g[i].shape)
        step = 10.3 * (3 * q + U * (8 + 2 * np.sqrt(n)))
        tol = sum(4.0 ** (steps - k) * step * max(norms[k - 1], norms[k]) for k in range(1, steps + 1)) * abs(scale)
        tol += 2.0 ** -8 * np.linalg.norm(ref) if o_type == "bf16" else 0
        assert np.isfinite(got[i]).all()
        assert np.linalg.norm(got[i] - ref) <= tol, (np.linalg.norm(got[i] - ref), tol, np.linalg.norm(ref))


SHAPES = [(1, 1, 1), (1, 1, 7), (2, 3, 2), (1, 16, 144), (4, 64, 576), (3, 65, 64), (2, 130, 70), (1, 64, 1),
          (2, 100, 333), (1, 200, 129), (1, 128, 1152), (1, 257, 256), (1, 300, 1000)]


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("batch,rows,cols", SHAPES)
def test_shapes(batch, rows, cols, types):
    import torch
    import paper_2004_11077_amd as wn
    gt, ot = types
    g = torch.from_numpy(gradients(batch, rows, cols, rows + cols)).to("cuda", dtype_of(gt))
    o = torch.full((batch, rows, cols), float("nan"), device="cuda").to(dtype_of(ot))
    desc = wn.OrthogonaliseDesc(batch, rows, cols, g_type=TYPES[gt], o_type=TYPES[ot])
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    torch.cuda.synchronize()
    compare(o.double().cpu().numpy(), g.double().cpu().numpy(), ot)
    again = torch.empty_like(o)
    wn.wino_orthogonalise(desc, g, again, room(wn, desc))
    assert torch.equal(o, again)


@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(40, 90), (90, 40), (128, 256)])
def test_strides(rows, cols, type):
    """Rows and matrices apart from each other, at any element; nothing between them is written."""
    import torch
    import paper_2004_11077_amd as wn
    batch, gs, os = 3, cols + 5, cols + 3
    gb, ob = rows * gs + 7, rows * os + 1
    dt = dtype_of(type)
    base = torch.zeros(batch * gb + 3, dtype=dt, device="cuda")
    g = torch.as_strided(base, (batch, rows, cols), (gb, gs, 1), 3)
    g.copy_(torch.from_numpy(gradients(batch, rows, cols, 1)))
    whole = torch.full((batch * ob + 1,), 9.0, device="cuda").to(dt)
    o = torch.as_strided(whole, (batch, rows, cols), (ob, os, 1), 1)
    desc = wn.OrthogonaliseDesc(batch, rows, cols, g_type=TYPES[type], o_type=TYPES[type], g_batch=gb, g_stride=gs, o_batch=ob, o_stride=os)
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    compare(o.double().cpu().numpy(), g.double().cpu().numpy(), type)
    mark = torch.full_like(whole, 9.0)
    torch.as_strided(mark, (batch, rows, cols), (ob, os, 1), 1).copy_(o)
    assert torch.equal(whole, mark)


@pytest.mark.parametrize("steps,scale", [(1, 1.0), (2, -0.5), (3, 0.2), (8, 1.0)])
def test_steps_and_scale(steps, scale):
    import torch
    import paper_2004_11077_amd as wn
    g = torch.from_numpy(gradients(2, 48, 100, 4)).float().cuda()
    o = torch.empty_like(g)
    desc = wn.OrthogonaliseDesc(2, 48, 100, steps=steps, scale=scale)
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    compare(o.double().cpu().numpy(), g.double().cpu().numpy(), "f32", steps=steps, scale=np.float64(np.float32(scale)))


@pytest.mark.parametrize("scale", [1e-25, 1e-3, 1e18, 1e30])
def test_magnitudes(scale):
    """Squares of the entries would under- or overflow fp32; 1e-25 lies far below eps = 1e-30's square."""
    import torch
    import paper_2004_11077_amd as wn
    g = torch.from_numpy(gradients(1, 33, 70, 2, scale=scale)).float().cuda()
    o = torch.empty_like(g)
    eps = 1e-30
    desc = wn.OrthogonaliseDesc(1, 33, 70, eps=eps)
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    ref, norms = tr.orthogonalise(g[0].double().cpu().numpy(), eps=eps)
    step = 10.3 * (9 * 2.0 ** -22 + U * (8 + 2 * np.sqrt(70)))
    tol = sum(4.0 ** (5 - k) * step * max(norms[k - 1], np.linalg.norm(ref)) for k in range(1, 6))
    assert np.linalg.norm(o[0].double().cpu().numpy() - ref) <= tol


def test_zeros_and_values_that_are_no_numbers():
    import torch
    import paper_2004_11077_amd as wn
    g = torch.from_numpy(gradients(4, 40, 70, 6)).float().cuda()
    g[0] = 0
    g[1, 3, 5] = float("nan")
    g[2, 39, 69] = float("inf")
    o = torch.empty_like(g)
    desc = wn.OrthogonaliseDesc(4, 40, 70)
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    assert not o[0].any() and torch.isnan(o[1]).all() and torch.isnan(o[2]).all()
    compare(o[3:].double().cpu().numpy(), g[3:].double().cpu().numpy(), "f32")


def test_a_rank_of_few():
    """Singular values of zero stay zero up to the error of the others."""
    import torch
    import paper_2004_11077_amd as wn
    g = torch.from_numpy(gradients(1, 96, 200, 7, kind="few")).float().cuda()
    o = torch.empty_like(g)
    desc = wn.OrthogonaliseDesc(1, 96, 200)
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    compare(o.double().cpu().numpy(), g.double().cpu().numpy(), "f32")


def test_nothing_to_do():
    import paper_2004_11077_amd as wn
    for shape in ((0, 4, 4), (1, 0, 4), (1, 4, 0)):
        wn.wino_orthogonalise(wn.OrthogonaliseDesc(*shape), None, None, None)
