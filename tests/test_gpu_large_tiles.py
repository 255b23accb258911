"""Cross entropies and updates on the tiles that large ones take, 128 and 256 to a side, at ragged sizes that take
them too: products that are few but long in one direction, or many small ones.  Each case names the tiles it is to
run on, which are held to the library's rules on the CPU (test_train_rules.py).  Tolerances: those derived in the
operators' own tests.
"""
import numpy as np
import pytest

from test_gpu_cross_entropy import TYPES, check, run
from test_gpu_orthogonalise import compare, dtype_of, gradients, room

pytestmark = pytest.mark.gpu

# ((rows, features, classes, type, piece), (sides of the tiles of the logits of the first piece and of the last, of dl, of
# dh, of dW of the first piece and of the last))
LOSSES = [
    ((655, 64, 4676, "f32", 0), (128, 128, 128, 64, 64, 64)),
    ((7083, 65, 1754, "f32", 0), (256, 256, 256, 64, 64, 64)),
    ((1250, 2459, 131, "f32", 0), (32, 32, 32, 128, 64, 64)),
    ((6505, 480, 131, "f32", 0), (64, 64, 64, 128, 64, 64)),
    ((334, 1903, 2481, "f32", 2048), (64, 32, 64, 128, 128, 64)),
    ((3805, 144, 2100, "f32", 2048), (128, 64, 128, 128, 64, 64)),
    ((1561, 1928, 261, "f32", 256), (32, 32, 32, 128, 64, 64)),
    ((7633, 1785, 191, "f32", 0), (64, 64, 64, 256, 64, 64)),
    ((5117, 2500, 129, "f32", 0), (64, 64, 64, 256, 64, 64)),
    ((3874, 132, 7707, "f32", 0), (256, 256, 256, 256, 64, 64)),
    ((6385, 142, 5427, "f32", 0), (128, 128, 128, 256, 64, 64)),
    ((208, 2264, 1355, "f32", 0), (32, 32, 32, 64, 128, 128)),
    ((202, 394, 7400, "f32", 0), (64, 64, 64, 64, 128, 128)),
    ((198, 2725, 4837, "f32", 0), (64, 64, 64, 128, 256, 256)),
    ((206, 2620, 5811, "f32", 0), (64, 64, 64, 128, 256, 256)),
    ((203, 2832, 1890, "f32", 1280), (32, 32, 32, 64, 128, 64)),
    ((8147, 1912, 442, "f32", 256), (64, 64, 64, 256, 64, 64)),
    ((1100, 772, 4100, "f32", 0), (64, 64, 64, 128, 128, 128)),
    ((2100, 2052, 4200, "f32", 2304), (64, 128, 64, 256, 64, 128)),
    ((452, 70, 6287, "bf16", 0), (128, 128, 128, 64, 64, 64)),
    ((3005, 73, 4318, "bf16", 0), (256, 256, 256, 64, 64, 64)),
    ((3000, 64, 4352, "bf16", 0), (256, 256, 256, 64, 64, 64)),
    ((6574, 479, 128, "bf16", 0), (64, 64, 64, 128, 64, 64)),
    ((6090, 516, 133, "bf16", 0), (64, 64, 64, 128, 64, 64)),
    ((1361, 2236, 346, "bf16", 256), (64, 32, 64, 128, 64, 64)),
    ((6298, 160, 1374, "bf16", 1024), (128, 64, 128, 128, 64, 64)),
    ((1265, 66, 11411, "bf16", 0), (256, 256, 256, 128, 64, 64)),
    ((5442, 2349, 142, "bf16", 0), (64, 64, 64, 256, 64, 64)),
    ((7334, 1700, 132, "bf16", 256), (64, 64, 64, 256, 64, 64)),
    ((2938, 2151, 1389, "bf16", 1280), (128, 64, 128, 256, 64, 64)),
    ((4041, 132, 7623, "bf16", 0), (256, 256, 256, 256, 64, 64)),
    ((157, 335, 8672, "bf16", 0), (64, 64, 64, 64, 128, 128)),
    ((129, 1568, 2006, "bf16", 0), (64, 64, 64, 64, 128, 128)),
    ((219, 2204, 1643, "bf16", 1536), (64, 32, 64, 64, 128, 64)),
    ((137, 2345, 5734, "bf16", 0), (64, 64, 64, 64, 256, 256)),
    ((145, 1220, 10326, "bf16", 0), (64, 64, 64, 64, 256, 256)),
    ((145, 1280, 10326, "bf16", 0), (64, 64, 64, 64, 256, 256)),
    ((2300, 1088, 6200, "bf16", 0), (256, 256, 256, 128, 128, 128)),
]
# ((batch, rows, cols), (whether A and whether P takes tiles of 32, side of A's tiles, ranges of its k, side of X's tiles))
UPDATES = [
    ((65, 1109, 33), (0, 1, 128, 2, 64)),
    ((11, 300, 400), (0, 0, 128, 1, 64)),
    ((3, 515, 1100), (0, 0, 64, 2, 64)),
    ((1, 1300, 1400), (0, 0, 128, 2, 64)),
    ((3, 512, 1600), (0, 0, 64, 3, 64)),
    ((202, 66, 75), (0, 0, 128, 1, 128)),
    ((203, 84, 69), (0, 0, 128, 1, 128)),
    ((21, 198, 2330), (0, 0, 64, 2, 256)),
    ((228, 216, 196), (0, 0, 128, 1, 256)),
    ((1, 2000, 520), (0, 0, 64, 4, 64)),
]


@pytest.mark.parametrize("case", [c[0] for c in LOSSES], ids=str)
def test_cross_entropy(case):
    T, D, V, type, piece = case
    check(run(T, D, V, type, seed=T, piece=piece), type)


@pytest.mark.parametrize("T,D,V,type", [(6505, 480, 131, "f32"), (3874, 132, 7707, "f32"), (208, 2264, 1355, "f32"), (206, 2620, 5811, "f32"),
                                        (6090, 516, 133, "bf16"), (7334, 1700, 132, "bf16"), (129, 1568, 2006, "bf16"), (145, 1220, 10326, "bf16")])
def test_gradients_that_start_at_any_element(T, D, V, type):
    """Sizes whose gradients are stored four values at a time, where they start on whole fours."""
    import torch
    import paper_2004_11077_amd as wn
    r = run(T, D, V, type)
    dt = dtype_of(type)
    cuda = lambda a, *t: torch.from_numpy(a).to("cuda", *t)
    h, w, b, target, lse = cuda(r["h"], dt), cuda(r["w"], dt), cuda(r["b"]), cuda(r["target"]), cuda(r["lse"], torch.float32)
    dloss = cuda(r["dloss"], torch.float32)
    whole = [torch.full((1 + rows * D + 9,), 7, device="cuda").to(dt) for rows in (T, V)]
    dh, dw = (t[1:1 + rows * D].view(rows, D) for t, rows in zip(whole, (T, V)))
    desc = wn.LossDesc(T, D, V, type=TYPES[type])
    ws = torch.full((wn.wino_linear_cross_entropy_backward_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    dbias = torch.empty(V, device="cuda")
    wn.wino_linear_cross_entropy_backward(desc, h, w, b, target, lse, dloss, dh, dw, dbias, ws)
    r["dh"], r["dw"], r["dbias"] = (t.double().cpu().numpy() for t in (dh, dw, dbias))
    check(r, type)
    for t in whole:
        assert t[0] == 7 and (t[-9:] == 7).all()


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("batch,rows,cols", [c[0] for c in UPDATES])
def test_updates(batch, rows, cols, types):
    import torch
    import paper_2004_11077_amd as wn
    gt, ot = types
    g = torch.from_numpy(gradients(batch, rows, cols, rows + cols)).to("cuda", dtype_of(gt))
    o = torch.full((batch, rows, cols), float("nan"), device="cuda").to(dtype_of(ot))
    desc = wn.OrthogonaliseDesc(batch, rows, cols, g_type=TYPES[gt], o_type=TYPES[ot])
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    got, g = o.double().cpu().numpy(), g.double().cpu().numpy()
    some = np.unique(np.linspace(0, batch - 1, 24).astype(int))       # in 64 bits; of the others, that they have values
    assert np.isfinite(got).all()
    compare(got[some], g[some], ot)
