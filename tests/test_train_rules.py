"""The GPU tests of large tiles name the tiles that their cases are to run on: checked against the library's rules, so
that a rule that moves cannot leave a tile untested."""
import test_gpu_large_tiles as large
from test_host_indexing import needs_hipcc, run_host_program

pytestmark = needs_hipcc


def rules(tmp_path, cases):
    out = run_host_program(tmp_path, "train_rules", [str(v) for case in cases for v in case])
    n = len(out) // len(cases)
    assert n * len(cases) == len(out)
    return [tuple(int(v) for v in out[i:i + n]) for i in range(0, len(out), n)]


def test_cross_entropies_run_the_tiles_they_name(tmp_path):
    shapes = [shape for shape, _ in large.LOSSES]
    got = rules(tmp_path, [("loss", T, D, V, int(type == "bf16"), piece) for T, D, V, type, piece in shapes])
    assert [g[1:7] for g in got] == [sides for _, sides in large.LOSSES]
    logits, dl, dh, dw = set(), set(), set(), set()
    for (T, D, V, type, piece), (size, first, last, side, side_h, side_w, last_w, ranges, ranges_w, two) in zip(shapes, got):
        four, pieces = D % 4 == 0, size < V
        logits |= {(type, first), (type, last)}
        dl |= {(type, side), (type, side, bool(two))}
        dh |= {(type, side_h, four, ranges > 1 or pieces), (type, side_h, "pieces", pieces)}
        dw |= {(type, side_w, four), (type, last_w, four)}
    for type in ("f32", "bf16"):
        for side in (128, 256):
            assert (type, side) in logits and (type, side) in dl
            assert (type, side, "pieces", True) in dh
            for four in (False, True):
                assert (type, side, four) in dw
                assert (type, side, four, False) in dh and (type, side, four, True) in dh
    assert ("bf16", 256, True) in dl and ("bf16", 256, False) in dl


def test_updates_run_the_tiles_they_name(tmp_path):
    shapes = [shape for shape, _ in large.UPDATES]
    got = rules(tmp_path, [("update", *shape) for shape in shapes])
    assert got == [sides for _, sides in large.UPDATES]
    assert {(g[2], g[3] > 1) for g in got if not g[0]} == {(64, True), (128, False), (128, True)}
    assert {g[1] for g in got} == {0, 1}
    assert {(g[4], shape[1] > shape[2]) for g, shape in zip(got, shapes)} >= {(side, tall) for side in (128, 256) for tall in (False, True)}
