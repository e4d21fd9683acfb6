"""How the cross entropy's products are cut (csrc/vocab_plan.hpp), on the host: the sizes of tests/vocab_cases.py take the
tiles that they are there for, and between them every tile that any size takes."""
import ctypes
import os
import subprocess

import pytest

import vocab_cases as C

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_05233_amd", "csrc")
WRAPPER = """
#include "vocab_plan.hpp"
using namespace mesa::vocab;
extern "C" void plan(int64_t rows, int64_t vocab, int64_t width, int dtype, int64_t* out) {
  const GradPlan g(rows, vocab, width, dtype, !may_lie(width, dtype));
  const ForwardPlan f(rows, vocab, width, dtype);
  const int planes = logit_planes(dtype);
  const int64_t at_once = streams(rows, planes) ? vocab : copy_rows(vocab, width, dtype);
  const int64_t x[] = {shape_of(at_once, rows, width, planes), ceil_div(vocab, at_once), g.logits, g.dh.shape, g.dh.layers,
                       g.de.shape, g.de.layers, g.de_last.shape, g.de_last.layers, ceil_div(vocab, g.piece), g.piece, g.sorts, f.bytes, grad_bytes(rows, vocab, width, dtype)};
  for (int i = 0; i < 14; ++i) out[i] = x[i];
}
"""
FIELDS = ("forward", "copies", "logits", "dh", "dh_layers", "de", "de_layers", "last", "last_layers", "pieces", "piece", "sorts", "forward_bytes",
          "bytes")
SHAPES = "WMNT"


def build(directory):
    src, lib = directory / "plan.cpp", directory / "plan.so"
    src.write_text(WRAPPER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fPIC", "-shared", "-I" + CSRC, "-o", str(lib), str(src)], check=True)
    p, i64 = ctypes.CDLL(str(lib)), ctypes.c_int64
    p.plan.argtypes, p.plan.restype = [i64, i64, i64, ctypes.c_int, ctypes.POINTER(i64)], None

    def plan(rows, vocab, width, dtype):
        out = (i64 * len(FIELDS))()
        p.plan(rows, vocab, width, dtype, out)
        r = dict(zip(FIELDS, out))
        return {k: SHAPES[v] if k in ("forward", "logits", "dh", "de", "last") else v for k, v in r.items()}

    return plan


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return build(tmp_path_factory.mktemp("vocab_plan"))


@pytest.mark.parametrize("case", C.TILES)
def test_tiles(plan, case):
    p = plan(*case[:4])
    assert (p["forward"], p["logits"], "%s%d" % (p["dh"], p["dh_layers"]), "%s%d" % (p["de"], p["de_layers"])) == case[4:]


@pytest.mark.parametrize("case", C.PIECES)
def test_pieces(plan, case):
    p = plan(*case[:4])
    assert (p["copies"], p["pieces"]) == case[4:]
    assert p["pieces"] == 1 or 0 < case[1] - (p["pieces"] - 1) * p["piece"] < p["piece"]


def _taken(p, dtype):
    return {(dtype, "forward", p["forward"], False), (dtype, "logits", p["logits"], False), (dtype, "dh", p["dh"], p["dh_layers"] > 1),
            (dtype, "de", p["de"], p["de_layers"] > 1)}


def test_every_tile_is_tested(plan):
    """What a spread of sizes takes is what the tested ones take."""
    tested = set().union(*(_taken(plan(*c[:4]), c[3]) for c in C.TILES))
    for dtype in (C.F32, C.BF16):
        for rows in (1, 20, 33, 70, 150, 300, 777, 1500, 4000, 9000, 16384):
            for vocab in (40, 300, 1201, 5003, 16003, 50257, 128000):
                for width in (16, 72, 200, 320, 768, 1000, 2048, 4096):
                    missing = _taken(plan(rows, vocab, width, dtype), dtype) - tested
                    assert not missing, (rows, vocab, width, missing)


@pytest.mark.parametrize("dtype", [C.F32, C.BF16])
@pytest.mark.parametrize("cap", [0.0, 7.0])
@pytest.mark.parametrize("rows", [30, 1030])
def test_reference(dtype, cap, rows):
    """The device's reference is the oracle's, and so are its bounds."""
    pytest.importorskip("torch")
    import numpy as np
    from oracle import language_ends as E
    h, table, targets, up = C.problem(rows, 50, 24, dtype, 1, "cpu")
    out, bound = C.reference(h, table, targets, up, cap, rows <= 1024)
    nh, nt, t, u = (x.double().numpy() for x in (h, table, targets, up))
    t = t.astype(np.int64)
    want, want_bound = dict(E.cross_entropy(nh, nt, t, cap), **E.cross_entropy_backward(nh, nt, t, u, cap)), E.cross_entropy_bounds(
        nh, nt, t, u, cap, dtype == C.BF16)
    for n in ("lse", "loss", "dh", "dtable", "best"):
        assert np.allclose(out[n].numpy(), want[n], rtol=1e-9, atol=1e-13), n
    for n in ("lse", "loss", "dh", "dtable"):
        assert np.allclose(bound[n].numpy(), want_bound[n], rtol=1e-6, atol=1e-30), n
