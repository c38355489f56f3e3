"""Exponents of attention's weights over the 8-bit cache, on the CPU: under scores of every size a tile ends after one more look, no weight passes fp16's
range, and what is weighed is the distance to the maximum."""
import ctypes
import os
import re
import subprocess
from pathlib import Path

import numpy as np
import pytest

HERE = Path(__file__).resolve().parent
CSRC = HERE.parent / "paper_2605_02905_b200" / "csrc"


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    so = tmp_path_factory.mktemp("kv8") / "kv8_exponents_probe.so"
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                           "--expt-relaxed-constexpr", "-I", str(CSRC), "-I", str(HERE.parent / "include"), "-o", str(so), str(HERE / "kv8_exponents_probe.cu")])
    lib = ctypes.CDLL(str(so))

    def tile(scores, ks, vlog, look, m):
        rows = scores.shape[0]
        s, k, v = (np.ascontiguousarray(x, np.float32) for x in (scores, ks, vlog))
        m, exps = np.array(m, np.float32), np.zeros((rows, 128), np.float32)
        looks = lib.probe_tile(*(ctypes.c_void_p(x.ctypes.data) for x in (s, k, v)), rows, int(look), *(ctypes.c_void_p(x.ctypes.data) for x in (m, exps)))
        return looks, m, exps

    return tile


@pytest.mark.parametrize("power", list(range(2, 41)) + [60, 80, 100])
def test_a_tile_that_is_much_louder_than_those_before(probe, power):
    """Maxima of ordinary size, then scores of 2^power in a tile that nothing is hidden in.  Exponents stay at 14 (half a step more where a product is not
    rounded before it meets the maximum, below 2^22), and are x - m + 6 up to the roundings of numbers as large as x."""
    r = np.random.RandomState(power)
    for turn in range(60):
        rows = int(r.randint(1, 33))
        scores = r.randn(rows, 128) * 3
        at = r.randint(0, 128, rows)
        scores[np.arange(rows), at] = 2.0 ** power * r.uniform(0.5, 1.0, rows) * r.choice([1.0, 1.0, -1.0], rows)
        if turn % 3 == 0:   # all of them
            scores = 2.0 ** power * r.uniform(-1.0, 1.0, (rows, 128))
        ks, vlog = r.uniform(0.5, 1.0, 8), r.uniform(-4, 4, 8)
        before = r.uniform(0, 20, rows).astype(np.float32)
        looks, m, exps = probe(scores, ks, vlog, False, before)
        assert looks <= 3
        assert np.isfinite(exps).all() and exps.max() <= 14.5
        assert (m >= before).all()
        s32, k32, v32 = (np.repeat(x.astype(np.float32).astype(np.float64), n, -1) for x, n in ((scores, 1), (ks, 16), (vlog, 16)))
        x = s32 * k32 + v32
        # (up to five roundings of numbers no larger than these, by 2^-24 of each: vlog + 6, that less m, with the product; then what m moves by, and its addition)
        assert (np.abs(exps - (x - m[:, None].astype(np.float64) + 6)) <= 5 * 2.0 ** -24 * (np.abs(x) + np.abs(m)[:, None] + 10)).all()


@pytest.mark.parametrize("power", list(range(18, 41)) + [90])
def test_scores_just_beyond_the_maximum(probe, power):
    """A maximum m of that size, and scores that are a few of fp32's steps, or up to the slack of 8, away from it: the maximum moves or the weights fit."""
    r = np.random.RandomState(power)
    one = np.ones(8)
    for _ in range(200):
        m = np.float32(2.0 ** power * r.uniform(1.0, 2.0) * r.choice([1.0, -1.0]))
        step = float(np.spacing(np.abs(m)))
        near = np.float64(m) + np.array([0, 8, -8, 7, 9] + [k * step for k in range(-3, 4)] + [r.uniform(-20, 20) for _ in range(20)])
        scores = np.full((1, 128), -np.inf)
        scores[0, : near.size] = near.astype(np.float32)
        for look in (False, True):
            looks, got, exps = probe(scores, one, 0 * one, look, [m])
            e = exps[np.isfinite(exps)]
            assert looks <= 3 and e.max() <= 14.5 and e.max() >= 5.0 - step   # (a maximum moves by whole powers of two: up to 1 beyond the largest)
            back = got[0].astype(np.float64) + e - 6
            if abs(got[0]) > 2.0 ** 22:
                assert np.array_equal(back, scores[0, : near.size])


def test_no_loop_over_a_tile_goes_back():
    """What bounds the loops of the warps that make weights is that each of them only counts up."""
    code = re.sub(r"//[^\n]*", "", (CSRC / "eosq_kv8_attend_tc.cu").read_text())
    code = code[code.index("if (warp < LOADER)"):code.index("else if (warp < ISSUER)")]
    for m in re.finditer(r"for \(int (\w+) = |for \(; (\w+) <", code):
        name = m.group(1) or m.group(2)
        assert not re.search(r"\b%s\s*-=|\b%s--|--%s\b" % (name, name, name), code), name
