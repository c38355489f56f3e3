"""Attention over the 8-bit cache where every logit is exact: whole-number queries and codes under scales that are powers of two, and a scale of ln 2, whose product
with log2(e) is 1 in fp32.  What is left are the roundings of the weights and the output, so the bounds are narrow however large the logits are, and a
maximum that is moved wrongly, or a weight beyond fp16's range, shows."""
import math

import numpy as np
import pytest
import torch

import paper_2605_02905_b200 as eosq
from test_gpu_kv8 import DT, HALF_STEP, Pair, _ints

pytestmark = pytest.mark.gpu

LN2 = math.log(2.0)
LEVEL = 56          # channels that carry a token's level; then one that is 1 in every query; the last one, 0 in every query, sets a page's scale


@pytest.fixture(scope="module")
def ctx():
    c = eosq.Context()
    yield c
    c.close()


def _cache(ctx, fmt, d, level, fine, powers, seed):
    """A sequence of len(level) tokens: code `level` in the level channels, `fine` in the next, small ones behind it, page p's scale 2^powers[p]."""
    n, page = len(level), 16
    p = Pair(ctx, pages=n // page + 3, heads=1, page=page, d=d, fmt=fmt, seqs=2, cols=n // page + 2, seed=seed)
    largest = 127.0 if fmt == 0 else 448.0
    g = np.random.RandomState(seed)
    k, v = np.zeros((n, 1, d)), g.randint(-8, 9, (n, 1, d)).astype(np.float64)
    k[:, 0, :LEVEL] = np.asarray(level)[:, None]
    k[:, 0, LEVEL] = fine
    k[:, 0, LEVEL + 1:d - 1] = g.randint(-1, 2, (n, d - LEVEL - 2))
    k[:, 0, d - 1] = largest
    v[:, 0, g.randint(0, d)] = largest
    k *= np.repeat(2.0 ** np.asarray(powers, float), page)[:n, None, None]
    to = lambda x: torch.tensor(x, dtype=torch.float32, device="cuda")
    p.store(0, to(k), to(v), [0], p.reserve([0], [n]), [0, n])
    p.same()
    got = p.m.scale[0][0][p.m.table[0, : -(-n // page)], 0]
    assert np.array_equal(got, 2.0 ** np.asarray(powers, float)[: got.size]) and (p.m.scale[1][0][p.m.table[0, : got.size], 0] == 1).all()
    return p


def _queries(dtype, rows, heads, d, by_row, rest, seed):
    """`by_row`: factors of the level channels, dealt out over rows; the channels behind the fine one take whole numbers up to `rest`."""
    g = np.random.RandomState(seed)
    q = np.zeros((rows, heads, d))
    q[:, :, :LEVEL] = g.choice(by_row, (rows, heads, 1))
    q[:, :, LEVEL] = 1
    q[:, :, LEVEL + 1:d - 1] = g.randint(-rest, rest + 1, (rows, heads, d - LEVEL - 2))
    return torch.tensor(q, device="cuda").to(DT[dtype])


def _hold(ctx, p, q, n, sign=1, **kw):
    """The library's answer against the oracle's: 2^-11 for a weight's rounding to fp16 (whole logits' weights are powers of two and lose nothing) and 2^-20 for its
    2^x, sums of n tokens that truncate once for 16 of them, weights below fp16's normal numbers (off by 2^-25 once and again where they are rescaled,
    the largest being held at 2^6 or more) times a code of at most 448, and the output's rounding.  Nothing for the logits."""
    rows, heads, _ = q.shape
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.zeros((rows, heads), dtype=torch.float32, device="cuda")
    eosq.eosq_kv8_attend(ctx, p.c, 0, q, _ints([0]), _ints([0, rows]), rows, scale=sign * LN2, out=out, lse=lse, **kw)
    assert eosq.eosq_kv8_check(ctx, p.c) == 0
    want, z, size, _, tiny = p.m.attend(0, q.double().cpu().numpy(), [0], [0, rows], sign * LN2, kw.get("causal", True), kw.get("window", 0))
    got, lg = out.double().cpu().numpy(), lse.double().cpu().numpy()
    bound = (2.0 ** -11 + 2.0 ** -20 + n / 16 * 2.0 ** -23) * size + (448 * 2.0 ** -30 * tiny)[..., None] + HALF_STEP[q.dtype] * np.abs(want) + 2.0 ** -25
    assert (bound <= 1e-2 * size.max(-1, keepdims=True)).all()      # it is narrow
    assert np.isfinite(got).all()
    off = float((np.abs(got - want) / bound).max())
    assert off <= 1.0
    # m - 6 + log2 of the sum, times ln 2: three roundings, 2^-24 each, of numbers no larger than that
    assert (np.abs(lg - z) <= 2.0 ** -22 * np.abs(z) + 2.0 ** -18).all()


@pytest.mark.parametrize("rows", [1, 4, 150])
@pytest.mark.parametrize("fmt,d,dtype", [(0, 128, "f16"), (1, 64, "bf16")])
@pytest.mark.parametrize("power", [4, 8, 16, 20, 22, 24, 25, 26, 27, 28, 30, 33, 36, 44, 60, 80])
def test_logits_that_become_large_in_a_later_tile(ctx, power, fmt, d, dtype, rows):
    """Two tiles of tokens with logits of ordinary size, then pages of ever larger ones, some rows' at the same place, others' later or never."""
    n, g = 700, np.random.RandomState(power)
    level = np.where(np.arange(n) < 256, 0, g.randint(-3, 4, n))
    start = power - 17                                              # 2048 * 56 is near 2^17
    powers = np.where(np.arange(-(-n // 16)) < 16, 0, np.minimum(np.maximum(start + np.arange(-(-n // 16)) // 14, -60), 63))
    p = _cache(ctx, fmt, d, level, g.randint(-8, 9, n), powers, power)
    q = _queries(dtype, rows, 3, d, [2048, -2048, 1024, 2, 0], 3, power)
    _hold(ctx, p, q, n)
    _hold(ctx, p, q, n, causal=False)
    _hold(ctx, p, q, n, sign=-1)
    _hold(ctx, p, q, n, window=400)


@pytest.mark.parametrize("rows", [1, 4, 150])
@pytest.mark.parametrize("fmt,d,dtype", [(0, 64, "bf16"), (1, 128, "f16")])
@pytest.mark.parametrize("power", range(-4, 9))
def test_large_logits_close_to_one_another(ctx, power, fmt, d, dtype, rows):
    """Logits near 2^(23.7 + power) that lie a few of fp32's steps, and so up to the slack of the maximum and a little more, from one another; later ones are larger."""
    n, g = 500, np.random.RandomState(100 + power)
    fine = np.minimum(np.sort(g.randint(-8, 9, n)) + g.randint(-2, 3, n), 8)
    p = _cache(ctx, fmt, d, np.full(n, 120), fine, np.full(-(-n // 16), power), power + 50)
    for factors in ([2048], [-2048], [2048, 1, 0]):
        q = _queries(dtype, rows, 3, d, factors, 0, power + 50)
        _hold(ctx, p, q, n)
        _hold(ctx, p, q, n, causal=False, sign=-1)


@pytest.mark.parametrize("rows", [1, 4, 150])
@pytest.mark.parametrize("fmt,d,dtype", [(0, 128, "f16"), (1, 64, "bf16"), (0, 64, "f16"), (1, 128, "bf16")])
@pytest.mark.parametrize("way", ["up", "down", "up_and_down", "steps", "at_random"])
def test_maxima_that_move_often(ctx, way, fmt, d, dtype, rows):
    """Logits of ordinary size that grow from page to page, by less and by more than the slack, so that maxima move at a tile's beginning, in its middle, under weights
    that have been made already, and in many tiles of a row tile; that become smaller again, so that nothing later counts; and any mixture."""
    n, g = 900, np.random.RandomState(7)
    pages = -(-n // 16)
    at = np.arange(pages) / pages
    powers = np.floor({"up": -6 + 18 * at, "down": 12 - 18 * at, "up_and_down": 12 - 36 * np.abs(at - 0.5), "steps": np.where(np.arange(pages) % 8 < 5, -4, -4 + 16 * at),
                       "at_random": g.uniform(-6, 12, pages)}[way]).astype(int)
    level = np.where(g.rand(n) < 0.3, g.randint(-3, 4, n), 0)
    p = _cache(ctx, fmt, d, level, g.randint(-8, 9, n), powers, 3)
    q = _queries(dtype, rows, 3, d, [2, -2, 1, 0], 3, 5)
    _hold(ctx, p, q, n)
    _hold(ctx, p, q, n, causal=False)
    _hold(ctx, p, q, n, sign=-1)
    _hold(ctx, p, q, n, window=500)
