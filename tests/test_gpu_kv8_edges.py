"""The 8-bit paged cache on the GPU at the edges of what its calls take."""
import math

import numpy as np
import pytest
import torch

import paper_2605_02905_b200 as eosq
from test_gpu_kv8 import Pair, _ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = eosq.Context()
    yield c
    c.close()


@pytest.mark.parametrize("fmt,d", [(0, 128), (1, 64)])
@pytest.mark.parametrize("rows", [3, 40])
def test_bf16_queries_from_the_smallest_to_the_largest(ctx, fmt, d, rows):
    """Rows whose largest value is anything that bf16 holds, under a scale that brings the logits back: each is held to fp16's precision by its own power of two."""
    p = Pair(ctx, pages=30, heads=1, page=16, d=d, fmt=fmt, seqs=2, cols=20, seed=1)
    p.append([0], [100], "f32")
    base = torch.randn((rows, 5, d), generator=p.gen, device="cuda").clamp(-3, 3)
    for power in (127, 126, 120, 117, 116, 115, 114, 113, 100, -100, -112, -113, -120, -126, -130):
        q = (base.double() * 2.0 ** (power - 2)).bfloat16()      # the largest is 2^-1 .. 3 of 2^(power - 2)
        assert bool(torch.isfinite(q).all()) and float(q.abs().max()) > 0
        q[0, 1] = q[0, 1] * 2.0 ** -60 if power > 0 else q[0, 1]     # small rows, and none, beside them
        q[1, 2] = 0.0
        p.attend(q, [0], [0, rows], scale=2.0 ** -max(min(power, 120), -120))
        p.attend(q, [0], [0, rows], scale=-(2.0 ** -max(min(power, 120), -120)), causal=False)
    top = torch.finfo(torch.bfloat16).max
    q = torch.full((rows, 5, d), top, device="cuda").bfloat16() * torch.sign(base).bfloat16()
    p.attend(q, [0], [0, rows], scale=1e-39)


def test_fork_with_a_padded_list(ctx):
    """More entries than the cache has sequences, most of them padding: the others are served as in a short list."""
    p = Pair(ctx, layers=2, pages=30, heads=2, page=16, d=64, seqs=6, cols=6, seed=3)
    p.append([0, 1], [40, 17])
    src, dst = [-1] * 700, [-1] * 700
    for i, a, b in ((3, 0, 2), (40, 1, 4), (41, -1, 5), (500, 0, -1), (698, 1, 3)):
        src[i], dst[i] = a, b
    eosq.eosq_kv8_fork(ctx, p.c, _ints(src), _ints(dst))
    p.m.fork(src, dst)
    p.same()


@pytest.mark.parametrize("bad", [-1, 30, 2 ** 31 - 1])
def test_fork_of_a_sequence_with_a_page_outside_the_pool(ctx, bad):
    """A whole page, or the last one, which would be copied: the copy names none there, counts add up, and a page taken for a copy is free again."""
    for col in (0, 2):
        p = Pair(ctx, layers=2, pages=30, heads=2, page=16, d=64, seqs=6, cols=6, seed=3)
        p.append([0, 1], [40, 17])
        p.same()
        good = int(p.c.table[0, col])
        p.c.table[0, col] = bad
        eosq.eosq_kv8_fork(ctx, p.c, _ints([0, 1]), _ints([2, 3]))
        assert eosq.eosq_kv8_check(ctx, p.c) == eosq.EOSQ_KV8_BAD_PAGE
        p.m.fork([0, 1], [2, 3])
        if col == 2:
            p.m.refs[p.m.table[2, col]] = 0
            for x in p.m.code + p.m.scale:   # (nothing was copied there)
                x[:, p.m.table[2, col]] = 0
        else:
            p.m.refs[good] -= 1
        taken = int(p.m.table[2, col])
        p.m.table[2, col] = -1
        p.c.table[0, col] = good
        if col == 2:
            for x in (p.c.k, p.c.v, p.c.k_scale, p.c.v_scale):
                x[:, taken] = 0
        p.same()
        eosq.eosq_kv8_free(ctx, p.c, _ints([2, 3, 0, 1]))
        p.m.free([2, 3, 0, 1])
        p.same()
        assert int(p.c.refs.sum()) == 0


def test_offsets_that_go_back_over_and_over(ctx):
    """Between entries of padding every entry claims all rows again: 4096 x 32 row tiles x 1026 units x 20 heads are 2.7e9, which 32 bits do not hold (the bound on
    a call's units goes by its rows).  Nothing is done, and a flag says so; the next call is answered."""
    n, total = 8192, 511
    p = Pair(ctx, pages=1030, heads=20, page=128, d=64, seqs=2, cols=1024, seed=3)
    p.reserve([0], [1024 * 128])
    p.append([1], [200])
    q = torch.randn((total, 20, 64), generator=p.gen, device="cuda").half()
    out = torch.full_like(q, 3.0)
    seqs, cu = _ints([0, -1] * (n // 2)), _ints([0, total] * (n // 2) + [0])
    eosq.eosq_kv8_attend(ctx, p.c, 0, q, seqs, cu, total, causal=False, out=out)
    assert eosq.eosq_kv8_check(ctx, p.c) == eosq.EOSQ_KV8_BAD_SEQ and bool((out == 3.0).all())
    p.attend(q[:3], [1], [0, 3])


def test_dimensions_of_one_with_any_stride(ctx):
    """One token, or one head, whose stride is no multiple of 16 bytes: torch calls such a tensor contiguous, and the stride is never used."""
    p = Pair(ctx, pages=12, heads=1, page=16, d=64, seqs=2, cols=6, seed=3)
    odd = lambda n, dtype=torch.float16: torch.randn((n, 1, 64), generator=p.gen, device="cuda").to(dtype).as_strided((n, 1, 64), (64 if n > 1 else 65, 1, 1))
    assert odd(1).is_contiguous() and odd(1).stride() == (65, 1, 1)
    for n in (1, 20):
        p.store(0, odd(n), odd(n), [0], p.reserve([0], [n]), [0, n])
    p.same()
    for n in (1, 5):
        q = odd(n)
        out = torch.empty((n, 1, 64), dtype=torch.float16, device="cuda").as_strided((n, 1, 64), q.stride())
        p.attend(q, [0], [0, n], out=out)
