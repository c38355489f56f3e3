"""The 8-bit paged cache on the GPU against the oracle in 64 bits: codes, scales, tables and counts are equal, attention lies within what its
roundings allow."""
import math

import numpy as np
import pytest
import torch

import kv8_oracle as o
import paper_2605_02905_b200 as eosq

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    c = eosq.Context()
    yield c
    c.close()


def _ints(v):
    return torch.tensor(list(map(int, v)), dtype=torch.int32, device="cuda")


class Pair:
    """A cache on the GPU and its model, taken through the same calls."""

    def __init__(self, ctx, *, layers=1, pages=40, heads=2, page=16, d=64, fmt=0, seqs=6, cols=20, seed=0):
        self.ctx, self.fmt = ctx, fmt
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.c = eosq.Kv8Cache.allocate(layers, pages, heads, page, d, fmt, seqs, cols)
        self.m = o.Model(layers, pages, heads, page, d, fmt, seqs, cols)
        # memory that nobody has written: bytes of every kind, also those that are no e4m3 number, and scales that are none
        for which, name in enumerate("kv"):
            x = torch.randint(0, 256, self.c.k.shape, generator=self.gen, device="cuda", dtype=torch.uint8)
            x[..., 1::3] = 0x7f
            x[..., 2::3] = 0xff
            getattr(self.c, name).copy_(x)
            self.m.code[which][:] = x.cpu().numpy()
            getattr(self.c, name + "_scale").fill_(float("nan"))
            self.m.scale[which][:] = np.nan

    def tokens(self, total, dtype="f16", loud=1.0, strided=False):
        c = self.c
        x = torch.randn((total, 2 * c.kv_heads + 1, c.d), generator=self.gen, device="cuda") * loud
        x = (x * torch.exp(torch.randn((total, 1, 1), generator=self.gen, device="cuda"))).to(DT[dtype])
        k, v = x[:, :c.kv_heads], x[:, c.kv_heads:2 * c.kv_heads]
        return (k, v) if strided else (k.contiguous(), v.contiguous())

    def reserve(self, seqs, add):
        got = eosq.eosq_kv8_reserve(self.ctx, self.c, _ints(seqs), _ints(add))
        want = self.m.reserve(seqs, add)
        assert got.tolist() == want
        return want

    def store(self, layer, k, v, seqs, first, cu, most=None, **kw):
        most = max(b - a for a, b in zip(cu, cu[1:])) if most is None else most
        eosq.eosq_kv8_store(self.ctx, self.c, layer, k, v, _ints(seqs), _ints(first), _ints(cu), most, **kw)
        self.m.store(layer, k.double().cpu().numpy(), v.double().cpu().numpy(), seqs, first, cu)

    def append(self, seqs, add, dtype="f16", loud=1.0, strided=False):
        """Room for new tokens, and the tokens, in every layer."""
        first = self.reserve(seqs, add)
        cu = np.concatenate([[0], np.cumsum(add)]).tolist()
        for layer in range(self.c.layers):
            self.store(layer, *self.tokens(cu[-1], dtype, loud, strided), seqs, first, cu)

    def same(self, flags=0):
        c, m = self.c, self.m
        torch.cuda.synchronize()
        for which, name in enumerate("kv"):
            assert np.array_equal(getattr(c, name).cpu().numpy(), m.code[which]), name
            assert np.array_equal(getattr(c, name + "_scale").double().cpu().numpy(), m.scale[which], equal_nan=True), name + "_scale"
        assert c.table.tolist() == m.table.tolist() and c.lengths.tolist() == m.lengths.tolist() and c.refs.tolist() == m.refs.tolist()
        assert m.flags == flags and eosq.eosq_kv8_check(self.ctx, c) == flags
        m.flags = 0

    def attend(self, q, seqs, cu, *, layer=0, scale=None, causal=True, window=0, out=None, most=None, **kw):
        """The library's answer, held to the oracle's; rows of no entry keep what was there."""
        total, H, d = q.shape
        scale = 1.0 / math.sqrt(d) if scale is None else scale
        most = max(b - a for a, b in zip(cu, cu[1:])) if most is None else most
        out = torch.full((total, H, d), 7.0, dtype=q.dtype, device="cuda") if out is None else out.fill_(7.0)
        lse = torch.full((total, H), 5.0, dtype=torch.float32, device="cuda")
        eosq.eosq_kv8_attend(self.ctx, self.c, layer, q, _ints(seqs), _ints(cu), most, scale=scale, causal=causal, window=window, out=out, lse=lse, **kw)
        assert eosq.eosq_kv8_check(self.ctx, self.c) == 0
        hold(self.m, q, seqs, cu, out, lse, layer, scale, causal, window)
        return out, lse


def hold(model, q, seqs, cu, out, lse, layer, scale, causal, window):
    want, z, size, reach, tiny = model.attend(layer, q.double().cpu().numpy(), seqs, cu, scale, causal, window)
    got, lg = out.double().cpu().numpy(), lse.double().cpu().numpy()
    mine = np.zeros(q.shape[0], bool)
    for i, s in enumerate(seqs):
        if s != -1:
            mine[cu[i]:cu[i + 1]] = True
    assert (got[~mine] == 7.0).all() and (lg[~mine] == 5.0).all()
    want, z, size, reach, tiny, got, lg = (x[mine] for x in (want, z, size, reach, tiny, got, lg))
    none = np.isinf(z)
    assert (lg[none] == -np.inf).all() and (got[none] == 0).all()
    # A weight's exponent x, in fp32, is off by its sum over d (truncated products and sums: 2^-16 of sum |q k| is generous) and by the roundings of
    # its parts, each below 256 (a few of 2^-17).  A weight is rounded to fp16: by 2^-11 of itself, or, with the largest one's product with its scale
    # held at 2^6 or more, by 2^-31 of that, times a code of at most 448.  Sums over keys truncate, 2^-23 each time, once for 16 keys.  The
    # output is rounded to its type.
    slop = 2.0 ** -16 * (reach * math.log2(math.e) + 1.0)
    keys = float(model.lengths.max())
    bound = (2.0 ** -11 + 2 * slop + keys / 16 * 2.0 ** -23)[..., None] * size + (448 * 2.0 ** -31 * tiny)[..., None] + HALF_STEP[q.dtype] * np.abs(want) + 2.0 ** -25
    far = np.abs(got - want)[~none] / bound[~none]
    assert far.size == 0 or far.max() <= 1.0, far.max()
    off = np.abs(lg[~none] - z[~none])
    assert off.size == 0 or (off <= 2 * slop[~none] + 2.0 ** -22 * np.abs(z[~none])).all(), off.max()


# ---- writing ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype,d,page,heads,strided", [("f16", 64, 16, 1, False), ("f16", 128, 64, 3, True), ("bf16", 128, 16, 2, True), ("bf16", 64, 128, 1, False),
                                                        ("f32", 64, 32, 3, True), ("f32", 128, 128, 2, False)])
def test_store(ctx, fmt, dtype, d, page, heads, strided):
    p = Pair(ctx, pages=60, heads=heads, page=page, d=d, fmt=fmt, seqs=5, cols=12, seed=d + page)
    p.append([3, 0, 4], [page + 1, 1, 2 * page - 1], dtype, 0.1, strided)
    p.same()
    p.append([0, 4], [0, 1], dtype, 3.0, strided)            # nothing for one, the page's last token for the other
    p.append([4, 3, 0, 1], [1, page - 1, 1, 5 * page + 3], dtype, 0.01, strided)
    p.same()
    for step in range(7):                                    # token by token: scales grow, older codes follow
        p.append([1, 0, 3, 4], [1, 1, 1, 1], dtype, 1.5 ** step * 0.05, strided)
    p.same()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_store_of_values_at_the_borders(ctx, fmt, dtype):
    p = Pair(ctx, pages=8, heads=1, page=32, d=64, fmt=fmt, seqs=3, cols=3, seed=5)
    x = torch.zeros((32, 1, 64), device="cuda")
    x[0] = torch.linspace(-127, 127, 64, device="cuda")[None]            # scale 1 of int8: halves in the rows below
    x[1] = torch.arange(64, device="cuda")[None] + 0.5
    x[2] = -x[1]
    x[3] = 448 / 3.5 - x[1]
    x[4] = 2.0 ** torch.linspace(-20, 6, 64, device="cuda").round()[None]
    x[5, 0, ::2], x[5, 0, 1::2] = float("nan"), float("inf")
    x[6, 0, ::2], x[6, 0, 1::2] = float("-inf"), -0.0
    x[7] = 1e-30
    x[8:] = torch.randn((24, 1, 64), generator=p.gen, device="cuda") * 40
    x = x.to(DT[dtype])
    p.store(0, x, -x, [0], p.reserve([0], [32]), [0, 32])
    p.same()
    for v in (float("nan"), 0.0, 1e-7, 6e4, float("inf")) + ((3e38,) if dtype != "f16" else ()):
        y = torch.full((3, 1, 64), v, device="cuda").to(DT[dtype])       # pages with nothing finite, nothing, little and much in them; from nothing to much
        p.store(0, y, -y, [1], p.reserve([1], [3]), [0, 3])
        p.same()


@pytest.mark.parametrize("fmt", [0, 1])
def test_store_rounds_quotients_as_if_exact(ctx, fmt):
    """Many values under scales with full mantissas: one wrong half among them would show."""
    p = Pair(ctx, pages=40, heads=2, page=128, d=128, fmt=fmt, seqs=1, cols=40, seed=9)
    p.append([0], [40 * 128], "f32")
    p.same()


def test_entries_that_make_no_sense_are_skipped(ctx):
    p = Pair(ctx, pages=20, heads=2, page=16, d=64, seqs=4, cols=5)
    p.append([0, 1], [20, 30])
    p.same()
    k, v = p.tokens(12)
    call = lambda seqs, first, cu, most: eosq.eosq_kv8_store(ctx, p.c, 0, k, v, _ints(seqs), _ints(first), _ints(cu), most)
    for seqs, first, cu, most in (([4], [0], [0, 4], 4), ([-2], [0], [0, 4], 4), ([0], [17], [0, 4], 4), ([0], [0], [0, 13], 13), ([0], [0], [-1, 4], 9),
                                  ([0], [0], [4, 2], 9), ([0], [0], [0, 8], 4)):
        call(seqs, first, cu, most)
        torch.cuda.synchronize()
        p.m.flags = eosq.EOSQ_KV8_BAD_SEQ
        p.same(eosq.EOSQ_KV8_BAD_SEQ)
    call([-1, 0], [0, -1], [0, 4, 8], 4)      # padding, and an entry that got no room
    p.same()
    for bad in (-1, 20, 2 ** 31 - 1):
        p.c.table[0, 1] = bad
        call([0], [16], [0, 4], 4)
        q = torch.randn((3, 4, 64), device="cuda").half()
        got = eosq.eosq_kv8_attend(ctx, p.c, 0, q, _ints([0, 1]), _ints([0, 1, 3]), 2)
        assert eosq.eosq_kv8_check(ctx, p.c) == eosq.EOSQ_KV8_BAD_PAGE
        assert bool(torch.isfinite(got).all())
        p.c.table[0, 1] = int(p.m.table[0, 1])
    for length in (-5, 81, 2 ** 31 - 1):
        p.c.lengths[0] = length
        got = eosq.eosq_kv8_attend(ctx, p.c, 0, q, _ints([0, 1]), _ints([0, 1, 3]), 2)
        call([0], [16], [0, 4], 4)
        assert eosq.eosq_kv8_check(ctx, p.c) == eosq.EOSQ_KV8_BAD_SEQ
        p.c.lengths[0] = 20
    p.same()
    got = torch.full((3, 4, 64), 3.0, device="cuda").half()
    eosq.eosq_kv8_attend(ctx, p.c, 0, q, _ints([7, 1]), _ints([0, 1, 3]), 1, out=got)   # no such sequence; more queries than announced
    assert eosq.eosq_kv8_check(ctx, p.c) == eosq.EOSQ_KV8_BAD_SEQ and bool((got == 3.0).all())


# ---- attention --------------------------------------------------------------------------------------------------------------

LENGTHS = [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 333]


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype,d,page,heads,G", [("f16", 128, 16, 2, 4), ("bf16", 128, 64, 1, 8), ("f16", 64, 32, 3, 1), ("bf16", 64, 128, 2, 3), ("f16", 128, 128, 1, 16),
                                                  ("bf16", 64, 16, 1, 7)])
def test_attention_of_a_token(ctx, fmt, dtype, d, page, heads, G):
    p = Pair(ctx, pages=130, heads=heads, page=page, d=d, fmt=fmt, seqs=13, cols=21, seed=G)
    p.append(range(12), LENGTHS, dtype)
    n = 13
    q = torch.randn((n + 2, heads * G, d), generator=p.gen, device="cuda").to(DT[dtype])
    seqs = [5, 12, 0, 11, -1, 3, 1, 7, 2, 10, 9, 8, 4]       # an empty sequence, padding, two rows behind the last
    p.attend(q, seqs, list(range(n + 1)))
    p.attend(q, seqs, list(range(n + 1)), causal=False)
    p.attend(q, seqs, list(range(n + 1)), window=1)
    p.attend(q, seqs, list(range(n + 1)), window=70)
    p.attend(q * 30, seqs, list(range(n + 1)), scale=-0.2)   # weights far apart
    p.attend(q, seqs, list(range(n + 1)), scale=0.0)         # all alike


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype,d,page,heads,G,news", [
    ("f16", 128, 16, 2, 4, [1, 0, 3, 40, 5]), ("bf16", 64, 32, 1, 1, [17, 16, 1, 0, 200]), ("bf16", 128, 64, 1, 5, [129, 1, 2, 64, 0]), ("f16", 64, 128, 2, 3, [2, 5, 4, 1, 3]),
    ("f16", 128, 32, 1, 2, [300, 0, 0, 128, 1]), ("bf16", 64, 16, 3, 8, [33, 32, 31, 1, 100]),
])
def test_attention_of_many_queries(ctx, fmt, dtype, d, page, heads, G, news):
    p = Pair(ctx, pages=130, heads=heads, page=page, d=d, fmt=fmt, seqs=6, cols=21, seed=G)
    p.append([4, 0, 2, 1, 3], [300, 1, 40, 64, 131], dtype)
    cu = np.concatenate([[0], np.cumsum(news)]).tolist()
    wide = torch.randn((cu[-1] + 3, heads * G + 2, d), generator=p.gen, device="cuda").to(DT[dtype])
    q, seqs = wide[:, 1:-1], [4, 2, -1, 3, 0]
    out = torch.empty((cu[-1] + 3, heads * G + 1, d), dtype=DT[dtype], device="cuda")[:, 1:]
    p.attend(q, seqs, cu, out=out)            # more queries than tokens in some: rows that see nothing
    p.attend(q, seqs, cu, causal=False)
    p.attend(q, seqs, cu, window=9, most=cu[-1] + 3)
    p.attend(q, seqs, cu, window=150)
    p.attend(q, seqs, cu, scale=-0.3)
    p.attend(q, seqs, cu, scale=0.0, window=77)


@pytest.mark.parametrize("cols,page", [(4, 128), (5, 128), (32, 16)])
@pytest.mark.parametrize("rows,G", [(1, 2), (3, 9), (140, 2)])
def test_attention_where_a_row_of_the_table_is_short(ctx, cols, page, rows, G):
    """Up to 512 tokens to a sequence row tiles are not shared between CTAs; above that they may be."""
    p = Pair(ctx, pages=200, heads=3, page=page, d=64, seqs=5, cols=cols, seed=2)
    p.append([0, 1, 2, 3], [512, 511, 1, 300])
    q = torch.randn((4 * rows, 3 * G, 64), generator=p.gen, device="cuda").half()
    cu = [rows * i for i in range(5)]
    p.attend(q, [3, 0, 1, 2], cu)
    p.attend(q, [3, 0, 1, 2], cu, window=100)
    p.attend(q, [3, 0, 4, 2], cu, causal=False)


@pytest.mark.parametrize("G,d,fmt,dtype", [(4, 128, 0, torch.float16), (1, 64, 1, torch.bfloat16), (9, 64, 0, torch.bfloat16),
                                           (16, 128, 1, torch.float16), (17, 64, 0, torch.float16)])
def test_attention_of_a_chunk_among_single_tokens(ctx, G, d, fmt, dtype):
    """A prompt's chunk with sequences of a few rows: entries at both sides of every border between the kernels, padding, an empty sequence."""
    p = Pair(ctx, pages=160, heads=2, page=32, d=d, fmt=fmt, seqs=24, cols=64, seed=3)
    most = -(-512 // G) + 3
    lens = [1, 2, 31, 32, 33, 127, 128, 129, 300, 700, 5, 64, 90, 200, 17, 3, 256, 40, 77, most + 150]
    p.append(list(range(20)), lens)
    counts = [1] * 11 + [max(1, 8 // G), 8 // G + 1, 16 // G + 1, 2, 1, 1, 0, 1, most]
    seqs = list(range(20))
    seqs[4] = -1
    seqs.insert(9, 22)   # empty
    counts.insert(9, 1)
    cu = [sum(counts[:i]) for i in range(len(counts) + 1)]
    q = torch.randn((cu[-1], 2 * G, d), generator=p.gen, device="cuda").to(dtype)
    p.attend(q, seqs, cu)
    p.attend(q, seqs, cu, window=50)
    p.attend(q, seqs, cu, causal=False)


@pytest.mark.parametrize("counts,most", [([140, 5, 5, 3, 5, 5, 5, 4], None), ([1] * 150, 150), ([2, 0, 1] * 60, 400)])
def test_attention_where_one_kernel_is_left_without_work(ctx, counts, most):
    """A chunk among entries that are too long for the other kernel, and single tokens under a bound of a chunk's length."""
    n = len(counts)
    p = Pair(ctx, pages=2 * n + 40, heads=2, page=16, d=64, seqs=n, cols=40, seed=4)
    p.append(list(range(n)), [max(c, 1) + 7 + i % 20 for i, c in enumerate(counts)])
    cu = [sum(counts[:i]) for i in range(n + 1)]
    q = torch.randn((cu[-1], 2 * 4, 64), generator=p.gen, device="cuda").half()
    p.attend(q, list(range(n)), cu, most=most)


@pytest.mark.parametrize("rows", [1, 40])
def test_attention_over_a_long_cache(ctx, rows):
    """Many CTAs share a row tile; the whole call is one sequence's, or one long one's among short ones."""
    p = Pair(ctx, pages=160, heads=2, page=64, d=128, fmt=1, seqs=4, cols=110, seed=3)
    p.append([0, 1, 2], [7000, 100, 1500])
    q = torch.randn((3 * rows, 8, 128), generator=p.gen, device="cuda").half()
    p.attend(q[:rows], [0], [0, rows])
    p.attend(q, [1, 0, 2], [0, rows, 2 * rows, 3 * rows])
    p.attend(q, [1, 0, 2], [0, rows, 2 * rows, 3 * rows], window=3000)


@pytest.mark.parametrize("fmt", [0, 1])
def test_scales_far_apart(ctx, fmt):
    """Pages whose scales are 2^-40 .. 2^40: the weights take the value scales in and out again; nothing overflows."""
    p = Pair(ctx, pages=30, heads=2, page=16, d=64, fmt=fmt, seqs=2, cols=20, seed=1)
    first = p.reserve([0], [150])
    k, v = p.tokens(150, "f32")
    v = v * torch.exp2(torch.randint(-40, 41, (10, 1, 1, 1), generator=p.gen, device="cuda").float()).expand(10, 15, 1, 1).reshape(150, 1, 1)
    p.store(0, k, v, [0], first, [0, 150])
    p.same()
    q = torch.randn((20, 4, 64), generator=p.gen, device="cuda").bfloat16()
    p.attend(q[:1], [0], [0, 1])
    p.attend(q, [0], [0, 20])


@pytest.mark.parametrize("fmt,d", [(0, 128), (1, 64), (1, 128)])
@pytest.mark.parametrize("every,by", [(16, 1.7), (33, 2.5), (7, 1.3)])
def test_maxima_that_move(ctx, fmt, d, every, by):
    """Keys that get louder on their way: a row's largest score is passed again and again, by a little and by much, at a tile's beginning and within it; and then
    quieter, so that nothing that comes counts."""
    p = Pair(ctx, pages=60, heads=1, page=16, d=d, fmt=fmt, seqs=2, cols=50, seed=every)
    first = p.reserve([0], [700])
    k, v = p.tokens(700, "f32")
    t = torch.arange(700, device="cuda")
    rise = torch.where(t < 400, t, 800 - t) // every
    k = k / k.norm(dim=2, keepdim=True) * torch.clamp(by ** rise.float(), max=3e4)[:, None, None]
    p.store(0, k, v, [0], first, [0, 700])
    for rows in (1, 12, 150):
        q = torch.randn((rows, 3, d), generator=p.gen, device="cuda").half()
        p.attend(q, [0], [0, rows])
        p.attend(q, [0], [0, rows], causal=False, scale=0.5)


def test_queries_of_any_size(ctx):
    """bf16 rows are brought to fp16's range by a power of two of their own; rows of zeros; a row that is not finite spoils itself alone."""
    p = Pair(ctx, pages=30, heads=1, page=16, d=128, fmt=0, seqs=2, cols=20, seed=1)
    p.append([0], [100], "f32")
    for rows in (3, 40):
        q = torch.randn((rows, 5, 128), generator=p.gen, device="cuda").bfloat16()
        q[0, 0], q[1, 1], q[2, 2], q[0, 3] = q[0, 0] * 1e30, q[1, 1] * 1e-30, 0.0, q[0, 3] * 1e5
        out, lse = p.attend(q, [0], [0, rows], scale=1e-3)
        p.attend(q * 1e-30, [0], [0, rows], scale=1e30)
        q[0, 1, 7], q[rows - 1, 2, 3] = float("nan"), float("inf")
        bad, bad_lse = eosq.eosq_kv8_attend(ctx, p.c, 0, q, _ints([0]), _ints([0, rows]), rows, scale=1e-3, want_lse=True)
        ok = torch.ones((rows, 5), dtype=torch.bool, device="cuda")
        ok[0, 1] = ok[rows - 1, 2] = False
        assert bool(torch.isnan(bad[~ok]).all()) and torch.equal(bad[ok], out[ok])
        assert bool(torch.isnan(bad_lse[~ok]).all()) and torch.equal(bad_lse[ok], lse[ok])


def test_same_bits_every_time_and_on_another_stream(ctx):
    p = Pair(ctx, pages=160, heads=2, page=64, d=128, fmt=0, seqs=4, cols=110, seed=3)
    p.append([0, 1, 2], [5000, 777, 1500])
    for rows in (1, 100):
        q = torch.randn((3 * rows, 8, 128), generator=p.gen, device="cuda").half()
        seqs, cu = _ints([1, 0, 2]), _ints([0, rows, 2 * rows, 3 * rows])
        want = eosq.eosq_kv8_attend(ctx, p.c, 0, q, seqs, cu, rows)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = [eosq.eosq_kv8_attend(ctx, p.c, 0, q, seqs, cu, rows, stream=side) for _ in range(5)]
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, want) for x in got)


# ---- pages ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("seed", range(6))
def test_pages_through_many_calls(ctx, seed):
    """Calls drawn at random, entries that have to be refused among them, against the model after each."""
    r = np.random.RandomState(seed)
    layers, heads, page, d = int(r.randint(1, 4)), int(r.randint(1, 4)), int(r.choice([16, 32, 64, 128])), int(r.choice([64, 128]))
    seqs = int(r.choice([3, 12, 40]))
    p = Pair(ctx, layers=layers, pages=int(r.randint(5, 60)), heads=heads, page=page, d=d, fmt=seed & 1, seqs=seqs, cols=8, seed=seed)
    for step in range(40):
        n = int(r.randint(1, seqs + 3))
        some = r.randint(-1, seqs, n).tolist()
        if r.rand() < 0.1:
            some[0] = int(r.choice([-7, seqs, 2 ** 30]))
        kind = r.choice(["reserve", "reserve", "fork", "free", "compact"])
        if kind == "reserve":
            add = r.randint(0, 3 * page, n).tolist()
            if r.rand() < 0.2:
                add[-1] = int(r.choice([-1, 9 * page, 2 ** 31 - 1]))
            p.reserve(some, add)
        elif kind == "fork":
            to = r.permutation(seqs)[:n].tolist() + r.randint(-1, seqs, max(0, n - seqs)).tolist()
            n = min(n, seqs)
            eosq.eosq_kv8_fork(ctx, p.c, _ints(some[:n]), _ints(to[:n]))
            p.m.fork(some[:n], to[:n])
        elif kind == "free":
            eosq.eosq_kv8_free(ctx, p.c, _ints(some[: n // 2 + 1]))
            p.m.free(some[: n // 2 + 1])
        else:
            assert eosq.eosq_kv8_compact(ctx, p.c).tolist() == p.m.compact().tolist()
        p.same(p.m.flags)


@pytest.mark.parametrize("pages", [1, 8191, 8192, 8193, 30000])
def test_a_large_pool(ctx, pages):
    """Prefix sums over more pages than the planning CTA looks at in a step; the free ones at the very end, at the beginning, nowhere."""
    p = Pair(ctx, pages=pages, heads=1, page=16, d=64, seqs=3, cols=pages + 1, seed=1)
    p.reserve([0, 1], [16 * (pages - pages // 4), 16])
    p.reserve([1, 2, 0], [16 * (pages // 4) + 1, 16 * (pages // 8), 1])
    p.same(p.m.flags)
    eosq.eosq_kv8_free(ctx, p.c, _ints([0]))
    p.m.free([0])
    assert eosq.eosq_kv8_compact(ctx, p.c).tolist() == p.m.compact().tolist()
    p.reserve([0], [40])
    p.same(p.m.flags)


def test_copies_between_pools(ctx):
    a, b = Pair(ctx, layers=3, pages=9, heads=3, page=128, d=128, seqs=2, cols=9, seed=1), Pair(ctx, layers=3, pages=14, heads=3, page=128, d=128, seqs=2, cols=9, seed=2)
    src, dst = [3, 3, 8, 0], [13, 0, 1, 7]
    eosq.eosq_kv8_copy_pages(ctx, a.c, b.c, _ints(src), _ints(dst))
    for x, y in zip(a.m.code + a.m.scale, b.m.code + b.m.scale):
        y[:, dst] = x[:, src]
    b.same()
    eosq.eosq_kv8_copy_pages(ctx, b.c, b.c, _ints([5, 6]), _ints([9, 10]))
    for y in b.m.code + b.m.scale:
        y[:, [9, 10]] = y[:, [5, 6]]
    b.same()
    eosq.eosq_kv8_copy_pages(ctx, a.c, b.c, _ints([9, 0, -1]), _ints([0, 14, 3]))    # none of them both in their pools
    b.m.flags = eosq.EOSQ_KV8_BAD_PAGE
    b.same(eosq.EOSQ_KV8_BAD_PAGE)
    a.same()


# ---- together ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt,dtype,G", [(0, "f16", 4), (1, "bf16", 3)])
def test_a_run_as_a_server_makes_it(ctx, fmt, dtype, G):
    """Prompts in chunks, each attending to what came before; tokens one by one; beams; sequences that end; compaction, after which every answer
    is the same to the bit; new prompts in the room that became free."""
    p = Pair(ctx, layers=2, pages=64, heads=2, page=16, d=128, fmt=fmt, seqs=8, cols=16, seed=4)
    q_of = lambda n: torch.randn((n, 2 * G, 128), generator=p.gen, device="cuda").to(DT[dtype])
    for chunk in ([50, 3, 17], [50, 30, 1]):
        p.append([0, 1, 2], chunk, dtype)
        cu = np.concatenate([[0], np.cumsum(chunk)]).tolist()
        for layer in (0, 1):
            p.attend(q_of(cu[-1]), [0, 1, 2], cu, layer=layer)
    eosq.eosq_kv8_fork(ctx, p.c, _ints([0, 0, 2]), _ints([3, 4, 5]))
    p.m.fork([0, 0, 2], [3, 4, 5])
    for step in range(20):
        live = [0, 1, 2, 3, 4, 5]
        p.append(live, [1] * 6, dtype)
        p.attend(q_of(6), live, list(range(7)), layer=step & 1)
    eosq.eosq_kv8_free(ctx, p.c, _ints([0, 2]))
    p.m.free([0, 2])
    p.same()
    q, live = q_of(4), [1, 3, 4, 5]
    before, _ = p.attend(q, live, [0, 1, 2, 3, 4])
    p.m.compact()
    eosq.eosq_kv8_compact(ctx, p.c)
    p.same()
    after, _ = p.attend(q, live, [0, 1, 2, 3, 4])
    assert torch.equal(before, after)
    p.append([0, 3], [90, 1], dtype)
    p.attend(q_of(91), [0, 3], [0, 90, 91], layer=1)
    # an encoder's states, kept in the cache, under a decoder's queries of any number
    p.append([7], [61], dtype)
    p.attend(q_of(75), [7], [0, 75], causal=False)
    p.same()


def test_a_captured_step_follows_the_cache(ctx):
    """Room, store, attention and fork in a graph, replayed with other tokens and lengths, beside a second graph with a workspace of its own on another stream."""
    p = Pair(ctx, pages=80, heads=2, page=16, d=64, seqs=6, cols=20, seed=8)
    p.append([0, 1, 4], [100, 15, 33])
    k, v = p.tokens(2)
    q = torch.randn((2, 4, 64), generator=p.gen, device="cuda").half()
    seqs, add, cu = _ints([0, 1]), _ints([1, 1]), _ints([0, 1, 2])
    first, outs = torch.zeros(2, dtype=torch.int32, device="cuda"), [torch.zeros_like(q) for _ in range(2)]
    ws = [torch.empty(eosq.eosq_kv8_workspace_bytes(p.c, 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    warm = eosq.Kv8Cache.allocate(1, 4, 2, 16, 64, 0, 6, 3)   # first calls load kernels: not while capturing
    eosq.eosq_kv8_reserve(ctx, warm, seqs, add, first=first)
    eosq.eosq_kv8_store(ctx, warm, 0, k, v, seqs, first, cu, 1)
    eosq.eosq_kv8_attend(ctx, warm, 0, q, seqs, cu, 1, out=outs[0], workspace=ws[0])
    torch.cuda.synchronize()
    step, look = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(step):
        eosq.eosq_kv8_reserve(ctx, p.c, seqs, add, first=first)
        eosq.eosq_kv8_store(ctx, p.c, 0, k, v, seqs, first, cu, 1)
        eosq.eosq_kv8_attend(ctx, p.c, 0, q, seqs, cu, 1, out=outs[0], workspace=ws[0])
    other = _ints([4, 4])
    with torch.cuda.graph(look):
        eosq.eosq_kv8_attend(ctx, p.c, 0, q, other, cu, 1, out=outs[1], workspace=ws[1])
    side = torch.cuda.Stream()
    for turn in range(5):
        nk, nv = p.tokens(2)
        k.copy_(nk)
        v.copy_(nv)
        q.copy_(torch.randn((2, 4, 64), generator=p.gen, device="cuda"))
        side.wait_stream(torch.cuda.current_stream())
        step.replay()
        with torch.cuda.stream(side):
            look.replay()
        torch.cuda.current_stream().wait_stream(side)
        want = p.m.reserve([0, 1], [1, 1])
        assert first.tolist() == want
        p.m.store(0, k.double().cpu().numpy(), v.double().cpu().numpy(), [0, 1], want, [0, 1, 2])
        p.same()
        for out, at in ((outs[0], [0, 1]), (outs[1], [4, 4])):
            _, lse = eosq.eosq_kv8_attend(ctx, p.c, 0, q, _ints(at), cu, 1, want_lse=True)
            hold(p.m, q, at, [0, 1, 2], out, lse, 0, 1 / 8, True, 0)
