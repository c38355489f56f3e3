"""The operators of the 8-bit paged cache, as cases that can be timed and compared.

The cache holds keys and values as one byte per number, in pages of ``page`` tokens; every page has, for each KV head, one fp32
scale for its keys and one for its values.  A number is its code times its scale; a code is a signed integer of -127 .. 127
("int8") or an e4m3 number ("e4m3").  ``kind`` says which operator a case passes through:

  store    new tokens' keys and values into the pages that ``reserve`` gave them: eosq_kv8_store.  A page's scale is
           a / 127 (int8) or the least power of two with a <= 448 times it (e4m3), a being the largest finite magnitude among
           its new tokens; a page that held tokens before keeps the larger scale, and its codes are brought to it.
  attend   attention of new queries over the cached tokens: eosq_kv8_attend.  A sequence's queries are its last positions;
           ``causal`` lets a query see its own and earlier positions, ``window`` the last so many of them only; without
           ``causal`` each sees every token (cross attention to an encoder's states).
  beam     one step of a beam search: eosq_kv8_free of the beams that were dropped, eosq_kv8_fork of the kept ones into
           their place, eosq_kv8_reserve of room for the next tokens.  Whole pages are shared, the last one is copied.
  compact  eosq_kv8_compact: the used pages move to the front of the pool, tables and counts follow.

Plain forms are in 32 bits; where a value is next to a rounding border they are in 64.
"""
from __future__ import annotations

import math
import random

import torch

own = False

F = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
SCALE_MIN, SCALE_MAX = 2.0 ** -64, 2.0 ** 64


def _store(name, fmt, dtype, n, lo, hi, heads, d, page, *, held=0, strided=False):
    """n sequences get lo .. hi new tokens each; they held up to ``held`` before."""
    return dict(name=name, kind="store", fmt=fmt, dtype=dtype, n=n, lo=lo, hi=hi, heads=heads, d=d, page=page, held=held, strided=strided)


def _attend(name, fmt, dtype, n, qlo, qhi, lo, hi, heads, G, d, page, *, causal=True, window=0, lse=False, strided=False):
    """n sequences of lo .. hi cached tokens, the last qlo .. qhi of which are the queries' positions; G query heads per KV head."""
    return dict(name=name, kind="attend", fmt=fmt, dtype=dtype, n=n, qlo=qlo, qhi=qhi, lo=lo, hi=hi, heads=heads, G=G, d=d, page=page,
                causal=causal, window=window, lse=lse, strided=strided)


def _beam(name, fmt, n, lo, hi, add, layers, heads, d, page):
    return dict(name=name, kind="beam", fmt=fmt, n=n, lo=lo, hi=hi, add=add, layers=layers, heads=heads, d=d, page=page)


def _compact(name, fmt, n, lo, hi, used, layers, heads, d, page):
    """n sequences; ``used`` of the pool's pages, in percent, hold something."""
    return dict(name=name, kind="compact", fmt=fmt, n=n, lo=lo, hi=hi, used=used, layers=layers, heads=heads, d=d, page=page)


def listed():
    return [
        # one layer of a decoding step of 64 sequences: a token each, into pages that are mostly begun
        _store("store_token_64", "int8", "bf16", 64, 1, 1, 8, 128, 64, held=2000),
        # a few short prompts of a small model kept in fp32
        _store("store_short_fp32_d64", "e4m3", "f32", 5, 1, 200, 3, 64, 16, held=37),
        # one layer of a prefill of 32k tokens in four prompts, keys and values still inside the fused projection's output
        _store("store_prefill_32k", "e4m3", "f16", 4, 2048, 14336, 8, 128, 64, strided=True),
        # the first steps of a single conversation: latency
        _attend("attend_token_short", "int8", "f16", 1, 1, 1, 300, 300, 8, 4, 128, 64),
        # a decoding step of a server: many lengths at once
        _attend("attend_token_ragged", "e4m3", "bf16", 48, 1, 1, 64, 8192, 8, 4, 128, 16, lse=True),
        # a decoding step over long contexts, the memory-bound end
        _attend("attend_token_long", "int8", "f16", 16, 1, 1, 32768, 32768, 8, 4, 128, 64),
        # a prompt's chunk of 128 tokens against the 32k before it
        _attend("attend_chunk_32k", "int8", "f16", 1, 128, 128, 32768, 32768, 8, 4, 128, 64),
        # prompts of several lengths side by side, the compute-bound end
        _attend("attend_prefill", "e4m3", "bf16", 4, 500, 2048, 2048, 12000, 8, 4, 128, 64, strided=True),
        # a decoder's tokens against an encoder's 1500 states, heads of 64
        _attend("attend_cross_d64", "int8", "f16", 24, 1, 60, 1500, 1500, 6, 1, 64, 32, causal=False),
        # a beam search of 32 beams
        _beam("beam_32", "int8", 32, 500, 4000, 1, 8, 8, 128, 64),
        # a small pool with a quarter in use
        _compact("compact_small", "e4m3", 7, 20, 300, 25, 2, 3, 64, 16),
        # a server's pool of 1 MB pages, half in use
        _compact("compact_pool", "int8", 24, 200, 2500, 50, 8, 8, 128, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = _drawn(rng)
    del case["name"]
    return case


def _drawn(rng):
    kind = rng.choice(["store", "store", "attend", "attend", "attend", "attend", "beam", "compact"])
    fmt, d, page = rng.choice(["int8", "e4m3"]), rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    heads, G = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8])
    if kind == "store":
        n = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, 32768 // n))
        return _store("", fmt, rng.choice(["f16", "bf16", "f32"]), n, rng.randint(1, hi), hi, heads, d, page, held=rng.choice([0, 5, 700]), strided=rng.random() < 0.5) | {"salt": rng.randrange(10 ** 6)}
    if kind == "attend":
        n = _log(rng, 1, 64)
        hi = _log(rng, 1, max(2, min(32768, 500000 // n)))
        lo = rng.randint(max(1, hi // 20), hi)
        causal = rng.random() < 0.75
        dtype = rng.choice(["f16", "bf16"])
        qhi = 1
        if rng.random() < 0.5:
            most = max(1, min(2048, 4 * 10 ** 8 // (n * hi * heads * G)))
            qhi = _log(rng, 1, min(most, hi) if causal else most)
        return _attend("", fmt, dtype, n, rng.randint(1, qhi), qhi, lo, hi, heads, G, d, page, causal=causal,
                       window=rng.choice([0, 0, 1, 100, 1024]) if causal else 0, lse=rng.random() < 0.5, strided=rng.random() < 0.5) | {"salt": rng.randrange(10 ** 6)}
    if kind == "beam":
        return _beam("", fmt, _log(rng, 1, 48), _log(rng, 1, 500), _log(rng, 500, 4000), rng.choice([1, 1, 7, 100]), rng.randint(1, 8), heads, d, page) | {"salt": rng.randrange(10 ** 6)}
    return _compact("", fmt, _log(rng, 1, 24), _log(rng, 1, 200), _log(rng, 200, 2500), rng.randint(10, 95), rng.randint(1, 8), heads, d, page) | {"salt": rng.randrange(10 ** 6)}


# ---- sizes that follow from a case alone ------------------------------------------------------------------------------

def _spread(case, n, lo, hi):
    """n lengths from lo to hi, spread over their logarithm, in an order of the case's own; the ends are among them."""
    v = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * (i / (n - 1) if n > 1 else 1.0)))) for i in range(n)]
    random.Random(str(sorted((k, v) for k, v in case.items() if k != "name"))).shuffle(v)
    return v


def _sizes(case):
    """(tokens held in all, tokens of this call) of every sequence."""
    n = case["n"]
    if case["kind"] == "store":
        new = _spread(case, n, case["lo"], case["hi"])
        held = _spread(case, n, 1, case["held"]) if case["held"] else [0] * n
        return [a + b for a, b in zip(held, new)], new
    if case["kind"] == "attend":
        held = _spread(case, n, case["lo"], case["hi"])
        new = _spread({**case, "q": 1}, n, case["qlo"], case["qhi"])
        return held, [min(a, b) for a, b in zip(new, held)] if case["causal"] else new
    held = _spread(case, n, min(case["lo"], case["hi"]), case["hi"])
    return held, [case.get("add", 0)] * n


def _pairs(case):
    """(query, visible token) pairs per head, and the tokens per head that any query sees."""
    pairs = seen = 0
    for total, q in zip(*_sizes(case)):
        if not case["causal"]:
            pairs, seen = pairs + q * total, seen + total
            continue
        w = case["window"] or total
        pairs += sum(min(p + 1, w) for p in range(total - q, total))
        seen += min(total, q + w - 1)
    return pairs, seen


def work(case):
    held, new = _sizes(case)
    page, d, heads = case["page"], case["d"], case["heads"]
    tokens = sum(new)
    if case["kind"] == "store":
        pages = sum(-(-t // page) - (t - m) // page for t, m in zip(held, new))
        return {"bytes": 2 * tokens * heads * d * (BYTES[case["dtype"]] + 1) + 2 * pages * heads * 4, "flops": 4 * tokens * heads * d}
    if case["kind"] == "attend":
        pairs, seen = _pairs(case)
        H = heads * case["G"]
        rows = 2 * tokens * H * d * BYTES[case["dtype"]] + (4 * tokens * H if case["lse"] else 0)
        return {"bytes": 2 * seen * heads * d + 8 * heads * (seen // page) + rows, "flops": 4 * pairs * H * d}
    row = 2 * case["layers"] * heads * (page * d + 4)   # one page, all layers, keys and values
    if case["kind"] == "beam":
        copied = sum(1 for t in held if t % page)
        return {"bytes": 2 * copied * row + 12 * sum(-(-t // page) for t in held), "flops": 0}
    moved = _pool(case)[1]
    return {"bytes": 2 * moved * row + 8 * (_pool(case)[0] + sum(-(-t // page) for t in held)), "flops": 0}


def _pool(case):
    """(pages of the pool, pages that a compaction moves): the used ones lie where a shuffle of the case's own puts them."""
    used = sum(-(-t // case["page"]) for t in _sizes(case)[0])
    pages = max(used + 1, used * 100 // case["used"])
    order = list(range(pages))
    random.Random(pages * 1000 + used).shuffle(order)
    return pages, sum(1 for p in order[:used] if p >= used)


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _codes(gen, fmt, shape):
    """Codes of keys or values: about normal, a few channels larger, as in a cache."""
    out = torch.empty(shape, dtype=torch.uint8, device="cuda")
    flat = out.view(-1, shape[-1])
    loud = torch.where(torch.rand(shape[-1], generator=gen, device="cuda") < 0.05, 3.0, 1.0)
    x = torch.randn(flat.shape, generator=gen, device="cuda") * loud
    if fmt == "int8":
        flat.view(torch.int8).copy_((x * 18).round_().clamp_(-127, 127))
    else:
        flat.view(torch.float8_e4m3fn).copy_((x * 64).clamp_(-448, 448))
    return out


def _scales(gen, fmt, shape):
    s = torch.exp(0.5 * torch.randn(shape, generator=gen, device="cuda")) * (0.05 if fmt == "int8" else 0.015)
    return s if fmt == "int8" else torch.exp2(torch.log2(s).round())


_ctx = None


def _handle(state, case):
    """The library's handle on the state's buffers, which a program makes once."""
    global _ctx
    import paper_2605_02905_b200 as eosq
    if _ctx is None:
        _ctx = eosq.Context()
    fmt = eosq.EOSQ_KV_INT8 if case["fmt"] == "int8" else eosq.EOSQ_KV_E4M3
    return _ctx, eosq.Kv8Cache(k=state["k"], v=state["v"], k_scale=state["k_scale"], v_scale=state["v_scale"], table=state["table"],
                               lengths=state["lengths"], refs=state["refs"], format=fmt)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    n, page, d, heads, fmt = case["n"], case["page"], case["d"], case["heads"], case["fmt"]
    held, new = _sizes(case)
    layers = case.get("layers", 1)
    kind = case["kind"]
    after = [t + (case["add"] if kind == "beam" else 0) for t in held]
    need = [-(-t // page) for t in held]
    width = max(-(-t // page) for t in after) + 1
    seqs = 2 * n if kind == "beam" else n
    if kind == "compact":
        pages = _pool(case)[0]
        order = list(range(pages))
        random.Random(pages * 1000 + sum(need)).shuffle(order)
        order = torch.tensor(order, dtype=torch.int32, device="cuda")
    else:
        pages = sum(need) + (sum(-(-a // page) for a in after) if kind == "beam" else 3)
        order = torch.randperm(pages, generator=gen, device="cuda").int()
    cols = torch.arange(width, device="cuda")
    rows = _ints(need)[:, None]
    start = torch.cumsum(rows, 0) - rows
    table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
    table[:n] = torch.where(cols[None] < rows, order[(start + cols[None]).clamp(max=pages - 1).long()], -1)
    lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    lengths[:n] = _ints(held)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order[: sum(need)].long()] = 1
    st = dict(case=dict(case), table=table, lengths=lengths, refs=refs)
    shape = (layers, pages, heads, page, d)
    for name in ("k", "v"):
        st[name] = _codes(gen, fmt, shape)
        st[name + "_scale"] = _scales(gen, fmt, shape[:3])
    st["seqs"] = torch.arange(n, dtype=torch.int32, device="cuda")
    if kind in ("store", "attend"):
        # the last tokens of every sequence are this call's
        cu = [0]
        for m in new:
            cu.append(cu[-1] + m)
        st["cu"], st["most"], total = _ints(cu), max(new), cu[-1]
        H = heads * case.get("G", 1)
        fused = torch.randn((total, H + 2 * heads, d), generator=gen, device="cuda") if case["strided"] else None
        dt = F[case["dtype"]]

        def take(a, b):
            return fused[:, a:b].to(dt) if case["strided"] else torch.randn((total, b - a, d), generator=gen, device="cuda").to(dt)
        if case["strided"]:
            fused = fused.to(dt)
        if kind == "attend":
            st["q"] = fused[:, :H] if case["strided"] else take(0, H)
        else:
            st["first"] = st["lengths"] - _ints(new)
            if case["strided"]:
                st["xk"], st["xv"] = fused[:, H:H + heads], fused[:, H + heads:]
            else:
                st["xk"], st["xv"] = take(H, H + heads), take(H + heads, H + 2 * heads)
            for name in ("xk", "xv"):   # tokens of different loudness, as rows of a cache are
                st[name].mul_(torch.exp(0.5 * torch.randn((total, 1, 1), generator=gen, device="cuda")).to(dt))
    if kind == "beam":
        parents = torch.randint(0, n, (n,), generator=gen, device="cuda")
        st["src"], st["dst"] = st["seqs"][parents].contiguous(), st["seqs"] + n
        st["add"] = torch.full((n,), case["add"], dtype=torch.int32, device="cuda")
    if kind == "compact":
        st["table0"], st["refs0"] = table.clone(), refs.clone()
    if own:
        st["ctx"], st["cache"] = _handle(st, case)
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _seen_as(case, codes):
    return codes.view(torch.int8 if case["fmt"] == "int8" else torch.float8_e4m3fn)


def run(st):
    case = st["case"]
    return {"store": _run_store, "attend": _run_attend, "beam": _run_beam, "compact": _run_compact}[case["kind"]](st, case)


def _run_store(st, case):
    if own:
        import paper_2605_02905_b200 as eosq
        eosq.eosq_kv8_store(st["ctx"], st["cache"], 0, st["xk"], st["xv"], st["seqs"], st["first"], st["cu"], st["most"])
    else:
        _plain_store(st, case, "k", st["xk"])
        _plain_store(st, case, "v", st["xv"])
    return {"k": _seen_as(case, st["k"]), "v": _seen_as(case, st["v"]), "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _scale_of(fmt, a):
    """The scale for a largest magnitude a (fp32)."""
    if fmt == "int8":
        return (a.double() / 127).float().clamp(SCALE_MIN, SCALE_MAX)
    m, e = torch.frexp(a)                       # a = m 2^e, m in [0.5, 1): 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(a > 0, torch.exp2(e.float()), 0.0).clamp(SCALE_MIN, SCALE_MAX)


def _quantised(fmt, x):
    """Codes of x, values over their scale in 64 bits."""
    if fmt == "int8":
        return torch.nan_to_num(x, 0.0, 127.0, -127.0).round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return torch.nan_to_num(x, 0.0, 448.0, -448.0).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_store(st, case, name, x):
    page, fmt, heads = case["page"], case["fmt"], case["heads"]
    codes, scale = st[name][0], st[name + "_scale"][0]
    total = x.shape[0]
    t = torch.arange(total, device="cuda")
    i = torch.searchsorted(st["cu"].long(), t, right=True) - 1
    pos = st["first"].long()[i] + t - st["cu"].long()[i]
    where, slot = st["table"][st["seqs"].long()[i], pos // page].long(), pos % page
    x = x.float()
    a = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    top = torch.zeros_like(scale).scatter_reduce(0, where[:, None].expand(-1, heads), a, "amax")
    touched = torch.zeros(scale.shape[0], dtype=torch.bool, device="cuda").index_fill(0, where, True)
    # a sequence's first page is the only one that may have held tokens
    before = st["first"].long() % page
    tail = st["table"][st["seqs"].long(), st["first"].long() // page].long()
    begun = torch.zeros(scale.shape[0], dtype=torch.bool, device="cuda")
    begun[tail] = before > 0
    fresh = _scale_of(fmt, top)
    after = torch.where(touched[:, None], torch.where(begun[:, None], torch.maximum(scale, fresh), fresh), scale)
    old = codes[tail]
    ratio = (scale[tail].double() / after[tail].double())[:, :, None, None]
    values = _seen_as(case, old).float().double()
    if fmt == "int8":
        again = _quantised(fmt, values * scale[tail].double()[:, :, None, None] / after[tail].double()[:, :, None, None])
    else:
        again = _quantised(fmt, values * ratio)
    kept = (torch.arange(page, device="cuda")[None] < before[:, None])[:, None, :, None] & (after[tail] > scale[tail])[:, :, None, None]
    codes[tail] = torch.where(kept, again, old)
    codes[where, :, slot] = _quantised(fmt, x.double() / after[where][:, :, None].double())
    scale.copy_(after)


def _padded(st, rows, most):
    """[n, most] row indices of a ragged list and which of them exist."""
    at = torch.arange(most, device="cuda")
    live = at[None] < (st["cu"][1:] - st["cu"][:-1])[:, None]
    return (st["cu"][:-1, None].long() + at[None]).clamp(max=rows - 1), live


def _gathered(st, case, name, pages):
    """[n, heads, tokens, d] values of the sequences' pages, fp32."""
    x = _seen_as(case, st[name][0][pages]).float() * st[name + "_scale"][0][pages][..., None, None]
    n, P, heads, page, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, heads, P * page, d)


def _run_attend(st, case):
    q, most = st["q"], st["most"]
    scale = 1.0 / math.sqrt(case["d"])
    if own:
        import paper_2605_02905_b200 as eosq
        got = eosq.eosq_kv8_attend(st["ctx"], st["cache"], 0, q, st["seqs"], st["cu"], most, scale=scale, causal=case["causal"],
                                   window=case["window"], want_lse=case["lse"])
        return {"out": got[0], "lse": got[1]} if case["lse"] else {"out": got}
    n, heads, G, d, page = case["n"], case["heads"], case["G"], case["d"], case["page"]
    total, H = q.shape[:2]
    at, live = _padded(st, total, most)
    used = (st["lengths"] + page - 1) // page
    pages = st["table"][st["seqs"].long()][:, : -(-max(_sizes(case)[0]) // page)]
    pages = torch.where(torch.arange(pages.shape[1], device="cuda")[None] < used[:, None], pages, 0).long()
    Q = q[at].float().view(n, most, heads, G, d).permute(0, 2, 3, 1, 4).reshape(n, heads, G * most, d)
    s = (Q * scale) @ _gathered(st, case, "k", pages).transpose(-1, -2)
    L = s.shape[-1]
    length = st["lengths"][st["seqs"].long()].long()
    j = torch.arange(L, device="cuda")
    ok = (j[None, None] < length[:, None, None]).expand(n, most, L)
    if case["causal"]:
        pos = (length - (st["cu"][1:] - st["cu"][:-1]))[:, None] + torch.arange(most, device="cuda")[None]
        ok = ok & (j[None, None] <= pos[..., None])
        if case["window"]:
            ok = ok & (j[None, None] > pos[..., None] - case["window"])
    s = s.view(n, heads, G, most, L).masked_fill(~ok[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    w = (s - top).exp()
    total_w = w.sum(-1, keepdim=True)
    o = (w.view(n, heads, G * most, L) @ _gathered(st, case, "v", pages)).view(n, heads, G, most, d) / torch.where(total_w > 0, total_w, 1.0)
    out = torch.zeros((total, H, d), dtype=q.dtype, device="cuda")
    out[at[live]] = o.permute(0, 3, 1, 2, 4).reshape(n, most, H, d)[live].to(q.dtype)
    if not case["lse"]:
        return {"out": out}
    lse = torch.zeros((total, H), dtype=torch.float32, device="cuda")
    lse[at[live]] = (top + total_w.log())[..., 0].permute(0, 3, 1, 2).reshape(n, most, H)[live]
    return {"out": out, "lse": lse}


def _free_pages(refs):
    """The pool's pages, the free ones first, each part in ascending order; and how many are free."""
    return torch.argsort((refs != 0).int(), stable=True)


def _plain_free(st, seqs):
    rows = st["table"][seqs]
    st["refs"].index_add_(0, rows.clamp(min=0).reshape(-1).long(), -(rows >= 0).int().reshape(-1))
    st["table"][seqs] = -1
    st["lengths"][seqs] = 0


def _plain_fork(st, page, src, dst):
    length = st["lengths"][src]
    rows, cols = st["table"][src], torch.arange(st["table"].shape[1], device="cuda")
    full, tail = (length // page)[:, None], (length % page > 0)
    shared = cols[None] < full
    st["refs"].index_add_(0, rows.clamp(min=0).reshape(-1).long(), shared.int().reshape(-1))
    fresh = _free_pages(st["refs"])[(torch.cumsum(tail.int(), 0) - tail.int()).long()].int()
    last = (cols[None] == full) & tail[:, None]
    st["table"][dst] = torch.where(shared, rows, torch.where(last, fresh[:, None], -1))
    st["lengths"][dst] = length
    to, of = fresh[tail].long(), rows[last].long()
    st["refs"][to] = 1
    for name in ("k", "v", "k_scale", "v_scale"):
        st[name][:, to] = st[name][:, of]


def _plain_reserve(st, page, seqs, add):
    length = st["lengths"][seqs]
    have, want = (length + page - 1) // page, (length + add + page - 1) // page
    cols = torch.arange(st["table"].shape[1], device="cuda")
    new = (cols[None] >= have[:, None]) & (cols[None] < want[:, None])
    need = want - have
    rank = (torch.cumsum(need, 0) - need)[:, None] + cols[None] - have[:, None]
    pages = _free_pages(st["refs"])[rank.clamp(0, st["refs"].shape[0] - 1).long()].int()
    st["table"][seqs] = torch.where(new, pages, st["table"][seqs])
    st["refs"][pages[new].long()] = 1
    st["lengths"][seqs] = length + add
    return length


def _run_beam(st, case):
    if own:
        import paper_2605_02905_b200 as eosq
        eosq.eosq_kv8_free(st["ctx"], st["cache"], st["dst"])
        eosq.eosq_kv8_fork(st["ctx"], st["cache"], st["src"], st["dst"])
        first = eosq.eosq_kv8_reserve(st["ctx"], st["cache"], st["dst"], st["add"])
    else:
        _plain_free(st, st["dst"].long())
        _plain_fork(st, case["page"], st["src"].long(), st["dst"].long())
        first = _plain_reserve(st, case["page"], st["dst"].long(), st["add"])
    return {"first": first, **_everything(st, case)}


def _everything(st, case):
    return {"k": st["k"], "v": st["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"], "table": st["table"], "lengths": st["lengths"],
            "refs": st["refs"]}


def _run_compact(st, case):
    st["table"].copy_(st["table0"])   # the next pass finds the same holes; the pages that move are where they were
    st["refs"].copy_(st["refs0"])
    if own:
        import paper_2605_02905_b200 as eosq
        remap = eosq.eosq_kv8_compact(st["ctx"], st["cache"])
    else:
        refs = st["refs"]
        at = torch.arange(refs.shape[0], device="cuda")
        live = refs > 0
        front = at < live.sum()
        to, of = at[~live & front], at[live & ~front]
        remap = torch.where(live, at, -1).int()
        remap[of] = to.int()
        for name in ("k", "v", "k_scale", "v_scale"):
            st[name][:, to] = st[name][:, of]
        refs[to] = refs[of]
        refs[of] = 0
        st["table"].copy_(torch.where(st["table"] >= 0, remap[st["table"].clamp(min=0).long()], -1))
    return {"remap": remap, **_everything(st, case)}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------

def _exact_grid(fmt, y):
    """The nearest value that a code can stand for, half to even, y in 64 bits."""
    y = torch.where(torch.isnan(y), 0.0, y)
    if fmt == "int8":
        return torch.round(y.clamp(-127.0, 127.0))
    y = y.clamp(-448.0, 448.0)
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20)))
    e = torch.where(torch.exp2(e) > y.abs(), e - 1, e).clamp(min=-6.0)   # (a logarithm that was rounded up)
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step


def _exact_scale(fmt, a):
    if a == 0:
        return SCALE_MIN
    if fmt == "int8":
        return float(torch.tensor(a / 127.0, dtype=torch.float64).float().clamp(SCALE_MIN, SCALE_MAX))
    e = math.ceil(math.log2(a / 448.0))
    while a <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    while a > 448.0 * 2.0 ** e:
        e += 1
    return min(max(2.0 ** e, SCALE_MIN), SCALE_MAX)


def _exact_store(st, case, name, x):
    page, fmt, heads = case["page"], case["fmt"], case["heads"]
    values = _seen_as(case, st[name][0]).float().double()
    scale = st[name + "_scale"][0].double().cpu().tolist()
    table, first, cu = st["table"].cpu().tolist(), st["first"].cpu().tolist(), st["cu"].cpu().tolist()
    x = x.double()
    tops = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1).cpu()
    jobs = []
    for i in range(case["n"]):
        t, end, pos = cu[i], cu[i + 1], first[i]
        while t < end:
            m = min(end - t, page - pos % page)
            jobs.append((t, m, table[i][pos // page], pos % page))
            t, pos = t + m, pos + m
    for t, m, p, slot in jobs:
        s = [_exact_scale(fmt, float(tops[t:t + m, h].max())) for h in range(heads)]
        was = scale[p]
        s = [max(a, b) for a, b in zip(s, was)] if slot else s
        now, old = torch.tensor(s, dtype=torch.float64, device="cuda"), torch.tensor(was, dtype=torch.float64, device="cuda")
        if slot and any(a > b for a, b in zip(s, was)):
            back = _exact_grid(fmt, values[p, :, :slot] * old[:, None, None] / now[:, None, None])
            values[p, :, :slot] = torch.where((now > old)[:, None, None], back, values[p, :, :slot])
        values[p, :, slot:slot + m] = _exact_grid(fmt, x[t:t + m] / now[None, :, None]).transpose(0, 1)
        scale[p] = s
    values = values[None]
    return (values.to(torch.int8) if fmt == "int8" else values), torch.tensor(scale, dtype=torch.float64, device="cuda")[None]


def _exact_attend(st, case):
    q, heads, G, d, page = st["q"], case["heads"], case["G"], case["d"], case["page"]
    total, H = q.shape[:2]
    out = torch.zeros((total, H, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((total, H), dtype=torch.float64, device="cuda")
    t0 = 0
    for i, (L, m) in enumerate(zip(*_sizes(case))):
        pages = st["table"][i, : -(-L // page)].long()
        kv = []
        for name in ("k", "v"):
            x = _seen_as(case, st[name][0][pages]).float().double() * st[name + "_scale"][0][pages].double()[..., None, None]
            kv.append(x.transpose(0, 1).reshape(heads, -1, d)[:, :L])
        for h in range(heads):
            rows = q[t0:t0 + m, h * G:(h + 1) * G].double().reshape(m * G, d)
            s = rows @ kv[0][h].T / math.sqrt(d)
            if case["causal"]:
                pos = (L - m + torch.arange(m, device="cuda")).repeat_interleave(G)[:, None]
                j = torch.arange(L, device="cuda")[None]
                hidden = j > pos
                if case["window"]:
                    hidden = hidden | (j <= pos - case["window"])
                s = torch.where(hidden, -math.inf, s)
            z = torch.logsumexp(s, -1, keepdim=True)
            out[t0:t0 + m, h * G:(h + 1) * G] = (torch.exp(s - z) @ kv[1][h]).reshape(m, G, d)
            lse[t0:t0 + m, h * G:(h + 1) * G] = z.reshape(m, G)
        t0 += m
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    if case["kind"] not in ("store", "attend"):
        return None   # whole numbers and copies
    st = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(st, case)
    got = {}
    for name, x in (("k", st["xk"]), ("v", st["xv"])):
        got[name], got[name + "_scale"] = _exact_store(st, case, name, x)
    return got
