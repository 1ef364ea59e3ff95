"""Chunk attention over pages of every kind on the GPU, against plain 64-bit forms.

Head layouts, head dims, page sizes, kinds and result types; sequences that take no part, segments of no
retained row, chunks of one token to many; padded tokens of NaN and unwritten rows of NaN (nothing of them may
show); rows of out and pages that the call does not own, byte for byte.
"""

import numpy as np
import pytest

from paper_2606_03075_amd import binding as bd
from tests.gpu_util import log
from tests.pages_util import KINDS, call, case, check, parts, reference, tolerance

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (2, 1, 128), (3, 1, 64), (7, 1, 128), (8, 1, 64), (16, 2, 64), (16, 1, 128), (10, 10, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("chunk", [1, 2, 5, 33])
def test_chunk_small(lib, hq, hkv, d, kind, chunk):
    """Every head layout at ragged lengths around the tiles: no retained row, one, 15 to 17, 63 to 65, 200."""
    log(f"chunk hq={hq} hkv={hkv} d={d} kind={kind} chunk={chunk}")
    n_new = [chunk, 1, max(1, chunk - 1), 0, chunk]
    c = case(hq * 100 + d + chunk, 5, 2, hq, hkv, d, chunk, kind, 16, [0, 1, 15, 17, 63, 65, 40, 40, 200, 129],
             [0, 3, 0, 1, 2], n_new, chunk + 4)
    check(c, out_bf16=bool(chunk & 1) and kind != bd.CACHE_BF16)


@pytest.mark.parametrize("page", [1, 2, 8, 16, 64, 256, 4096])
@pytest.mark.parametrize("kind", KINDS)
def test_chunk_pages(lib, page, kind):
    """Page sizes from one row to one page per segment; chunks that cross a page's end."""
    log(f"chunk page={page} kind={kind}")
    c = case(page, 2, 2, 6, 2, 128, 9, kind, page, [61, 120, 7, 255], [5, 0], [9, 8], 16)
    check(c)


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 128), (7, 1, 64), (12, 4, 128)])
@pytest.mark.parametrize("kind,out_bf16", [(bd.CACHE_BF16, False), (bd.CACHE_BF16, True), (bd.CACHE_FP8, True),
                                           (bd.CACHE_INT8, False)])
@pytest.mark.parametrize("chunk", [64, 150, 257])
def test_chunk_long(lib, hq, hkv, d, kind, out_bf16, chunk):
    """Chunks of several row tiles, their causal edge inside a key tile."""
    log(f"chunk long hq={hq} hkv={hkv} d={d} kind={kind} bf16={out_bf16} chunk={chunk}")
    c = case(chunk + d, 3, 1, hq, hkv, d, chunk, kind, 32, [70, 0, 333], [1, 0, 2], [chunk, chunk - 7, 1], chunk + 3)
    check(c, out_bf16=out_bf16)


@pytest.mark.parametrize("hq,hkv,d,chunk", [(1, 1, 128, 1), (7, 1, 128, 1), (4, 2, 64, 4), (7, 1, 128, 6)])
@pytest.mark.parametrize("kind", KINDS)
def test_chunk_few_long_segments(lib, hq, hkv, d, chunk, kind):
    """One or two long segments, where the work is split over the keys; lengths far apart."""
    log(f"chunk few hq={hq} hkv={hkv} d={d} chunk={chunk} kind={kind}")
    c = case(7 + chunk, 2, 1, hq, hkv, d, chunk, kind, 64, [6001, 37], [3, 2], None, chunk + 5)
    check(c)
    c = case(8 + chunk, 1, 1, hq, hkv, d, chunk, kind, 16, [2047], [0], None, chunk, order=False)
    check(c, out_bf16=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("chunk", [3, 40])
def test_widest_table(lib, kind, chunk):
    """4096 one-row pages, the widest table (its page ids lie in LDS beside the staged keys)."""
    log(f"chunk widest table kind={kind} chunk={chunk}")
    c = case(14, 1, 1, 4, 2, 128, chunk, kind, 1, [4096 - chunk - 2], [2], None, chunk + 2, order=False)
    assert c["table"].shape[1] == 4096
    check(c)


@pytest.mark.parametrize("chunk", [3, 70])
@pytest.mark.parametrize("size", [1e37, 1e-30])
def test_large_and_small_values(lib, chunk, size):
    """V of the largest and of small magnitudes: no product or sum leaves the range on the way."""
    from tests.pages_util import bits
    log(f"chunk values of {size}")
    c = case(15, 1, 2, 6, 2, 128, chunk, bd.CACHE_BF16, 16, [90, 7], [0], None, chunk)
    v = c["pool"].x[1].astype(np.uint32) << 16
    c["pool"].x[1] = np.where(c["pool"].x[1] == 0x7FC1, 0x7FC1, bits(v.view(np.float32) * np.float32(size))).astype(np.uint16)
    c["v_new"] = bits((c["v_new"].astype(np.uint32) << 16).view(np.float32) * np.float32(size))
    check(c)


def test_chunk_many_layers_uneven(lib):
    """Layers of very different budgets, some empty, in a given order."""
    rng = np.random.default_rng(4)
    b = np.minimum(rng.exponential(120, (3, 9)).astype(np.int32), 900)
    b[:, 4] = 0
    log("chunk uneven layers")
    check(case(5, 3, 9, 8, 2, 128, 4, bd.CACHE_FP8, 16, b, [0, 9, 4], [4, 2, 3], 16))


@pytest.mark.parametrize("kind", KINDS)
def test_sequences_that_take_no_part(lib, kind):
    """Idle, exhausted, empty and oversized counts; a table row too narrow for its segment's rows."""
    log(f"chunk no part kind={kind}")
    c = case(3, 7, 1, 4, 2, 64, 3, kind, 8, [20, 20, 20, 20, 20, 20, 0], [-1, 8, 6, 0, 0, 7, 0], [3, 1, 3, 0, 4, -2, 3], 8)
    c["table"] = np.ascontiguousarray(c["table"][:, :3])  # 24 rows: 20 retained rows and 4 more
    assert [n for _, n in parts(c)] == [0, 0, 0, 0, 0, 0, 3]
    check(c)
    c = case(4, 2, 2, 4, 2, 64, 3, kind, 8, [22, 10, 5, 21], [0, 0], None, 8)
    c["table"] = np.ascontiguousarray(c["table"][:, :3])
    assert [n for _, n in parts(c)] == [0, 3, 3, 3]
    check(c)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("chunk", [6, 70])
@pytest.mark.parametrize("where", ["k_new", "v_new", "q"])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_later_tokens_do_not_show(lib, kind, chunk, where, value):
    """A non-finite value in a token's key, value or query leaves the tokens before it as they were."""
    from tests.pages_util import bits
    at = chunk - 3
    log(f"chunk non-finite {where} {value} kind={kind} chunk={chunk}")
    c = case(6, 2, 1, 6, 2, 128, chunk, kind, 16, [50, 3], [0, 1], None, chunk + 1)
    c[where][:, :, at, :, 5] = bits(value)
    before = case(6, 2, 1, 6, 2, 128, chunk, kind, 16, [50, 3], [0, 1], None, chunk + 1)
    out, _ = call(c)
    want, mag, qk = reference(before)
    tol = tolerance(before, want, mag, qk, False)
    assert np.all(np.abs(out - want)[:, :, :at] <= tol[:, :, :at])
    if where == "q":  # nor the tokens after it
        assert np.all(np.abs(out - want)[:, :, at + 1:] <= tol[:, :, at + 1:])
        assert np.all(np.isnan(out[:, :, at]))
    elif where == "v_new" and np.isnan(value):
        g = c["hq"] // c["hkv"]
        dims = [5] if kind == bd.CACHE_BF16 else list(range(c["d"]))
        assert np.all(np.isnan(out[:, :, at:][..., dims])), g
        if kind == bd.CACHE_BF16:  # the other dims keep their values
            rest = [e for e in range(c["d"]) if e != 5]
            assert np.all((np.abs(out - want) <= tol)[:, :, at:][..., rest])
    elif where == "v_new" and kind == bd.CACHE_BF16:  # an infinity times its probability
        got = out[:, :, at:, :, 5]
        assert np.all(np.isnan(got) | (got == value)) and np.any(got == value)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("chunk", [2, 70])
@pytest.mark.parametrize("where", [0, 1])
def test_bad_retained_rows(lib, kind, chunk, where):
    """A NaN in a retained key makes every result of its segment NaN; in a retained value, that dim's, or with 8-bit
    rows every dim's.  The other segment is as it was."""
    log(f"chunk bad retained row kind={kind} chunk={chunk} where={where}")
    c = case(16, 2, 1, 6, 2, 128, chunk, kind, 16, [50, 33], [0, 1], None, chunk + 1)
    from tests.pages_util import bits
    row = bits(np.ones((2, 128)))
    row[:, 9] = 0x7FC0
    c["pool"].write(where, c["table"][0], 20, row)
    out, _ = call(c)
    dims = [9] if where == 1 and kind == bd.CACHE_BF16 else list(range(128))
    assert np.all(np.isnan(out[0][..., dims]))
    if len(dims) == 1:
        assert np.all(np.isfinite(np.delete(out[0], 9, axis=-1)))
    want, mag, qk = reference(c)
    assert np.all((np.abs(out - want) <= tolerance(c, want, mag, qk, False))[1])


@pytest.mark.parametrize("hq,hkv,d,chunk", [(4, 4, 64, 1), (8, 2, 128, 4), (7, 1, 64, 4), (2, 2, 128, 40), (3, 1, 64, 30), (4, 2, 128, 70)])
@pytest.mark.parametrize("kind,rows", [(bd.CACHE_BF16, 130), (bd.CACHE_BF16, 700), (bd.CACHE_BF16, 6001), (bd.CACHE_FP8, 500),
                                       (bd.CACHE_INT8, 500)])
def test_probabilities_of_24_bits(lib, hq, hkv, d, chunk, kind, rows):
    """32-bit results take the probabilities whole: results that are one probability each, across waves and shares, are
    off by less than a probability in two bf16 parts would be."""
    from tests.pages_util import ONE_TERM_BOUND, one_term_case, one_term_shares
    log(f"24 bits hq={hq} hkv={hkv} d={d} chunk={chunk} kind={kind} rows={rows}")
    c, at = one_term_case(rows + chunk, hq, hkv, d, chunk, kind, rows)
    out = call(c)[0][0, 0]
    want, total = one_term_shares(c, at)
    got = out.sum(-1)
    off = np.abs(out / got[..., None] / want - 1).max()
    print(f"    off by {off:.2e}")
    assert off <= ONE_TERM_BOUND
    # the sum of the probabilities: a lane adds a quarter of the rows at most, one rounding each, and the joins
    assert np.abs(got / total - 1).max() <= ONE_TERM_BOUND + ((rows + chunk) / 4 + 40) * 2.0 ** -24


# (query heads, KV heads, chunk): few query rows (16 and 32), 64-row tiles, two 128-row tiles
SHAPES = [(2, 2, 1), (2, 2, 4), (14, 2, 4), (2, 2, 40), (6, 2, 70)]


def _odd_values(c, rows, low):
    """Infinities and NaN in the values of `rows` of every segment: one sign, both signs, a NaN beside an infinity, in dims
    of their own.  low: these rows' logits lie 150 (natural units) below the others', a probability of e^-150, which is 0
    in 32 bits."""
    from tests.pages_util import bits, set_value
    q = bits(np.sqrt(c["d"]))
    if low:
        c["q"][:] = 0
        c["q"][..., 0] = q
    for i, (f, m) in enumerate(parts(c)):
        for r in range(f + m) if low else []:
            set_value(c, 0, i, r, slice(0, 1), bits(2.0))
        here = [r for r in rows(f, m) if 0 <= r < f + m]
        for x, r in enumerate(here):
            if low:
                set_value(c, 0, i, r, slice(0, 1), bits(-148.0))
            set_value(c, 1, i, r, slice(3, 4), bits(np.inf))
            set_value(c, 1, i, r, slice(40, 41), bits(-np.inf))
            set_value(c, 1, i, r, slice(17, 18), bits(-np.inf if x % 2 else np.inf))
            set_value(c, 1, i, r, slice(c["d"] - 1, c["d"]), bits(np.nan if x == 0 else np.inf))


@pytest.mark.parametrize("hq,hkv,chunk", SHAPES)
@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_infinite_new_values(lib, hq, hkv, chunk, low, out_bf16):
    """An infinity in a new token's value is the result's infinity, however small its probability: in segments of no,
    few and many retained rows (shares), for the tokens that see it and no other."""
    from tests.pages_util import check_all
    log(f"infinite new values hq={hq} hkv={hkv} chunk={chunk} low={low} bf16={out_bf16}")
    c = case(60 + chunk, 2, 2, hq, hkv, 64, chunk, bd.CACHE_BF16, 16, [0, 70, 1500, 33], [0, 2], None, chunk + 2)
    _odd_values(c, lambda f, m: [f + m // 2, f + m - 1], low)
    check_all(c, out_bf16)


@pytest.mark.parametrize("hq,hkv,chunk", SHAPES)
@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("out_bf16", [False, True])
@pytest.mark.parametrize("where", ["first", "last", "scattered"])
def test_infinite_retained_values(lib, hq, hkv, chunk, low, out_bf16, where):
    """The same in retained rows, and in retained and new ones together: in the first block and in the last one, which
    ends inside a block, in every wave's blocks and in shares."""
    from tests.pages_util import check_all
    log(f"infinite retained values hq={hq} hkv={hkv} chunk={chunk} low={low} bf16={out_bf16} {where}")
    c = case(70 + chunk, 2, 2, hq, hkv, 128, chunk, bd.CACHE_BF16, 16, [1, 75, 1500, 33], [0, 2], None, chunk + 2)
    rows = dict(first=lambda f, m: [0, 5], last=lambda f, m: [f - 1], scattered=lambda f, m: [7, 31, 32, f // 2, 700, f - 3, f + m // 2])
    _odd_values(c, rows[where], low)
    check_all(c, out_bf16)


def test_infinite_values_one_by_one(lib):
    """Tokens whose values are infinite as one chunk and one by one, by extend and by decode: the same infinities."""
    import torch
    log("infinite values one by one")
    from tests.pages_util import bits
    c = case(80, 2, 2, 2, 2, 64, 3, bd.CACHE_BF16, 16, [40, 7, 300, 0], [0, 1], None, 8)
    for t, e, x in ((0, 4, np.inf), (1, 9, -np.inf), (2, 4, np.inf), (2, 9, np.inf), (1, 33, np.nan)):
        c["v_new"][:, :, t, :, e] = bits(x)
    whole, _ = call(c)
    assert np.all(whole[..., 4] == np.inf) and np.all(whole[:, :, 1, :, 9] == -np.inf) and np.all(np.isnan(whole[:, :, 2, :, 9]))
    odd = ~np.isfinite(whole)
    extend, decode = c["pool"].device(), c["pool"].device()
    p = bd.make_problem(2, 2, 2, 2, 64, 1, 0, 0)
    ws = torch.zeros(max(1, bd.workspace_size(p, None, bd.CALL_DECODE)), dtype=torch.uint8, device="cuda")
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    b16 = lambda a: up(a.view(np.int16)).view(torch.bfloat16)  # noqa: E731
    for t in range(3):
        s = dict(c, chunk=1, steps=c["steps"] + t, **{n: np.ascontiguousarray(c[n][:, :, t:t + 1]) for n in ("q", "k_new", "v_new")})
        got, _ = call(s, pool=extend)
        out = torch.empty(2, 2, 2, 64, device="cuda")
        decode.decode(p, None, up(c["table"]), up(c["budgets"]), 8, up(s["steps"]), *(b16(s[n][:, :, 0]) for n in ("q", "k_new", "v_new")),
                      out, ws)
        torch.cuda.synchronize()
        want, here = whole[:, :, t], odd[:, :, t]
        for x in (got[:, :, 0], out.double().cpu().numpy()):
            assert np.array_equal(x[here], want[here], equal_nan=True) and np.all(np.isfinite(x[~here])), t


def test_extreme_logits(lib):
    """Logits far apart (one key takes all), equal, and so low that a key of probability 0 has a value of 1e38."""
    from tests.pages_util import bits
    log("chunk extreme logits")
    for spread in (8.0, 0.0):
        check(case(9, 2, 2, 7, 1, 128, 5, bd.CACHE_BF16, 16, [100, 3, 64, 0], [0, 1], None, 8, spread=spread))
    c = case(9, 1, 1, 4, 4, 64, 3, bd.CACHE_INT8, 16, [90], [0], None, 8)
    c["k_new"][:, :, 0], c["q"][:] = bits(-30.0), bits(30.0)
    c["v_new"][:, :, 0] = bits(1e38)
    c["k_new"][:, :, 1:] = bits(30.0)
    out, _ = call(c)
    assert np.all(np.isfinite(out[:, :, 1:])) and np.abs(out[:, :, 1:]).max() < 10


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(2, 2), (7, 1)])
def test_a_chunk_is_its_tokens_one_by_one(lib, kind, hq, hkv):
    """The same tokens in one chunk, in two, and as decode steps: the same pages byte for byte, results within
    the bound of two calls."""
    import torch
    log(f"chunk as steps kind={kind} hq={hq}")
    c = case(11, 2, 3, hq, hkv, 128, 6, kind, 16, [33, 90, 5, 64, 200, 1], [0, 2], None, 9)
    whole, pool = call(c)
    got = np.full_like(whole, np.nan)
    other = c["pool"].device()
    for t in range(6):
        s = dict(c, chunk=1, steps=c["steps"] + t, **{n: np.ascontiguousarray(c[n][:, :, t:t + 1]) for n in ("q", "k_new", "v_new")})
        got[:, :, t:t + 1], _ = call(s, pool=other)
    want, mag, qk = reference(c)
    tol = tolerance(c, want, mag, qk, False)
    assert np.all(np.abs(whole - want) <= tol) and np.all(np.abs(got - want) <= tol)
    c["pool"].check(pool)
    c["pool"].check(other)
    if kind == bd.CACHE_BF16:  # and decode's own call on the same pool
        fresh = case(11, 2, 3, hq, hkv, 128, 6, kind, 16, [33, 90, 5, 64, 200, 1], [0, 2], None, 9)
        pool = fresh["pool"].device()
        p = bd.make_problem(2, 3, hq, hkv, 128, 1, 0, 0)
        ws = torch.zeros(max(1, bd.workspace_size(p, None, bd.CALL_DECODE)), dtype=torch.uint8, device="cuda")
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        b16 = lambda a: up(a.view(np.int16)).view(torch.bfloat16)  # noqa: E731
        out = torch.empty(2, 3, hq, 128, device="cuda")
        for t in range(6):
            pool.decode(p, None, up(c["table"]), up(c["budgets"]), 9, up(c["steps"] + t), b16(c["q"][:, :, t]),
                        b16(c["k_new"][:, :, t]), b16(c["v_new"][:, :, t]), out, ws)
            assert np.all(np.abs(out.double().cpu().numpy() - want[:, :, t]) <= tol[:, :, t])
        c["pool"].check(pool)


@pytest.mark.parametrize("kind", [bd.CACHE_BF16, bd.CACHE_INT8])
def test_offsets_beyond_32_bits(lib, kind):
    """Pages at the far end of a pool of more than 2^32 bytes."""
    import torch
    hkv, d, page = 8, 128, 128
    n_pages = (1 << 32) // (hkv * d * page * (2 if kind == bd.CACHE_BF16 else 1)) + 64
    log(f"chunk far pages kind={kind} n_pages={n_pages}")
    c = case(12, 2, 1, 16, hkv, d, 5, kind, page, [200, 90], [0, 3], [5, 4], 16)
    small = c["pool"].device()
    big = bd.PagedPool(hkv, d, page, n_pages, kind=kind)
    n = small.n_pages
    for name in ("k_pool", "v_pool", "k_exp", "v_exp"):
        t = getattr(small, name)
        if t is not None:
            as_bytes = lambda x: x.view(torch.int16) if kind == bd.CACHE_BF16 else x.view(torch.uint8)  # noqa: E731
            as_bytes(getattr(big, name))[-n:] = as_bytes(t)
    moved = dict(c, table=np.where(c["table"] >= 0, c["table"] + n_pages - n, -1).astype(np.int32))
    out, _ = call(moved, pool=big)
    want, mag, qk = reference(c)
    there = ~np.isnan(want)
    assert np.all(np.abs(out - want)[there] <= tolerance(c, want, mag, qk, False)[there])
    for name in ("k_pool", "v_pool", "k_exp", "v_exp"):
        if getattr(big, name) is not None:
            setattr(big, name, getattr(big, name)[-n:])
    c["pool"].check(big)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_without_a_page_are_not_written(lib, kind):
    """Table entries outside the pool: nothing is written for their rows, and no page is disturbed."""
    log(f"chunk rows without a page kind={kind}")
    c = case(13, 1, 1, 4, 2, 64, 4, kind, 8, [7], [0], None, 16)
    c["table"][0, 1] = -1  # rows 8 .. 15
    out, pool = call(c)
    for w, name in ((0, "k_new"), (1, "v_new")):
        c["pool"].write(w, c["table"][0], 7, c[name][0, 0, 0])
    c["pool"].check(pool)


@pytest.mark.parametrize("hq,hkv,chunk,kind", [(4, 4, 3, bd.CACHE_FP8), (7, 1, 1, bd.CACHE_INT8), (7, 1, 4, bd.CACHE_BF16),
                                               (4, 2, 80, bd.CACHE_BF16)])
def test_graph_replays(lib, hq, hkv, chunk, kind):
    """Two calls of different lengths on one workspace in one graph, replayed with eager calls of both between."""
    import torch
    log(f"chunk graph hq={hq} hkv={hkv} chunk={chunk} kind={kind}")
    cases = [case(20, 1, 2, hq, hkv, 128, chunk, kind, 16, [3000, 411], [2], None, chunk + 2),
             case(21, 2, 3, hq, hkv, 128, chunk, kind, 16, [40, 900, 0, 1500, 7, 77], [0, 1], None, chunk + 1)]
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    b16 = lambda a: up(a.view(np.int16)).view(torch.bfloat16)  # noqa: E731
    probs = [bd.make_problem(c["B"], c["L"], hq, hkv, 128, 1, 0, 0) for c in cases]
    ws = torch.full((max(1, *(bd.chunk_workspace_size(p, None, chunk) for p in probs)),), 255, dtype=torch.uint8, device="cuda")
    calls = [(c["pool"].device(), p, (up(c["table"]), up(c["budgets"]), c["reserve"], up(c["steps"]), None, b16(c["q"]),
                                      b16(c["k_new"]), b16(c["v_new"]), torch.empty(c["q"].shape, device="cuda"), ws))
             for c, p in zip(cases, probs)]

    def step(x):
        x[0].extend(x[1], None, *x[2])
    want = []
    for x in calls:
        ws.fill_(255)
        step(x)
        want.append(x[2][8].clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x in calls + calls[:1]:
            step(x)
    for rep in range(4):
        for x in calls:
            x[2][8].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x[2][8], w) for x, w in zip(calls, want)), rep
        x = calls[rep % 2]
        x[2][8].fill_(float("nan"))
        step(x)
        torch.cuda.synchronize()
        assert torch.equal(x[2][8], want[rep % 2]), rep


@pytest.mark.parametrize("hq,hkv,chunk,kind", [(7, 1, 3, bd.CACHE_FP8), (4, 2, 40, bd.CACHE_INT8), (16, 2, 40, bd.CACHE_BF16)])
def test_a_serving_graph(lib, hq, hkv, chunk, kind):
    """One captured call whose steps and n_new change between replays, as a loop around it does: sequences pause and
    come back, so long segments are cut into shares in one replay and take no part in the next."""
    import torch
    log(f"chunk serving graph hq={hq} hkv={hkv} chunk={chunk} kind={kind}")
    c = case(25, 2, 2, hq, hkv, 128, chunk, kind, 16, [3000, 411, 2200, 5], [3 * chunk, 3 * chunk], None, 4 * chunk)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    b16 = lambda a: up(a.view(np.int16)).view(torch.bfloat16)  # noqa: E731
    p = bd.make_problem(2, 2, hq, hkv, 128, 1, 0, 0)
    size = bd.chunk_workspace_size(p, None, chunk)
    pool, steps = c["pool"].device(), torch.zeros(2, dtype=torch.int32, device="cuda")
    n_new, out = torch.full_like(steps, chunk), torch.empty(c["q"].shape, device="cuda")
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    args = (up(c["table"]), up(c["budgets"]), c["reserve"], steps, n_new, b16(c["q"]), b16(c["k_new"]), b16(c["v_new"]), out)
    pool.extend(p, None, *args, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pool.extend(p, None, *args, ws)
    for st, n in [((0, 0), (chunk, chunk)), ((chunk, chunk), (2, 0)), ((chunk + 2, chunk), (0, 3)),
                  ((chunk + 2, -1), (1, 3)), ((chunk + 3, chunk + 3), (chunk, chunk)), ((3 * chunk, 0), (chunk, 0))]:
        steps.copy_(torch.tensor(st, dtype=torch.int32))
        n_new.copy_(torch.tensor(n, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(float("nan"))
        pool.extend(p, None, *args, torch.full((size,), 255, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int32), out.view(torch.int32)), (st, n)
        for b in range(2):
            here = 0 if st[b] < 0 else n[b]
            assert not got[b, :, :here].isnan().any() and got[b, :, here:].isnan().all(), (st, n)


@pytest.mark.parametrize("kind", [bd.CACHE_BF16, bd.CACHE_INT8])
def test_a_loop_keeps_one_workspace(lib, kind):
    """A workspace made for the largest chunk, whose own calls need none (2560 items), and exactly as large as it is said
    to be: single tokens, drafts and questions of every tile size on it."""
    import torch
    log(f"chunk one workspace kind={kind}")
    B, L, hq, hkv, d = 8, 16, 8, 4, 64
    p = bd.make_problem(B, L, hq, hkv, d, 1, 0, 0)
    size = bd.chunk_workspace_size(p, None, 320)
    assert size >= 896 * 128 * (d + 2) * 4
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    budgets = np.random.default_rng(3).integers(0, 3, (B, L)).astype(np.int32)
    budgets[1, 3], budgets[6, 15] = 700, 300
    for chunk, n_new in ((1, None), (320, [1, 3, 0, 0, 0, 0, 17, 0]), (8, [1, 8, 0, 0, 0, 2, 5, 0]), (12, [0, 12, 0, 0, 0, 0, 9, 1]),
                         (32, [0, 32, 0, 0, 0, 0, 4, 0]), (40, [0, 7, 1, 0, 0, 0, 33, 0]), (1, None)):
        log(f"  chunk={chunk}")
        check(case(50 + chunk, B, L, hq, hkv, d, chunk, kind, 16, budgets, np.arange(B) % 3, n_new, chunk + 4), ws=ws)


def test_the_most_segments(lib):
    """One less sequence than would make 2^24 workgroups: the first and the last are served, idle ones are left alone; a read
    of twice as many segments, by one wave each."""
    import torch
    log("chunk the most segments")
    B, L, d = (1 << 15) - 1, 512, 64
    p, n = bd.make_problem(B, L, 1, 1, d, 1, 0, 0), B * L
    full = lambda v, *s, t=torch.int32: torch.full(s, v, dtype=t, device="cuda")  # noqa: E731
    pool = bd.PagedPool(1, d, 8, 4)
    table, steps = full(0, n, 1), full(-1, B)
    steps[0], steps[-1], table[:L], table[-L:] = 0, 0, 2, 3
    new, out = full(1.0, B, L, 1, 1, d, t=torch.bfloat16), full(7.0, B, L, 1, 1, d, t=torch.float32)
    ws = full(0, max(16, bd.chunk_workspace_size(p, None, 1)), t=torch.uint8)
    pool.extend(p, None, table, full(0, n), 4, steps, None, new, new, new, out, ws)
    torch.cuda.synchronize()
    assert torch.all(out[0] == 1) and torch.all(out[-1] == 1) and torch.all(out[1:-1] == 7)
    del new, out
    p, m = bd.make_problem(B, L, 2, 2, d, 1, 0, 0), 2 * n
    pool = bd.PagedPool(2, d, 8, 4)
    pool.k_pool.fill_(3.0)
    pool.v_pool.fill_(-3.0)
    k, v = full(0.0, m * d, t=torch.bfloat16), full(0.0, m * d, t=torch.bfloat16)
    pool.read(p, None, table, full(1, n), torch.arange(n + 1, dtype=torch.int64, device="cuda"), k, v)
    torch.cuda.synchronize()
    assert torch.all(k == 3) and torch.all(v == -3)


def test_other_streams(lib):
    """Two calls at once, each on a stream of its own with a workspace of its own, and the stream argument."""
    import torch
    log("chunk on two streams")
    cs = [case(30 + i, 2, 2, 7, 1, 128, 3, bd.CACHE_FP8, 16, [1500, 20, 300, 900], [0, 1], None, 8) for i in range(2)]
    refs = []
    for c in cs:
        pool = c["pool"].device()
        refs.append((pool, *reference(c)))
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    b16 = lambda a: up(a.view(np.int16)).view(torch.bfloat16)  # noqa: E731
    p = bd.make_problem(2, 2, 7, 1, 128, 1, 0, 0)
    args = [(up(c["table"]), up(c["budgets"]), 8, up(c["steps"]), None, b16(c["q"]), b16(c["k_new"]), b16(c["v_new"]),
             torch.empty(c["q"].shape, device="cuda"),
             torch.empty(max(1, bd.chunk_workspace_size(p, None, 3)), dtype=torch.uint8, device="cuda")) for c in cs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(streams[0]):
            refs[0][0].extend(p, None, *args[0])
        refs[1][0].extend(p, None, *args[1], stream=streams[1])
    torch.cuda.synchronize()
    for c, a, (pool, want, mag, qk) in zip(cs, args, refs):
        assert np.all(np.abs(a[8].double().cpu().numpy() - want) <= tolerance(c, want, mag, qk, False))
        c["pool"].check(pool)


@pytest.mark.parametrize("kind", KINDS)
def test_repeated_calls_give_the_same_bits(lib, kind):
    import torch
    log(f"chunk repeat kind={kind}")
    c = case(40, 2, 2, 7, 1, 128, 5, kind, 16, [2500, 90, 700, 3], [0, 1], None, 8)
    first, _ = call(c)
    for _ in range(3):
        assert np.array_equal(call(c)[0], first)
    torch.cuda.synchronize()
