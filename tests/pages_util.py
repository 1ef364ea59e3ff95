"""Paged pools of every kind, and plain 64-bit forms of what the library does with them.

The forms here are written from the definitions in include/tgvkv.h, on the CPU with NumPy, and share no code
with the library: the quantiser works on exact float64 values and a table of the kind's grid.
"""

from __future__ import annotations

import numpy as np

from paper_2606_03075_amd import binding as bd
from workloads import bf16_bits_to_f32

MOST = {bd.CACHE_FP8: 448.0, bd.CACHE_INT8: 127.0}
KINDS = [bd.CACHE_BF16, bd.CACHE_FP8, bd.CACHE_INT8]


def bits(x):
    """float -> bf16 bits, round to nearest even."""
    from workloads import f32_to_bf16_bits
    return f32_to_bf16_bits(np.asarray(x, np.float32))


def e4m3_values():
    """The value of every e4m3 code (NaN for 0x7F and 0xFF)."""
    out = np.zeros(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = (-1) ** s * x
        if e == 15 and m == 7:
            out[c] = np.nan
    return out


E4M3 = e4m3_values()


def quantise(b, kind):
    """bf16 bits [..., D] -> (codes uint8 [..., D], exponent bytes uint8 [...]) by definition."""
    x = bf16_bits_to_f32(b).astype(np.float64)
    finite = np.isfinite(x).all(-1)
    x = np.where(finite[..., None], x, 0.0)
    amax = np.abs(x).max(-1)
    e = np.full(amax.shape, -100)
    for t in range(-100, 129):  # the least e with amax <= M 2^e
        e = np.where(amax > MOST[kind] * 2.0 ** t, t + 1, e)
    y = x / 2.0 ** e[..., None]
    if kind == bd.CACHE_INT8:
        codes = np.rint(y).astype(np.int8).view(np.uint8)
    else:
        grid = E4M3[:0x7F]  # ascending from 0 to 448; a tie takes the even mantissa
        a = np.abs(y)
        hi = np.searchsorted(grid, a)  # first grid value >= a
        lo = np.maximum(hi - 1, 0)
        down, up = a - grid[lo], grid[np.minimum(hi, 0x7E)] - a
        pick = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
        codes = (pick | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)
    return np.where(finite[..., None], codes, 0).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def values(codes, exp, kind):
    """What codes and exponent bytes stand for, float64; the byte 255 is NaN."""
    c = E4M3[codes] if kind == bd.CACHE_FP8 else codes.view(np.int8).astype(np.float64)
    return np.where(exp[..., None] == 255, np.nan, c * 2.0 ** (exp.astype(np.float64)[..., None] - 127))


def held(b, kind):
    """The values that rows of bf16 bits are held as."""
    return bf16_bits_to_f32(b).astype(np.float64) if kind == bd.CACHE_BF16 else values(*quantise(b, kind), kind)


class Pool:
    """A pool on the host: codes (or bf16 bits) and exponent bytes, every unwritten row a NaN of its kind."""

    def __init__(self, n_pages, hkv, page, d, kind):
        self.kind, self.page = kind, page
        self.x, self.e = [], []
        for _ in range(2):
            if kind == bd.CACHE_BF16:
                self.x.append(np.full((n_pages, hkv, page, d), 0x7FC1, np.uint16))
                self.e.append(None)
            else:
                self.x.append(np.full((n_pages, hkv, page, d), 0x7F, np.uint8))
                self.e.append(np.full((n_pages, hkv, page), 255, np.uint8))

    def write(self, which, table_row, n, b):
        """Row n of a segment, b [hkv][D] bf16 bits."""
        p, r = table_row[n // self.page], n % self.page
        if self.kind == bd.CACHE_BF16:
            self.x[which][p, :, r] = b
        else:
            self.x[which][p, :, r], self.e[which][p, :, r] = quantise(b, self.kind)

    def rows(self, which, table_row, n0, n1):
        """Values [hkv][n1 - n0][D] of a segment's rows."""
        n = np.arange(n0, n1)
        p, r = np.asarray(table_row)[n // self.page], n % self.page
        x = self.x[which][p, :, r].swapaxes(0, 1)
        if self.kind == bd.CACHE_BF16:
            return bf16_bits_to_f32(x).astype(np.float64)
        return values(x, self.e[which][p, :, r].swapaxes(0, 1), self.kind)

    def device(self):
        """The same pool as a PagedPool on the GPU."""
        import torch
        n, hkv, page, d = self.x[0].shape
        pool = bd.PagedPool(hkv, d, page, 1, kind=self.kind)
        up = lambda a, t: None if a is None else torch.from_numpy(a.copy()).cuda().view(t)  # noqa: E731
        kinds = (torch.bfloat16, torch.float8_e4m3fn, torch.int8)
        x = [a.view(np.int16) if self.kind == bd.CACHE_BF16 else a.view(np.int8) for a in self.x]
        pool.attach(up(x[0], kinds[self.kind]), up(x[1], kinds[self.kind]), up(self.e[0], torch.uint8),
                    up(self.e[1], torch.uint8))
        return pool

    def check(self, pool):
        """Every byte of the device pool equals this one's."""
        import torch
        for name, x, e in (("k", self.x[0], self.e[0]), ("v", self.x[1], self.e[1])):
            t = getattr(pool, name + "_pool")
            got = t.view(torch.int16 if self.kind == bd.CACHE_BF16 else torch.uint8).cpu().numpy().view(x.dtype)
            if self.kind == bd.CACHE_FP8:  # +0 and -0 alike
                got, x = np.where(got == 0x80, 0, got), np.where(x == 0x80, 0, x)
            assert np.array_equal(got, x), f"{name}_pool: {np.count_nonzero(got != x)} of {x.size} differ"
            if e is not None:
                assert np.array_equal(getattr(pool, name + "_exp").cpu().numpy(), e), f"{name}_exp"


def parts(c):
    """(first row, new tokens) of every (sequence, layer); (0, 0) where it takes no part."""
    out = []
    for b in range(c["B"]):
        st, n = int(c["steps"][b]), c["chunk"] if c["n_new"] is None else int(c["n_new"][b])
        for l in range(c["L"]):
            f = int(c["budgets"][b, l]) + st
            ok = st >= 0 and 1 <= n <= c["chunk"] and st + n <= c["reserve"] and f + n <= c["table"].shape[1] * c["page"]
            out.append((f, n) if ok else (0, 0))
    return out


def case(seed, B, L, hq, hkv, d, chunk, kind, page, budgets, steps, n_new, reserve, spread=1.0, order=True):
    """One call's inputs: a pool with the segments' rows in scattered pages, new tokens, padded rows of NaN."""
    rng = np.random.default_rng(seed)
    budgets = np.asarray(budgets, np.int32).reshape(B, L)
    steps = np.asarray(steps, np.int32)
    n_new = None if n_new is None else np.asarray(n_new, np.int32)
    need = -(-(budgets.reshape(-1).astype(np.int64) + reserve) // page)
    n_pages = int(need.sum()) + 4
    table = np.full((B * L, max(1, int(need.max()))), -1, np.int32)
    ids, at = rng.permutation(n_pages).astype(np.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = ids[at:at + n]
        at += n
    c = dict(B=B, L=L, hq=hq, hkv=hkv, d=d, chunk=chunk, kind=kind, page=page, budgets=budgets, steps=steps, n_new=n_new,
             reserve=reserve, table=table)
    pool = Pool(n_pages, hkv, page, d, kind)
    for i, (f, n) in enumerate(parts(c)):
        rows = f if n else min(int(budgets.reshape(-1)[i]), 2)
        b = bits(spread * rng.standard_normal((2, rows, hkv, d)))
        b[0, :1] = bits(4 * bf16_bits_to_f32(b[0, :1]))  # an attention sink
        for w in range(2):
            for r in range(rows):
                pool.write(w, table[i], r, b[w, r])
    c["pool"] = pool
    c["q"] = bits(spread * rng.standard_normal((B, L, chunk, hq, d)))
    c["k_new"], c["v_new"] = (bits(spread * rng.standard_normal((B, L, chunk, hkv, d))) for _ in range(2))
    for i, (f, n) in enumerate(parts(c)):
        for name in ("q", "k_new", "v_new"):
            c[name].reshape(B * L, chunk, -1)[i, n:] = 0x7FC1  # a token that is not there
    c["order"] = rng.permutation(B * L).astype(np.int32) if order else None
    return c


def reference(c):
    """The call in 64 bits: (out [B, L, chunk, hq, d], sums of p |v| alike, largest sum |q k| per output row);
    the host pool gets the appended rows.  Rows that the call does not write are NaN."""
    B, L, hq, hkv, d, g = c["B"], c["L"], c["hq"], c["hkv"], c["d"], c["hq"] // c["hkv"]
    out = np.full((B * L, c["chunk"], hq, d), np.nan)
    mag, qk = np.full_like(out, np.nan), np.zeros((B * L, c["chunk"], hq, 1))
    for i, (f, n) in enumerate(parts(c)):
        if n == 0:
            continue
        for r in range(n):
            for w, name in ((0, "k_new"), (1, "v_new")):
                c["pool"].write(w, c["table"][i], f + r, c[name].reshape(B * L, c["chunk"], hkv, d)[i, r])
        k, v = (c["pool"].rows(w, c["table"][i], 0, f + n) for w in range(2))
        q = bf16_bits_to_f32(c["q"].reshape(B * L, c["chunk"], hq, d)[i, :n]).astype(np.float64)
        for h in range(hq):
            for t in range(n):  # only the visible rows enter, whatever the others hold
                kk, vv, m = k[h // g, :f + t + 1], v[h // g, :f + t + 1], q[t, h]
                z = kk @ m / np.sqrt(d)
                p = np.exp(z - z.max())
                p = p / p.sum()
                out[i, t, h], mag[i, t, h] = p @ vv, p @ np.abs(vv)
                qk[i, t, h] = (np.abs(kk) @ np.abs(m)).max()
    shape = (B, L, c["chunk"], hq)
    return out.reshape(*shape, d), mag.reshape(*shape, d), qk.reshape(*shape, 1)


def tolerance(c, out, mag, qk, out_bf16):
    """How far a result may be off, element by element.

    A logit is d products summed in 32 bits: (d + 2) 2^-24 sum|q k| / sqrt(d), which changes a probability by
    that share, and its normaliser by as much again.  exp2 and the sums over n rows add (n + 8) 2^-23.  With
    32-bit results the probabilities enter the product with V as bf16 parts, two in decode's own call (16 significant
    bits: 2^-16), three here.  With bf16 results they
    are one bf16, off by 2^-8 at most, and the result is rounded once more, by 2^-8 of itself at most.
    """
    n = max(f + m for f, m in parts(c))
    share = 2 * (c["d"] + 2) * 2.0 ** -24 * qk / np.sqrt(c["d"]) + (n + 8) * 2.0 ** -23
    if out_bf16:
        return (share + 2.0 ** -8) * mag + 2.0 ** -8 * (np.abs(out) + (share + 2.0 ** -8) * mag)
    return (share + 2.0 ** -16) * mag


def call(c, out_bf16=False, pool=None, out=None, ws=None, stream=None, problem=None):
    """The library's call on the case; (out as float64, pool)."""
    import torch
    up = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    b16 = lambda a: up(a.view(np.int16)).view(torch.bfloat16)  # noqa: E731
    p = problem or bd.make_problem(c["B"], c["L"], c["hq"], c["hkv"], c["d"], 1, 0, 0)
    pool = c["pool"].device() if pool is None else pool
    if out is None:
        out = torch.full(c["q"].shape, float("nan"), dtype=torch.bfloat16 if out_bf16 else torch.float32, device="cuda")
    if ws is None:
        ws = torch.full((max(1, bd.chunk_workspace_size(p, None, c["chunk"])),), 255, dtype=torch.uint8, device="cuda")
    args = (up(c["table"]), up(c["budgets"]), c["reserve"], up(c["steps"]), up(c["n_new"]), b16(c["q"]), b16(c["k_new"]),
            b16(c["v_new"]), out, ws)
    torch.cuda.synchronize()
    pool.extend(p, None, *args, stream=stream, unit_order=up(c["order"]))
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), pool


def check(c, out_bf16=False, **kw):
    """One call against the 64-bit form: results, rows left alone, and every byte of the pool."""
    out, pool = call(c, out_bf16, **kw)  # the device pool is made before the host's gets the new rows
    want, mag, qk = reference(c)
    there = ~np.isnan(want)
    assert np.all(np.isnan(out[~there])), "rows that the call does not own were written"
    err, tol = np.abs(out - want)[there], tolerance(c, want, mag, qk, out_bf16)[there]
    assert np.all(err <= tol), f"{np.count_nonzero(~(err <= tol))} of {err.size} off; worst {np.nanmax(err / tol):.2f} of the bound"
    c["pool"].check(pool)
    return out, pool


def set_value(c, which, i, n, dims, b):
    """Elements `dims` of row n of segment i, every KV head, in a bf16 pool or, for a new token's row, its input."""
    f, m = parts(c)[i]
    if n < f:
        c["pool"].x[which][c["table"][i][n // c["page"]], :, n % c["page"], dims] = b
    else:
        c[("k_new", "v_new")[which]].reshape(c["B"] * c["L"], c["chunk"], c["hkv"], c["d"])[i, n - f, :, dims] = b


def check_all(c, out_bf16=False, **kw):
    """check() where results may be infinities and NaN: these have to be where the 64-bit form has them."""
    out, pool = call(c, out_bf16, **kw)
    with np.errstate(invalid="ignore"):
        want, mag, qk = reference(c)
        rows = np.zeros((c["B"] * c["L"], c["chunk"]), bool)  # the rows that the call writes
        for i, (f, n) in enumerate(parts(c)):
            rows[i, :n] = True
        rows = rows.reshape(c["B"], c["L"], c["chunk"])
        got, want, mag, qk = (x[rows] for x in (out, want, mag, qk))
        odd = ~np.isfinite(want)
        assert np.array_equal(got[odd], want[odd], equal_nan=True), \
            f"{np.count_nonzero(~((got == want) | (np.isnan(got) & np.isnan(want)))[odd])} of {odd.sum()} non-finite results differ"
        # a finite result of a row with non-finite ones: its own dim's magnitudes
        err, tol = np.abs(got - want)[~odd], np.broadcast_to(tolerance(c, want, mag, qk, out_bf16), got.shape)[~odd]
        assert np.all(err <= tol), f"{np.count_nonzero(~(err <= tol))} of {err.size} finite results off"
    c["pool"].check(pool)


# How far the products with V may change a probability.  In the inputs of one_term_case() a logit is one product (its sum
# exact), a result one probability over the common sum, and the results' shares of their total free of that sum's errors.
# A share is off by twice the following, relative to itself, with probabilities of all their 24 bits:
#   2^-21 ln 2   the exponent, in [8, 16) below the reference: one rounding of an fma
#   3 2^-24      the logit's scale: sm_scale, log2 e and their product rounded, times at most 1.5 (base 2) and ln 2
#   3 2^-23      exp2 of the exponent and of the factors that join waves and shares, one unit in the last place each
#   3 2^-24      the two joins' products and the division or the product with the reciprocal
# A probability in two bf16 parts is off by up to 2^-18 of itself.
ONE_TERM_BOUND = 2 * (2.0 ** -21 * np.log(2) + (3 * 1.5 * np.log(2) + 3 * 2 + 3) * 2.0 ** -24)


def one_term_case(seed, hq, hkv, d, chunk, kind, rows, page=16):
    """One segment of `rows` retained rows and `chunk` new ones, in which every key and query is one value in dim 0, and
    every dim of V one 1 in a row of its own; (case, the dims' rows)."""
    rng = np.random.default_rng(seed)
    c = case(seed, 1, 1, hq, hkv, d, chunk, kind, page, [0], [rows], None, rows + chunk, order=False)
    at = rng.choice(rows, d, replace=False)
    x = np.zeros((2, rows + chunk, hkv, d), np.float32)
    x[0, ..., 0] = rng.uniform(0, 8, (rows + chunk, hkv))
    x[1, at, :, np.arange(d)] = 1.0
    for w in range(2):
        for n in range(rows):
            c["pool"].write(w, c["table"][0], n, bits(x[w, n]))
        c[("k_new", "v_new")[w]][0, 0] = bits(x[w, rows:])
    c["q"][:] = 0
    c["q"][..., 0] = bits(1.0)
    return c, at


def one_term_shares(c, at):
    """(results' shares of their total, the total), [chunk, hq, d] and [chunk, hq], in 64 bits; to be called after the call."""
    reference_pool, (f, m) = c["pool"], parts(c)[0]
    for r in range(m):
        reference_pool.write(0, c["table"][0], f + r, c["k_new"][0, 0, r])
    z = reference_pool.rows(0, c["table"][0], 0, f + m)[..., 0] / np.sqrt(c["d"])  # [hkv][rows]
    p = np.exp(z)[np.arange(c["hq"]) // (c["hq"] // c["hkv"])]  # [hq][rows]
    sums = np.cumsum(p, 1)[:, f:].T  # over the rows that token i sees
    mine = p[:, at]
    total = mine.sum(1)
    return np.broadcast_to(mine / total[:, None], (m, *mine.shape)), total[None] / sums
