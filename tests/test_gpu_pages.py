"""The paged cache in 8 bits on the GPU: rows quantised as they are written, and read back.

Codes and exponent bytes equal a plain quantiser's (float64, a table of the grid) bit for bit; what is read
back is exactly what they stand for; a serving loop over 8-bit pages from eviction to decode.
"""

import numpy as np
import pytest

from paper_2606_03075_amd import binding as bd
from tests.gpu_util import bf16_host_bits, dev_bf16, host, log
from tests.pages_util import KINDS, Pool, bits, check, held, quantise, values
from workloads import bf16_bits_to_f32, make_prefill_tensors, total_budget
from workloads.configs import custom_config

pytestmark = pytest.mark.gpu
Q8 = [bd.CACHE_FP8, bd.CACHE_INT8]


def _up(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _store_rows(rows, kind, page=16):
    """Rows [n][D] of bf16 bits through tgvkv_compact_pages, one KV head: (codes, exponent bytes), host."""
    import torch
    n, d = rows.shape
    k = dev_bf16(rows.reshape(1, 1, 1, n, d))
    pool = bd.PagedPool(1, d, page, -(-n // page), kind=kind)
    p = bd.make_problem(1, 1, 1, 1, d, 0, n, 0)
    pool.store(p, None, k, k, _up(np.arange(n, dtype=np.int32)), _up(np.array([[n]], np.int32)), _up(np.array([0, n])), n,
               _up(np.arange(-(-n // page), dtype=np.int32)[None]))
    torch.cuda.synchronize()
    codes = [t.view(torch.uint8).cpu().numpy().reshape(-1, d)[:n] for t in (pool.k_pool, pool.v_pool)]
    exps = [t.cpu().numpy().reshape(-1)[:n] for t in (pool.k_exp, pool.v_exp)]
    assert np.array_equal(codes[0], codes[1]) and np.array_equal(exps[0], exps[1])
    return codes[0], exps[0]


def _special_rows(d):
    """Rows at the quantiser's borders."""
    rng = np.random.default_rng(0)
    rows = [np.zeros(d), np.full(d, 3.3e38), np.full(d, 1e-38), np.full(d, 9e-41)]
    for m in (1.0, 1.5, 1.7421875, 1.75, 1.7578125, 1.984375, 1.9921875):  # where the exponent steps up
        for s in (-120, -93, -60, 0, 7, 100, 126):
            r = rng.uniform(-1, 1, d) * m * 2.0 ** s
            r[rng.integers(d)] = (-1) ** (s & 1) * m * 2.0 ** s
            rows.append(r)
    for m in (1.0, 1.25, 1.5, 1.75):  # ties: every multiple of a half, a quarter ... of the grid's steps
        r = (np.arange(d) - d / 2) / 64 * m
        rows.append(r)
        rows.append(2.0 ** -rng.integers(0, 22, d) * m)
        rows.append((2.0 ** -rng.integers(0, 22, d) + 2.0 ** -rng.integers(3, 26, d)) * m)
    b = bits(np.stack(rows))
    bad = bits(rng.standard_normal((4, d)))
    bad[0, 3], bad[1, d - 1], bad[2, 0], bad[3, 7] = 0x7F80, 0xFF80, 0x7FC0, 0xFFFF  # inf, -inf, NaN, NaN
    return np.concatenate([b, bad, bits(rng.standard_normal((200, d)) * np.exp(3 * rng.standard_normal((200, 1))))])


@pytest.mark.parametrize("kind", Q8)
@pytest.mark.parametrize("d", [64, 128])
def test_quantiser_bits(lib, kind, d):
    log(f"quantise kind={kind} d={d}")
    rows = _special_rows(d)
    codes, exps = _store_rows(rows, kind)
    want, wexp = quantise(rows, kind)
    assert np.array_equal(exps, wexp)
    if kind == bd.CACHE_FP8:
        codes, want = np.where(codes == 0x80, 0, codes), np.where(want == 0x80, 0, want)
    assert np.array_equal(codes, want)


@pytest.mark.parametrize("kind", Q8)
def test_rounding_is_within_its_bound(lib, kind):
    """Per value: e4m3 2^-4 of it, at least 2^(e-10); whole numbers 2^(e-1)."""
    rows = bits(np.random.default_rng(1).standard_normal((300, 128)) * 2.0 ** np.random.default_rng(2).integers(-40, 40, (300, 1)))
    x = bf16_bits_to_f32(rows).astype(np.float64)
    codes, exps = _store_rows(rows, kind)
    unit = 2.0 ** (exps.astype(np.float64) - 127)[:, None]
    bound = np.maximum(2.0 ** -4 * np.abs(x), unit * 2.0 ** -10) if kind == bd.CACHE_FP8 else np.broadcast_to(unit / 2, x.shape)
    assert np.all(np.abs(values(codes, exps, kind) - x) <= bound)


def _retained(kind, page, heads, cfg_kw, rho, head_mode=0, seed=0, vision_only=False, reserve=3):
    import torch
    hq, hkv, d = heads
    cfg = custom_config(name="q8", heads_q=hq, heads_kv=hkv, head_dim=d, **cfg_kw)
    t = make_prefill_tensors(cfg, seed=seed)
    k, v = dev_bf16(t["k"]), dev_bf16(t["v"])
    p, o = bd.problem_from(cfg), bd.make_opts(head_mode=head_mode, vision_only=vision_only)
    tot = total_budget(rho, cfg.n_vis if vision_only else cfg.n_tokens, cfg.layers)
    buf = bd.EvictionBuffers(p, o, tot, reserve)
    buf.evict(dev_bf16(t["q_text"]), k, v)
    _, bound = bd.page_plan(p, o, tot, reserve, page)
    pool = bd.PagedPool(hkv, d, page, bound + 3, kind=kind)
    ref = Pool(bound + 3, hkv, page, d, kind)
    for name, x, e in (("k", ref.x[0], ref.e[0]), ("v", ref.x[1], ref.e[1])):
        getattr(pool, name + "_pool").view(torch.uint8).copy_(_up(x.view(np.uint8)))
        if e is not None:
            getattr(pool, name + "_exp").copy_(_up(e))
    pool.free = [int(i) for i in np.random.default_rng(seed).permutation(bound + 3)]
    table = pool.admit(buf, k, v)
    torch.cuda.synchronize()
    bud, idx, io, tab = host(buf.budgets), host(buf.idx), host(buf.idx_offsets), host(table)
    for bl in range(cfg.batch * cfg.layers):
        b, l, n = bl // cfg.layers, bl % cfg.layers, int(bud.reshape(-1)[bl])
        sel = [idx[io[bl] + (h * n if head_mode else 0):][:n] for h in range(hkv)]
        for w, x in enumerate((t["k"], t["v"])):
            rows = np.stack([x[b, l, h][sel[h]] for h in range(hkv)], 1)
            for r in range(n):
                ref.write(w, tab[bl], r, rows[r])
    return cfg, t, buf, pool, table, ref


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page,heads,kw", [
    (16, (8, 4, 128), dict(batch=2, layers=4, n_sys=6, n_vis=230, n_qst=21)),
    (1, (2, 1, 64), dict(batch=1, layers=2, n_sys=3, n_vis=70, n_qst=9)),
    (64, (16, 2, 64), dict(batch=2, layers=3, n_sys=4, n_vis=300, n_qst=19)),
    (4096, (4, 4, 128), dict(batch=1, layers=1, n_sys=8, n_vis=144, n_qst=16))])
@pytest.mark.parametrize("rho,head_mode,vision_only", [(0.0, 0, False), (0.2, 0, False), (0.3, 1, False), (0.1, 0, True), (1.0, 1, False)])
def test_admit_and_read(lib, kind, page, heads, kw, rho, head_mode, vision_only):
    """An evicted batch into a pool of every kind: every byte of the pool (pages of others untouched), and the
    rows read back in the contiguous cache's layout with its free slots left alone."""
    import torch
    log(f"admit kind={kind} page={page} {heads} rho={rho} head_mode={head_mode} vision_only={vision_only}")
    cfg, t, buf, pool, table, ref = _retained(kind, page, heads, kw, rho, head_mode, vision_only=vision_only)
    ref.check(pool)
    kc, vc = (torch.full_like(buf.kc, 7.0) for _ in range(2))
    pool.read(buf.problem, buf.opts, table, buf.budgets, buf.seg_offsets, kc, vc)
    torch.cuda.synchronize()
    bud, so, tab = host(buf.budgets).reshape(-1), host(buf.seg_offsets), host(table)
    hkv, d = cfg.heads_kv, cfg.head_dim
    for w, got in enumerate((kc, vc)):
        want = np.full(got.numel(), bits(7.0), np.uint16)
        for bl, n in enumerate(bud):
            seg = want[so[bl] * hkv * d:so[bl + 1] * hkv * d].reshape(hkv, -1, d)
            seg[:, :n] = bits(ref.rows(w, tab[bl], 0, int(n)))
        got = bf16_host_bits(got)
        assert np.array_equal(np.where(got == 0x8000, 0, got), np.where(want == 0x8000, 0, want))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,page,head_mode", [(128, 16, 0), (64, 4, 1)])
@pytest.mark.parametrize("drop", [0, 1, 100])
def test_store_into_a_narrow_table(lib, kind, d, page, head_mode, drop):
    """A table as wide as its longest segment needs, and narrower ones: the rows that it names are stored as into a wide
    one, the others nowhere."""
    import torch
    log(f"narrow table kind={kind} d={d} page={page} head_mode={head_mode} drop={drop}")
    rng = np.random.default_rng(7)
    B, L, hkv, N = 2, 3, 2, 300
    bud = np.array([[40, 130, 10], [1, 90, 89]], np.int32)  # one layer may hold all 180 of a sequence
    k, v = (bits(rng.standard_normal((B, L, hkv, N, d))) for _ in range(2))
    longest = -(-int(bud.max()) // page)
    width = max(1, longest - drop)
    p, o = bd.make_problem(B, L, hkv, hkv, d, 0, N, 0), bd.make_opts(head_mode=head_mode)
    assert width < bd.page_plan(p, o, 180, 0, page)[0]
    ref = Pool(B * L * longest + 2, hkv, page, d, kind)
    table = rng.permutation(B * L * longest)[:B * L * width].reshape(B * L, width).astype(np.int32)
    g = hkv if head_mode else 1
    pick = [[np.sort(rng.choice(N, n, replace=False)) for _ in range(g)] for n in bud.reshape(-1)]
    off = np.concatenate([[0], np.cumsum(bud.reshape(-1).astype(np.int64) * g)])
    pool = ref.device()
    pool.store(p, o, dev_bf16(k), dev_bf16(v), _up(np.concatenate([x for q in pick for x in q]).astype(np.int32)), _up(bud),
               _up(off), 180, _up(table))
    torch.cuda.synchronize()
    for bl in range(B * L):
        for w, x in enumerate((k, v)):
            rows = np.stack([x.reshape(B * L, hkv, N, d)[bl, h][pick[bl][h if head_mode else 0]] for h in range(hkv)], 1)
            for r in range(min(len(rows), width * page)):
                ref.write(w, table[bl], r, rows[r])
    ref.check(pool)


@pytest.mark.parametrize("kind", KINDS)
def test_read_parts(lib, kind):
    """Rows from `first` on, counts of nothing, above the segment's room and negative, pages that end inside."""
    import torch
    log(f"read parts kind={kind}")
    rng = np.random.default_rng(5)
    hkv, d, page, need = 3, 64, 8, [40, 40, 7, 40, 24]
    ref = Pool(30, hkv, page, d, kind)
    table = np.full((5, 5), -1, np.int32)
    ids, at = rng.permutation(30).astype(np.int32), 0
    for i, n in enumerate(need):
        m = -(-n // page)
        table[i, :m] = ids[at:at + m]
        at += m
        b = bits(rng.standard_normal((2, n, hkv, d)))
        for w in range(2):
            for r in range(n):
                ref.write(w, table[i], r, b[w, r])
    pool = ref.device()
    first, count, room = [0, 33, 6, 5, 11], [40, 7, 1, 50, -3], [40, 9, 1, 20, 4]
    so = np.concatenate([[0], np.cumsum(room)]).astype(np.int64)
    p = bd.make_problem(5, 1, hkv, hkv, d, 1, 0, 0)
    out = [torch.full((int(so[-1]) * hkv * d,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pool.read(p, None, _up(table), _up(np.array(count, np.int32)), _up(so), *out, first=_up(np.array(first, np.int32)))
    torch.cuda.synchronize()
    for w, got in enumerate(out):
        want = np.full(got.numel(), bits(7.0), np.uint16)
        for i in range(5):
            n = max(0, min(count[i], room[i]))
            seg = want[so[i] * hkv * d:so[i + 1] * hkv * d].reshape(hkv, room[i], d)
            seg[:, :n] = bits(ref.rows(w, table[i], first[i], first[i] + n))
        got = bf16_host_bits(got)
        assert np.array_equal(np.where(got == 0x8000, 0, got), np.where(want == 0x8000, 0, want))


@pytest.mark.parametrize("kind", KINDS)
def test_read_stays_in_the_output(lib, kind):
    """A segment that ends behind the output is left out, the others are read; nor is anything behind the table's rows."""
    import torch
    log(f"read bounds kind={kind}")
    rng = np.random.default_rng(6)
    ref = Pool(6, 2, 8, 64, kind)
    table = np.array([[3, 1], [0, 4], [5, 2]], np.int32)
    for w in range(2):
        for i in range(3):
            for r in range(16):
                ref.write(w, table[i], r, bits(rng.standard_normal((2, 64))))
    p = bd.make_problem(3, 1, 2, 2, 64, 1, 0, 0)
    so = np.array([0, 10, 40, 52], np.int64)
    out = [torch.full((45 * 2 * 64,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ref.device().read(p, None, _up(table), _up(np.array([10, 30, 5], np.int32)), _up(so), *out,
                      first=_up(np.array([2, 4, 0], np.int32)))
    torch.cuda.synchronize()
    for w, got in enumerate(out):
        want = np.full(got.numel(), bits(7.0), np.uint16)
        want[:10 * 128].reshape(2, 10, 64)[:] = bits(ref.rows(w, table[0], 2, 12))
        want[10 * 128:40 * 128].reshape(2, 30, 64)[:, :12] = bits(ref.rows(w, table[1], 4, 16))
        got = bf16_host_bits(got)
        assert np.array_equal(np.where(got == 0x8000, 0, got), np.where(want == 0x8000, 0, want))


@pytest.mark.parametrize("kind", Q8)
def test_bad_rows_read_as_nan(lib, kind):
    """A retained row with an infinity reads as NaN in every place, its neighbours do not."""
    import torch
    rows = bits(np.random.default_rng(3).standard_normal((20, 128)))
    rows[7, 100] = 0x7F80
    k = dev_bf16(rows.reshape(1, 1, 1, 20, 128))
    pool = bd.PagedPool(1, 128, 16, 2, kind=kind)
    p = bd.make_problem(1, 1, 1, 1, 128, 0, 20, 0)
    table, n = _up(np.array([[1, 0]], np.int32)), _up(np.array([[20]], np.int32))
    pool.store(p, None, k, k, _up(np.arange(20, dtype=np.int32)), n, _up(np.array([0, 20])), 20, table)
    out = [torch.zeros(20 * 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pool.read(p, None, table, n, _up(np.array([0, 20])), *out)
    torch.cuda.synchronize()
    want = held(rows, kind)
    for o in out:
        assert np.array_equal(o.double().cpu().numpy().reshape(20, 128), want, equal_nan=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", [(8, 8, 128), (14, 2, 64)])
def test_a_serving_loop(lib, kind, heads):
    """Evict, admit, two decode steps, a ragged chunk, the appended rows read back, and the whole cache read into a
    contiguous one that the next decode step runs on: each step against the 64-bit form on the same pages."""
    import torch
    log(f"serving loop kind={kind} heads={heads}")
    cfg, t, buf, pool, table, ref = _retained(kind, 16, heads, dict(batch=3, layers=2, n_sys=5, n_vis=200, n_qst=14), 0.2,
                                              reserve=12, seed=2)
    hq, hkv, d = heads
    B, L = 3, 2
    rng = np.random.default_rng(8)
    bud, tab = host(buf.budgets), host(table)
    c = dict(B=B, L=L, hq=hq, hkv=hkv, d=d, kind=kind, page=16, budgets=bud, reserve=12, table=tab, pool=ref, order=None)
    steps = np.zeros(B, np.int32)
    for chunk, n_new in ((1, None), (1, None), (6, [6, 3, 1]), (1, [1, 0, 1])):
        c.update(chunk=chunk, steps=steps.copy(), n_new=None if n_new is None else np.array(n_new, np.int32))
        for name, h in (("q", hq), ("k_new", hkv), ("v_new", hkv)):
            c[name] = bits(rng.standard_normal((B, L, chunk, h, d)))
        # the host pool is appended to after the call; the device pool is the loop's own
        check(c, pool=pool)
        added = np.full(B, chunk, np.int32) if n_new is None else np.array(n_new, np.int32)
        seg = np.concatenate([[0], np.cumsum(np.repeat(added, L))]).astype(np.int64)
        out = [torch.zeros(int(seg[-1]) * hkv * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        first = (bud + steps[:, None]).astype(np.int32)
        pool.read(buf.problem, None, table, _up(np.repeat(added, L)), _up(seg), *out, first=_up(first))
        torch.cuda.synchronize()
        for w, name in enumerate(("k_new", "v_new")):
            for bl in range(B * L):
                got = out[w][seg[bl] * hkv * d:seg[bl + 1] * hkv * d].double().cpu().numpy().reshape(hkv, -1, d)
                new = held(c[name].reshape(B * L, chunk, hkv, d)[bl, :added[bl // L]], kind).swapaxes(0, 1)
                assert np.array_equal(got, new)
        steps += added
    # into a contiguous cache, sequence 0 alone, and one decode step there
    one = bd.make_problem(1, L, hq, hkv, d, 1, 0, 0)
    so = np.concatenate([[0], np.cumsum(bud[0].astype(np.int64) + 12)])
    kc, vc = (torch.zeros(int(so[-1]) * hkv * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pool.read(one, None, table[:L].contiguous(), _up((bud[0] + steps[0]).astype(np.int32)), _up(so), kc, vc)
    new = [bits(rng.standard_normal((1, L, h, d))) for h in (hq, hkv, hkv)]
    out = torch.empty(1, L, hq, d, device="cuda")
    ws = torch.zeros(max(1, bd.workspace_size(one, None, bd.CALL_DECODE)), dtype=torch.uint8, device="cuda")
    bd.tgvkv_decode_attn(one, None, kc, vc, _up(bud[0]), _up(so), 12, int(steps[0]), *(dev_bf16(x) for x in new), out, ws)
    torch.cuda.synchronize()
    for l in range(L):
        n = int(bud[0, l] + steps[0])
        for h in range(hq):
            k = np.concatenate([ref.rows(0, tab[l], 0, n)[h // (hq // hkv)], bf16_bits_to_f32(new[1][0, l, h // (hq // hkv)])[None]])
            v = np.concatenate([ref.rows(1, tab[l], 0, n)[h // (hq // hkv)], bf16_bits_to_f32(new[2][0, l, h // (hq // hkv)])[None]])
            z = k @ bf16_bits_to_f32(new[0][0, l, h]).astype(np.float64) / np.sqrt(d)
            pr = np.exp(z - z.max())
            want = (pr / pr.sum()) @ v
            # decode's 16-bit probabilities, and logits of d 32-bit products (see tests/pages_util.py)
            assert np.abs(out[0, l, h].double().cpu().numpy() - want).max() <= 1e-4 * np.abs(v).max()


@pytest.mark.parametrize("kind", KINDS)
def test_a_captured_admission(lib, kind):
    """Store, a chunk and a read in one graph, on a stream of its own, replayed with other keys, values, budgets and steps:
    the same bits as the calls made one by one on another pool, which run between the replays."""
    import torch
    log(f"captured admission kind={kind}")
    B, L, hq, hkv, d, N, page, chunk, reserve, kept = 2, 2, 4, 2, 64, 200, 16, 3, 8, 90
    p, width = bd.make_problem(B, L, hq, hkv, d, 0, N, 0), -(-(80 + reserve) // page)
    pools = [bd.PagedPool(hkv, d, page, B * L * width, kind=kind) for _ in range(2)]
    for pool in pools:  # unwritten pages alike
        for t in (pool.k_pool, pool.v_pool, pool.k_exp, pool.v_exp):
            if t is not None:
                t.view(torch.uint8).zero_()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    zeros = lambda dtype, *s: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    table = torch.randperm(B * L * width, generator=gen, device="cuda").to(torch.int32).view(B * L, width)
    k, v = rand(B, L, hkv, N, d), rand(B, L, hkv, N, d)
    q, kn, vn = rand(B, L, chunk, hq, d), rand(B, L, chunk, hkv, d), rand(B, L, chunk, hkv, d)
    idx, budgets, steps, n_new = zeros(torch.int32, B * kept), zeros(torch.int32, B, L), zeros(torch.int32, B), zeros(torch.int32, B)
    ioff, seg, count = zeros(torch.int64, B * L + 1), zeros(torch.int64, B * L + 1), zeros(torch.int32, B * L)
    outs = [(zeros(torch.float32, B, L, chunk, hq, d), rand(B * (kept + L * reserve) * hkv * d), rand(B * (kept + L * reserve) * hkv * d))
            for _ in range(2)]
    ws = [torch.empty(max(16, bd.chunk_workspace_size(p, None, chunk)), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def go(i):
        out, kc, vc = outs[i]
        pools[i].store(p, None, k, v, idx, budgets, ioff, kept, table)
        pools[i].extend(p, None, table, budgets, reserve, steps, n_new, q, kn, vn, out, ws[i])
        pools[i].read(p, None, table, count, seg, kc, vc)
    rng = np.random.default_rng(5)

    def change(rep):
        first = rng.integers(10, 81, B)
        bud = np.stack([first, kept - first], 1).astype(np.int32)
        st, n = rng.integers(0, reserve - chunk + 1, B), rng.integers(0, chunk + 1, B)
        budgets.copy_(_up(bud))
        steps.copy_(_up(st.astype(np.int32)))
        n_new.copy_(_up(n.astype(np.int32)))
        idx.copy_(_up(np.concatenate([np.sort(rng.choice(N, m, replace=False)) for m in bud.reshape(-1)]).astype(np.int32)))
        ioff.copy_(_up(np.concatenate([[0], np.cumsum(bud.reshape(-1))]).astype(np.int64)))
        seg.copy_(_up(np.concatenate([[0], np.cumsum(bud.reshape(-1) + reserve)]).astype(np.int64)))
        count.copy_(_up((bud + (st + n)[:, None]).reshape(-1).astype(np.int32)))
        for x in (k, v, q, kn, vn):
            x.copy_(rand(*x.shape))
        for x, y in zip(*outs):
            x.fill_(rep)
            y.fill_(rep)
    change(0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        go(0)
    go(1)  # the rows between the budgets and the steps, which this test does not write, are of earlier calls: the same in both
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        go(0)
    for rep in range(5):
        change(rep)
        torch.cuda.synchronize()
        graph.replay()
        go(1)
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.int8), y.view(torch.int8)) for x, y in zip(*outs)), rep
        for name in ("k_pool", "v_pool", "k_exp", "v_exp"):
            x, y = (getattr(pool, name) for pool in pools)
            assert x is None or torch.equal(x.view(torch.int8), y.view(torch.int8)), (rep, name)


def test_pool_arguments_are_checked(lib):
    import torch
    log("pool checks")
    with pytest.raises(ValueError):
        bd.PagedPool(2, 64, 8, 4, kind=3)
    pool = bd.PagedPool(2, 64, 8, 4, kind=bd.CACHE_FP8)
    p = bd.make_problem(1, 1, 4, 2, 64, 1, 0, 0)
    z = torch.zeros(1, 1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    kn = torch.zeros(1, 1, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    i32 = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(1, bd.chunk_workspace_size(p, None, 1)), dtype=torch.uint8, device="cuda")
    out = torch.full((1, 1, 1, 4, 64), 7.0, device="cuda")

    def go(**kw):
        a = dict(table=table, budgets=i32, reserve=4, steps=i32, n_new=None, q=z, k=kn, v=kn, out=out)
        a.update(kw)
        pool.extend(p, None, a["table"], a["budgets"], a["reserve"], a["steps"], a["n_new"], a["q"], a["k"], a["v"], a["out"], ws)
    for bad, err in [(dict(q=z.float()), TypeError), (dict(out=out.half()), TypeError), (dict(q=z[..., :32]), ValueError),
                     (dict(k=z), ValueError), (dict(n_new=torch.zeros(2, dtype=torch.int32, device="cuda")), ValueError),
                     (dict(steps=i32.cpu()), ValueError), (dict(table=table[0]), ValueError),
                     (dict(budgets=i32.long()), TypeError), (dict(reserve=-1), bd.TgvkvError)]:
        with pytest.raises(err):
            go(**bad)
    keep = pool.k_exp
    for exp in (None, keep[:, :, :4].contiguous(), keep.float()):
        pool.k_exp = exp
        with pytest.raises((ValueError, TypeError)):
            go()
    pool.k_exp = keep
    pool.k_pool = pool.k_pool.view(torch.int8)
    with pytest.raises(TypeError):
        go()
    torch.cuda.synchronize()
    assert torch.all(out == 7.0)


def test_memory_elsewhere_is_refused(lib, monkeypatch):
    """Every tensor has to be in the current GPU's memory: host tensors, and a pool of another device than the current."""
    import torch
    log("pool on another device")
    dev = lambda dtype, *shape: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
    p = bd.make_problem(1, 1, 4, 2, 64, 1, 0, 0)
    i32, b16 = torch.int32, torch.bfloat16
    for kind in KINDS:
        pool = bd.PagedPool(2, 64, 8, 4, kind=kind)
        calls = [(pool.extend, [dev(i32, 1, 2), dev(i32, 1), 4, dev(i32, 1), dev(i32, 1), dev(b16, 1, 1, 1, 4, 64),
                                dev(b16, 1, 1, 1, 2, 64), dev(b16, 1, 1, 1, 2, 64), dev(b16, 1, 1, 1, 4, 64),
                                dev(torch.uint8, max(16, bd.chunk_workspace_size(p, None, 1)))]),
                 (pool.read, [dev(i32, 1, 2), dev(i32, 1), dev(torch.int64, 2), dev(b16, 128), dev(b16, 128)])]
        for f, args in calls:
            for i, a in enumerate(args):
                if torch.is_tensor(a):
                    with pytest.raises(ValueError, match="memory"):
                        f(p, None, *args[:i], a.cpu(), *args[i + 1:])
            with monkeypatch.context() as m:
                m.setattr(torch.cuda, "current_device", lambda: 1)
                with pytest.raises(ValueError, match="current GPU"):
                    f(p, None, *args)
