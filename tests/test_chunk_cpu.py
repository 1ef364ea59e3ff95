"""Refusals of the calls on pages of any kind, and the plain quantiser's own properties (no GPU)."""

import ctypes
import os

import numpy as np
import pytest

from paper_2606_03075_amd import binding as bd
from tests.pages_util import E4M3, bits, quantise, values
from workloads import bf16_bits_to_f32


def _gpu():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


@pytest.fixture(scope="module")
def so():
    if not os.path.exists(bd.LIB_PATH):
        from paper_2606_03075_amd import build
        build.build()
    return bd.load_library()


def P(**kw):
    base = dict(batch=1, layers=2, heads_q=4, heads_kv=2, head_dim=128, n_sys=3, n_vis=40, n_qst=5)
    base.update(kw)
    return bd.make_problem(**base)


FAKE, ODD, BIG, S = 0x10000, 0x10008, 1 << 40, ctypes.c_void_p(0)


def pages(k=FAKE, v=FAKE, ke=FAKE, ve=FAKE, n=64, size=8, kind=1):
    return ctypes.byref(bd.TgvkvPages(k, v, ke, ve, n, size, kind))


BAD_POOLS = [(dict(n=0), -1), (dict(n=1 << 31), -2), (dict(size=12), -1), (dict(size=0), -1), (dict(size=8192), -1),
             (dict(kind=3), -1), (dict(kind=-1), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(k=ODD), -1),
             (dict(ke=None), -1), (dict(ve=None, kind=2), -1), (dict(ve=ODD), -1)]


@pytest.mark.skipif(_gpu(), reason="fake pointers are used only where no GPU exists")
def test_chunk_refusals(so):
    def go(problem=None, pool=pages(), table=FAKE, width=2, budgets=FAKE, reserve=4, steps=FAKE, chunk=3, q=FAKE, kn=FAKE,
           vn=FAKE, out=FAKE, ws=FAKE, n=BIG, opts=None):
        return so.tgvkv_chunk_attn_pages(ctypes.byref(problem or P()), opts, pool, table, width, budgets, reserve, steps,
                                         None, chunk, q, kn, vn, out, 0, ws, n, None, S)
    for bad, code in BAD_POOLS:
        assert go(pool=pages(**bad)) == code, bad
    assert go(pool=None) == -1
    for bad, code in [(dict(table=None), -1), (dict(width=0), -1), (dict(width=5000), -2), (dict(budgets=None), -1),
                      (dict(reserve=-1), -1), (dict(steps=None), -1), (dict(chunk=0), -1), (dict(chunk=-3), -1),
                      (dict(chunk=1 << 30), -2), (dict(q=None), -1), (dict(kn=None), -1), (dict(vn=None), -1),
                      (dict(out=None), -1), (dict(q=ODD), -1), (dict(kn=ODD), -1), (dict(vn=ODD), -1), (dict(out=ODD), -1),
                      (dict(problem=P(head_dim=96)), -2), (dict(problem=P(heads_q=3)), -1),
                      (dict(problem=P(heads_q=34)), -2), (dict(opts=ctypes.byref(bd.make_opts(head_mode=2))), -1)]:
        assert go(**bad) == code, bad
    need = bd.chunk_workspace_size(P(), None, 3)
    if need:
        assert go(ws=None) == -3 and go(n=need - 1) == -3 and go(ws=ODD) == -3
    assert go(problem=P(batch=0), pool=pages(k=None), q=None, ws=None, n=0) == 0
    assert so.tgvkv_chunk_attn_pages(None, None, pages(), FAKE, 2, FAKE, 4, FAKE, None, 3, FAKE, FAKE, FAKE, FAKE, 0, FAKE, BIG,
                                     None, S) == -1


@pytest.mark.skipif(_gpu(), reason="fake pointers are used only where no GPU exists")
def test_store_and_read_refusals(so):
    def store(problem=None, pool=pages(), k=FAKE, v=FAKE, idx=FAKE, budgets=FAKE, offs=FAKE, total=10, table=FAKE, width=2):
        return so.tgvkv_compact_pages(ctypes.byref(problem or P()), None, k, v, idx, budgets, offs, total, pool, table, width,
                                      None, S)

    def read(problem=None, pool=pages(), table=FAKE, width=2, count=FAKE, seg=FAKE, rows=9, k=FAKE, v=FAKE):
        return so.tgvkv_read_pages(ctypes.byref(problem or P()), None, pool, table, width, None, count, seg, rows, k, v, S)
    for bad, code in BAD_POOLS:
        assert store(pool=pages(**bad)) == code, bad
        assert read(pool=pages(**bad)) == code, bad
    assert store(pool=None) == read(pool=None) == -1
    for bad, code in [(dict(k=None), -1), (dict(v=ODD), -1), (dict(idx=None), -1), (dict(budgets=None), -1),
                      (dict(offs=None), -1), (dict(total=-1), -1), (dict(total=2 * 48 + 1), -4), (dict(width=1), -4),
                      (dict(table=None), -1), (dict(problem=P(heads_q=3)), -1)]:
        assert store(**bad) == code, bad
        assert store(pool=pages(kind=0), **bad) == code, bad  # as tgvkv_compact_paged
    for bad, code in [(dict(table=None), -1), (dict(width=0), -1), (dict(width=4097), -2), (dict(count=None), -1),
                      (dict(seg=None), -1), (dict(rows=-1), -1), (dict(k=None), -1), (dict(v=ODD), -1), (dict(problem=P(head_dim=32)), -2)]:
        assert read(**bad) == code, bad
    assert read(rows=0, k=None) == 0
    assert store(problem=P(batch=0), pool=pages(k=None)) == read(problem=P(batch=0), pool=pages(k=None)) == 0


@pytest.mark.skipif(_gpu(), reason="fake pointers are used only where no GPU exists")
def test_a_store_takes_a_table_of_any_width(so):
    """Refusals as tgvkv_compact_pages', but for the width.  (A null tensor behind the width check tells that it passed
    without reaching a launch.)"""
    def store(problem=None, pool=pages(), k=FAKE, v=FAKE, idx=FAKE, budgets=FAKE, offs=FAKE, total=10, table=FAKE, width=2,
              call=None):
        return (call or so.tgvkv_store_pages)(ctypes.byref(problem or P()), None, k, v, idx, budgets, offs, total, pool, table,
                                              width, None, S)
    for bad, code in BAD_POOLS:
        assert store(pool=pages(**bad)) == code, bad
    assert store(pool=None) == -1
    for kind in (0, 1, 2):
        pool = pages(kind=kind)
        for bad, code in [(dict(k=None), -1), (dict(v=ODD), -1), (dict(idx=None), -1), (dict(budgets=None), -1),
                          (dict(offs=None), -1), (dict(total=-1), -1), (dict(total=2 * 48 + 1), -4), (dict(width=0), -1),
                          (dict(width=4097), -2), (dict(table=None), -1), (dict(problem=P(heads_q=3)), -1)]:
            assert store(pool=pool, **bad) == code, (kind, bad)
            assert store(pool=pool, width=bad.pop("width", 1), **bad) == code, (kind, bad)
        assert store(pool=pool, width=1, idx=None, call=so.tgvkv_compact_pages) == -4
    # one image question kept at a tenth: 32 layers share 2083 tokens, the longest holds 208 of them
    image = P(layers=32, heads_q=32, heads_kv=32, n_sys=0, n_vis=651, n_qst=0)
    need = bd.page_plan(image, None, 2083, 0, 16)[0]
    assert need == 41
    for width, code in ((13, -4), (41, -1)):
        assert store(problem=image, pool=pages(size=16), total=2083, width=width, idx=None, call=so.tgvkv_compact_pages) == code
        assert store(problem=image, pool=pages(size=16), total=2083, width=width, idx=None) == -1
    assert store(problem=P(batch=0), pool=pages(k=None)) == 0


@pytest.mark.skipif(_gpu(), reason="fake pointers are used only where no GPU exists")
def test_more_workgroups_than_a_launch_numbers(so):
    """A launch's threads are numbered in 32 bits; one of 2^24 workgroups of 256 runs only a part of them, without an error
    (33000 x 512 segments: the last sequence's results were left as they were).  Such calls are refused."""
    def calls(batch, layers, hq, hkv, chunk=1):
        p = ctypes.byref(P(batch=batch, layers=layers, heads_q=hq, heads_kv=hkv, head_dim=64, n_sys=0, n_vis=4, n_qst=0))
        yield "chunk", so.tgvkv_chunk_attn_pages(p, None, pages(), FAKE, 1, FAKE, 4, FAKE, None, chunk, FAKE, FAKE, FAKE, FAKE, 0,
                                                 FAKE, BIG, None, S)
        if chunk == 1:
            for kind in (0, 1):
                for call in (so.tgvkv_compact_pages, so.tgvkv_store_pages):
                    yield "store", call(p, None, FAKE, FAKE, FAKE, FAKE, FAKE, layers, pages(kind=kind, size=1024), FAKE, 1, None, S)
            yield "store", so.tgvkv_store_pages(p, None, FAKE, FAKE, FAKE, FAKE, FAKE, layers, pages(kind=0, size=1), FAKE, 1, None, S)
            yield "compact", so.tgvkv_compact(p, None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, layers, 1, FAKE, FAKE, None, S)
            yield "decode", so.tgvkv_decode_attn(p, None, FAKE, FAKE, FAKE, FAKE, 4, 0, FAKE, FAKE, FAKE, FAKE, FAKE, BIG, None, S)
            yield "decode", so.tgvkv_decode_attn_paged(p, None, FAKE, FAKE, 64, 8, FAKE, 1, FAKE, 4, FAKE, FAKE, FAKE, FAKE, FAKE,
                                                       FAKE, BIG, None, S)
    read = lambda batch, layers, hkv: so.tgvkv_read_pages(ctypes.byref(P(  # noqa: E731
        batch=batch, layers=layers, heads_q=hkv, heads_kv=hkv, head_dim=64)), None, pages(), FAKE, 1, None, FAKE, FAKE, 9, FAKE, FAKE, S)
    for shape in [(1 << 15, 512, 1, 1), (33000, 512, 2, 1), (1 << 14, 512, 2, 2), (1 << 12, 512, 8, 8), (1 << 13, 512, 2, 2, 130)]:
        for name, status in calls(*shape):
            assert status == -2, (name, shape)
    assert read(1 << 17, 512, 1) == read(1 << 15, 512, 4) == -2  # reads take one wave per segment there


def test_stores_check_their_tensors_sizes(so, monkeypatch):
    """A tensor too small for the problem is refused before the call, which reads by the problem's sizes: a short `budgets`
    or `idx` would be read out of range on the GPU.  (Host tensors, taken for the GPU's; the library's calls only count.)"""
    import torch
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    real = bd.load_library()
    Library.tgvkv_sizes = staticmethod(lambda *a: real.tgvkv_sizes(*a))
    monkeypatch.setattr(bd, "load_library", lambda path=None: Library())
    monkeypatch.setattr(bd, "_pages", lambda pool, hkv, d: (bd.TgvkvPages(), -1))  # host tensors' device number
    monkeypatch.setattr(bd, "_stream_on", lambda stream, device: 0)
    bd._import_torch()
    zeros = lambda n, dtype: torch.zeros(n, dtype=dtype)  # noqa: E731
    B, L, hkv, N, d = 2, 3, 2, 48, 64
    for head_mode, vision_only, kept in ((0, False, 90), (1, False, 90), (0, True, 90 + 3 * 8)):
        p, o = P(batch=B, layers=L, heads_kv=hkv, head_dim=d), bd.make_opts(head_mode=head_mode, vision_only=vision_only)
        good = dict(k=zeros(B * L * hkv * N * d, torch.bfloat16), v=zeros(B * L * hkv * N * d, torch.bfloat16),
                    idx=zeros(B * kept * (hkv if head_mode else 1), torch.int32), budgets=zeros(B * L, torch.int32),
                    idx_offsets=zeros(B * L + 1, torch.int64), table=zeros((B * L, 6), torch.int32),
                    unit_order=zeros(B * L, torch.int32))

        def go(call, **kw):
            a = dict(good, **kw)
            call(p, o, a["k"], a["v"], a["idx"], a["budgets"], a["idx_offsets"], 90, None, a["table"], unit_order=a["unit_order"])
        for call in (bd.tgvkv_compact_pages, bd.tgvkv_store_pages):
            del calls[:]
            go(call)
            go(call, unit_order=None, idx=torch.cat([good["idx"], good["idx"]]))  # room to spare
            assert calls == [call.__name__] * 2
            for name in ("k", "v", "idx", "budgets", "idx_offsets", "unit_order"):
                with pytest.raises(ValueError, match=name):
                    go(call, **{name: good[name][:-1].contiguous()})
            with pytest.raises(ValueError):
                go(call, table=good["table"][1:].contiguous())
            assert len(calls) == 2


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_attached_pools_are_checked(kind):
    """attach() takes only tensors of the pool's own layout and kind, and leaves the pool as it was otherwise; no page is
    free for admit() but those that the caller names, for its tables may use any."""
    import torch
    dtype = (torch.bfloat16, torch.float8_e4m3fn, torch.int8)[kind]
    make = lambda n, hkv=2, page=8, d=64, t=dtype: torch.empty(n, hkv, page, d, dtype=t)  # noqa: E731
    exps = lambda n, hkv=2, page=8, t=torch.uint8: None if kind == 0 else torch.zeros(n, hkv, page, dtype=t)  # noqa: E731
    pool = bd.PagedPool(2, 64, 8, 3, device="cpu", kind=kind)
    assert pool.free == [0, 1, 2]
    before = (pool.k_pool, pool.v_pool, pool.k_exp, pool.v_exp)
    k, v, ke, ve = make(5), make(5), exps(5), exps(5)
    bad = [(make(5, hkv=3), v, ke, ve), (k, make(4), ke, ve), (make(5, page=16), make(5, page=16), ke, ve),
           (make(5, d=128), make(5, d=128), ke, ve), (k.view(torch.uint8), v, ke, ve), (k, None, ke, ve), (None, v, ke, ve),
           (make(10)[::2], v, ke, ve), (k, v.transpose(0, 1), ke, ve), (make(0), make(0), exps(0), exps(0)), (k[0], v[0], ke, ve)]
    if kind:
        bad += [(k, v, None, ve), (k, v, ke, exps(4)), (k, v, ke.to(torch.int8), ve), (k, v, ke, exps(10)[::2])]
    else:
        bad += [(k, v, torch.zeros(5, 2, 8, dtype=torch.uint8), None)]
    for args in bad:
        with pytest.raises((ValueError, TypeError)):
            pool.attach(*args)
    for free in ([5], [-1], [1, 2, 1]):
        with pytest.raises(ValueError):
            pool.attach(k, v, ke, ve, free=free)
    assert all(a is b for a, b in zip(before, (pool.k_pool, pool.v_pool, pool.k_exp, pool.v_exp)))
    assert pool.free == [0, 1, 2] and pool.n_pages == 3
    pool.attach(k, v, ke, ve)
    assert pool.free == [] and pool.n_pages == 5 and pool.k_pool is k and pool.v_exp is ve
    pool.attach(k, v, ke, ve, free=range(2, 5))
    assert pool.free == [2, 3, 4]
    pool.release(torch.tensor([[0, 1, -1]], dtype=torch.int32))
    assert pool.free == [2, 3, 4, 0, 1]


def test_chunk_workspace_size(so):
    assert bd.chunk_workspace_size(P(head_dim=96), None, 1) == 0
    assert bd.chunk_workspace_size(P(), None, 0) == 0
    assert bd.chunk_workspace_size(P(), None, 1 << 30) == 0
    for batch in (1, 7, 64):
        for chunk in (1, 4, 64, 1000):
            assert 0 <= bd.chunk_workspace_size(P(batch=batch, layers=32), None, chunk) <= 1 << 30


@pytest.mark.parametrize("g", [1, 4, 7, 16])
@pytest.mark.parametrize("batch,layers,hkv", [(1, 1, 1), (1, 5, 2), (8, 28, 4), (4, 32, 8), (16, 40, 40), (64, 40, 1)])
def test_one_workspace_serves_every_smaller_chunk(so, g, batch, layers, hkv):
    """chunk_workspace_size is for chunks of UP TO its argument: it never falls as the argument grows, also where larger
    chunks need none themselves.  Up to 2048 items (units times row tiles) a call needs 896 partials of the tile's rows
    (16, 32, 64 or 128, by the chunk's query rows), each of head_dim + 2 floats, and a mark of 8 bytes each."""
    p = P(batch=batch, layers=layers, heads_q=g * hkv, heads_kv=hkv)

    def need(chunk):
        rows = chunk * g
        tile, tiles = (16, 1) if rows <= 16 else (32, 1) if rows <= 32 else (64, 1) if rows <= 64 else (128, -(-rows // 128))
        if batch * layers * hkv * tiles > 2048 or batch * layers > 2048:
            return 0
        return -(-896 * (tile * (128 + 2) * 4 + 8) // 256) * 256
    most = 0
    for chunk in [*range(1, 300), 1000, 4096]:
        most = max(most, need(chunk))
        assert bd.chunk_workspace_size(p, None, chunk) == most, chunk


def test_an_older_library_is_refused(tmp_path):
    """A library without the calls on pages of any kind does not load."""
    import subprocess
    src = tmp_path / "old.c"
    names = [n for n in bd.EXPORTS + bd.CEILING_EXPORTS if "pages" not in n]
    src.write_text("".join(f"long {n}(void) {{ return {bd.ABI_VERSION if n == 'tgvkv_abi_version' else -1}; }}\n" for n in names))
    lib = tmp_path / "libold.so"
    r = subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(lib), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    with pytest.raises(RuntimeError, match="rebuild"):
        bd.load_library(str(lib))


def test_one_term_bound_tells_two_parts_from_three():
    """The arithmetic of the products with V in float32: probabilities in three bf16 parts stay below the bound that the
    GPU tests hold the kernels to, in two parts they do not."""
    from tests.pages_util import ONE_TERM_BOUND
    f32 = np.float32

    def parts_of(p, n):
        out = np.zeros_like(p)
        for _ in range(n):
            b = bf16_bits_to_f32(bits(p))
            out, p = out + b, p - b
        return out.astype(np.float64)
    rng = np.random.default_rng(0)
    worst = {2: [], 3: []}
    for d in (64, 128):
        for _ in range(20):
            a = bf16_bits_to_f32(bits(rng.uniform(0, 8, (4, d))))
            want = np.exp(a.astype(np.float64) / np.sqrt(d))
            want /= want.sum(1, keepdims=True)
            scale2 = f32(f32(1) / np.sqrt(f32(d))) * f32(1.4426950408889634)
            ref = (a * scale2).max(1, keepdims=True) + f32(8)
            p = np.exp2((a * scale2 - ref).astype(np.float64)).astype(f32)
            for n in worst:
                x = parts_of(p, n)
                worst[n].append(np.abs(x / x.sum(1, keepdims=True) / want - 1).max())
    assert max(worst[3]) <= ONE_TERM_BOUND < min(worst[2])


def test_plain_quantiser():
    """The grid is e4m3's (torch's cast agrees on every code), the exponent is the least that fits, a row of its own
    values is left as it is."""
    import torch
    assert np.array_equal(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(), E4M3, equal_nan=True)
    rng = np.random.default_rng(0)
    rows = bits(rng.standard_normal((50, 64)) * 2.0 ** rng.integers(-30, 30, (50, 1)))
    x = bf16_bits_to_f32(rows).astype(np.float64)
    for kind, most in ((bd.CACHE_FP8, 448.0), (bd.CACHE_INT8, 127.0)):
        codes, exp = quantise(rows, kind)
        unit = 2.0 ** (exp.astype(int) - 127)
        amax = np.abs(x).max(-1)
        assert np.all(amax <= most * unit) and np.all(amax > most * unit / 2)
        v = values(codes, exp, kind)
        again = quantise(bits(v), kind)
        assert np.array_equal(values(*again, kind), v)
        if kind == bd.CACHE_FP8:
            y = torch.from_numpy((x / unit[:, None]).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            assert np.array_equal(y, codes)
