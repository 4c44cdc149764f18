"""Operators on pages of the 4-bit cache that requests share or pick from, against the oracle: tables and counts, attention behind common pages, bounds, selection, attention over selected pages,
and runs of them as a server makes them."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages as ref
from oracle import requests as q4
from paper_2505_00232_amd import binding as B
from test_requests import DEV, _close, _filled, _normal, _pages, _requests, _t

gpu = pytest.mark.gpu


def _i(x):
    return torch.tensor(np.asarray(x, dtype=np.int32)).to(DEV)


def _space(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)


# ---------------------------------------------------------------- refusals, without a GPU
def test_page_refusals_before_any_launch():
    L, A, odd, s, size = B.lib(), 0x1000, 0x1002, ctypes.c_void_p(0), ctypes.c_size_t(0)
    cache = lambda pages=A, num=4, h=2, d=64: ctypes.byref(B.CacheDesc(pages, num, h, d))
    far, big = 0x100000, 1 << 40
    assert L.qfc_pages_workspace_size(cache(None), 3, ctypes.byref(size)) == 0 and size.value > 0
    assert L.qfc_pages_workspace_size(cache(), 0, ctypes.byref(size)) == 1 and L.qfc_pages_workspace_size(cache(), 3, None) == 1 and L.qfc_pages_workspace_size(None, 3, ctypes.byref(size)) == 1
    assert L.qfc_pages_workspace_size(cache(d=96), 3, ctypes.byref(size)) == 2 and L.qfc_pages_workspace_size(cache(), (1 << 22) + 1, ctypes.byref(size)) == 2
    take = lambda c=cache(), r=A, t=A, p=A, b=2, w=3, m=A, ws=A, n=big: L.qfc_take_pages(c, r, t, p, b, w, m, ws, n, s)
    fork = lambda c=cache(), r=A, f=far, fb=2, fw=3, pa=A, p=A, t=A, b=2, w=3, m=A, ws=A, n=big, bd=None: L.qfc_fork_pages(c, r, f, fb, fw, pa, p, t, b, w, m, bd, ws, n, s)
    free = lambda c=cache(), r=A, t=A, k=A, b=2, w=3: L.qfc_free_pages(c, r, t, k, b, w, s)
    compact = lambda c=cache(), r=A, t=A, b=2, w=3, m=A, ws=A, n=big, bd=None: L.qfc_compact_pages(c, r, t, b, w, m, bd, ws, n, s)
    for call in (take, fork, free, compact):
        assert call(c=None) == 1 and call(c=cache(num=0)) == 1 and call(r=None) == 1 and call(t=None) == 1 and call(b=0) == 1 and call(w=0) == 1 and call(b=-1) == 1
        assert call(c=cache(d=80)) == 2 and call(b=(1 << 22) + 1) == 2 and call(c=cache(h=1 << 20)) == 2
        assert call(b=1 << 22, w=512) == 2 and call(b=3, w=(1 << 31) - 1) == 2  # tables of 2^31 entries and more
        assert call(r=odd) == 4 and call(t=odd) == 4
    for call in (take, fork, compact):
        assert call(ws=None) == 1 and call(c=cache(None)) == 1 and call(n=8) == 3 and call(ws=0x1008) == 4 and call(m=odd) == 4 and call(c=cache(0x1008)) == 4
    assert take(p=None) == 1 and take(p=odd) == 4 and free(k=odd) == 4
    for name in ("f", "pa", "p"):
        assert fork(**{name: None}) == 1 and fork(**{name: odd}) == 4
    assert fork(fb=0) == 1 and fork(fw=0) == 1
    assert fork(f=A) == 1 and fork(f=A + 20) == 1 and fork(f=A - 20) == 1  # tables that overlap
    copy = lambda f=cache(), t=cache(num=9), a=A, b=A, n=2, fb=None, tb=None: L.qfc_copy_pages(f, t, a, b, n, fb, tb, s)
    bounds = lambda c=A, t=A: ctypes.byref(B.BoundsDesc(c, t))
    for call in (fork, compact, lambda bd: copy(fb=bd, tb=bounds()), lambda bd: copy(fb=bounds(), tb=bd)):
        assert call(bd=bounds(None)) == 1 and call(bd=bounds(t=None)) == 1 and call(bd=bounds(0x1008)) == 4 and call(bd=bounds(t=odd)) == 4
    assert copy(fb=bounds()) == 1 and copy(tb=bounds()) == 1
    assert copy(f=None) == 1 and copy(t=None) == 1 and copy(t=cache(h=3)) == 1 and copy(t=cache(d=128)) == 1 and copy(n=-1) == 1 and copy(a=None) == 1 and copy(b=None) == 1
    assert copy(f=cache(None)) == 1 and copy(f=cache(0x1008)) == 4 and copy(a=odd) == 4 and copy(b=odd) == 4 and copy(f=cache(d=32), t=cache(d=32)) == 2
    assert copy(n=0) == 0 and copy(n=0, a=None, b=None) == 0  # nothing to do


def test_attention_and_selection_refusals_before_any_launch():
    L, A, odd, s, size, big = B.lib(), 0x1000, 0x1002, ctypes.c_void_p(0), ctypes.c_size_t(0), 1 << 60
    cache = lambda pages=A, num=4, h=2, d=64: ctypes.byref(B.CacheDesc(pages, num, h, d))
    req = lambda start=A, ctx=A, table=A, batch=2, tokens=2, most=1, longest=128, width=2: ctypes.byref(B.RequestsDesc(start, ctx, table, batch, tokens, most, longest, width))
    shared = lambda g=A, p=A, n=1, tokens=2, longest=128: ctypes.byref(B.SharedDesc(g, p, n, tokens, longest))
    bounds = lambda c=A, t=A: ctypes.byref(B.BoundsDesc(c, t))
    common = lambda r=req(), c=cache(), h=4, sh=shared(), q=A, ws=A, n=big, o=A: L.qfc_attention_shared_q4(q, r, sh, h, c, ws, n, o, s)
    bound = lambda r=req(), c=cache(), b=bounds(): L.qfc_bound_pages_q4(r, c, b, s)
    select = lambda r=req(), c=cache(), h=4, b=bounds(), first=1, last=1, count=4, q=A, ws=A, n=big, o=A: L.qfc_select_pages_q4(q, r, h, c, b, first, last, count, ws, n, o, s)
    some = lambda r=req(), c=cache(), h=4, sel=A, count=4, q=A, ws=A, n=big, o=A: L.qfc_attention_selected_q4(q, r, h, c, sel, count, ws, n, o, s)
    for call in (common, bound, select, some):
        for bad in (None, req(start=None), req(ctx=None), req(table=None), req(batch=0), req(tokens=-1), req(most=0), req(longest=0), req(longest=129), req(width=0)):
            assert call(r=bad) == 1
        for bad in (None, cache(None), cache(num=0), cache(h=0)):
            assert call(c=bad) == 1
        assert call(c=cache(d=80)) == 2 and call(c=cache(odd)) == 4 and call(r=req(start=odd)) == 4 and call(r=req(batch=40000)) == 2
        assert call(r=req(tokens=0)) == 0  # nothing to do, nothing launched
    for call in (common, select, some):
        assert call(h=3) == 1 and call(h=0) == 1 and call(h=65534) == 2 and call(q=None) == 1 and call(ws=None) == 1 and call(o=None) == 1 and call(q=odd) == 4 and call(ws=odd) == 4
        assert call(o=0x1001) == 4 and call(n=8) == 3
    for bad in (None, shared(None), shared(p=None), shared(n=0), shared(tokens=0), shared(longest=0)):
        assert common(sh=bad) == 1
    assert common(sh=shared(n=32768)) == 2 and common(sh=shared(odd)) == 4 and common(sh=shared(p=odd)) == 4 and common(o=0x1008) == 4
    for call in (bound, select):
        assert call(b=None) == 1 and call(b=bounds(None)) == 1 and call(b=bounds(t=None)) == 1 and call(b=bounds(0x1008)) == 4 and call(b=bounds(t=odd)) == 4
    assert select(first=-1) == 1 and select(last=-1) == 1 and select(count=0) == 1 and select(first=3, last=2) == 1 and select(first=2 ** 31 - 1, last=2 ** 31 - 1) == 1 and select(count=65537) == 2
    assert some(sel=None) == 1 and some(sel=0x1001) == 4 and some(count=0) == 1 and some(count=65537) == 2 and some(o=0x1008) == 4
    q = ctypes.byref(size)
    for f in (lambda r, h, c, o: L.qfc_attention_shared_q4_workspace_size(r, shared(None, None), h, c, o), L.qfc_select_pages_q4_workspace_size,
              lambda r, h, c, o: L.qfc_attention_selected_q4_workspace_size(r, h, c, 5, o)):
        assert f(req(None, None, None), 4, cache(None), q) == 0 and size.value >= 256
        assert f(req(), 4, cache(), None) == 1 and f(None, 4, cache(), q) == 1 and f(req(), 3, cache(), q) == 1 and f(req(), 4, cache(d=96), q) == 2
    assert L.qfc_attention_shared_q4_workspace_size(req(), None, 4, cache(), q) == 1 and L.qfc_attention_selected_q4_workspace_size(req(), 4, cache(), 0, q) == 1


def test_binding_refuses_host_tensors_and_other_shapes():
    c = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.SharedPrefixes(torch.zeros(3, dtype=torch.int32), c, 2, 64)
    with pytest.raises(ValueError):
        B._table(torch.zeros(3, dtype=torch.int32), "page_table")
    with pytest.raises(ValueError):
        B._table(torch.zeros((3, 2), dtype=torch.int32), "page_table")


def _sizes(tokens, batch, most, longest, groups, group_tokens, common, h_q, h_kv, d, count):
    """Workspaces of attention behind common pages, of selection, of attention over selected pages."""
    L, out = B.lib(), []
    req = ctypes.byref(B.RequestsDesc(None, None, None, batch, tokens, most, longest, (longest + 63) // 64))
    cache = ctypes.byref(B.CacheDesc(None, 4, h_kv, d))
    for f in (lambda p: L.qfc_attention_shared_q4_workspace_size(req, ctypes.byref(B.SharedDesc(None, None, groups, group_tokens, common)), h_q, cache, p),
              lambda p: L.qfc_select_pages_q4_workspace_size(req, h_q, cache, p), lambda p: L.qfc_attention_selected_q4_workspace_size(req, h_q, cache, count, p)):
        size = ctypes.c_size_t(0)
        assert f(ctypes.byref(size)) == 0
        out.append(size.value)
    return np.array(out)


def _check_sizes():
    rng = np.random.default_rng(63)
    some = lambda most: int(np.exp(rng.uniform(0, np.log(most))))
    for _ in range(3000):
        d, h_kv, g = int(rng.choice([64, 128, 256])), int(rng.choice([1, 2, 4, 8])), int(rng.choice([1, 2, 4, 8, 20]))
        large = [some(2000), some(300), some(200), some(1 << 22), some(50), some(2000), some(1 << 22)]
        small = [max(1, int(x * rng.choice([1.0, 0.99, 0.5, rng.random()]))) for x in large]
        count = some(300)
        less = max(1, int(count * rng.random()))
        assert np.all(_sizes(*small, h_kv * g, h_kv, d, less) <= _sizes(*large, h_kv * g, h_kv, d, count)), (small, large, h_kv, g, d, less, count)


def test_workspaces_of_large_calls_serve_small_ones():
    _check_sizes()
    sizes = lambda tokens, longest: _sizes(tokens, tokens, 1, longest, 1, tokens, longest, 32, 8, 128, 32)[1]
    assert sizes(1, 32768) == 256 and sizes(1, 32769) == 256 + 8 * 513 * 4 and sizes(500, 1 << 20) == 256 + 512 * 16384 * 4


@gpu
def test_workspaces_of_large_calls_serve_small_ones_on_the_device(rows_rule):
    """One workspace each, of the largest batch's size, for all smaller ones: around the numbers of tokens and pages at which calls are made in another way."""
    _check_sizes()
    rng = np.random.default_rng(64)
    h_q, h_kv, d, pages, T, count = 16, 8, 64, 700, 40, 32
    cache = B.PagedCache(pages, h_kv, d)
    n = pages * 64
    k, v = _normal(rng, n, h_kv, d), _normal(rng, n, h_kv, d)
    table = rng.permutation(pages).astype(np.int32)[None]
    whole = _requests([n], [n], table)
    B.qfc_append_q4(_t(np.concatenate([k, k, v], 1).reshape(n, -1)), whole, h_kv, None, None, cache, torch.empty((n, h_kv * d), dtype=torch.float16, device=DEV))
    bounds = B.PageBounds(cache)
    B.qfc_bound_pages_q4(whole, cache, bounds)
    q = _t(_normal(rng, T, h_q * d))

    def call(tokens, longest, less, spaces):
        req = _requests([1] * tokens, [longest - i for i in range(tokens)], np.repeat(table[:, :(longest + 63) // 64], tokens, 0))
        shared = B.SharedPrefixes(_i([0, tokens]), _i([longest - tokens - 70]), tokens, longest)
        selected = torch.full((tokens, h_kv, less), -7, dtype=torch.int32, device=DEV)
        one, two = (torch.full((tokens, h_q * d), 3.0, dtype=torch.float16, device=DEV) for _ in range(2))
        a, b, c = spaces or [_space(x) for x in (B.qfc_attention_shared_q4_workspace_size(req, shared, h_q, cache), B.qfc_select_pages_q4_workspace_size(req, h_q, cache),
                                                 B.qfc_attention_selected_q4_workspace_size(req, h_q, cache, less))]
        B.qfc_attention_shared_q4(q[:tokens], req, shared, h_q, cache, a, one)
        B.qfc_select_pages_q4(q[:tokens], req, h_q, cache, bounds, 1, 1, selected, b)
        B.qfc_attention_selected_q4(q[:tokens], req, h_q, cache, selected, c, two)
        assert bool((selected >= 0).all()) and not bool((one == 3.0).all()) and not bool((two == 3.0).all())
        return [one, selected, two], [a, b, c]

    spaces = call(T, n, count, None)[1]
    for tokens in (40, 33, 32, 31, 20, 17, 16, 15, 5, 2, 1):
        for longest in (n, 513 * 64, 512 * 64, 3000):
            for less in (count, count - 1, 9, 4):
                for got, want in zip(call(tokens, longest, less, spaces)[0], call(tokens, longest, less, None)[0]):
                    assert torch.equal(got, want), (tokens, longest, less)


# ---------------------------------------------------------------- the oracle by hand
def test_oracle_pages_by_hand():
    table, refs, missing = ref.take(np.array([[3, -1, -1], [7, 9, -1]]), np.array([0, 1, 0, 1, 0]), [130, 64])
    assert np.array_equal(table, [[3, 0, 2], [4, 9, -1]]) and np.array_equal(refs, [1, 1, 1, 1, 1]) and missing == 0
    pages = np.arange(5)[:, None]
    table, refs, pages, missing = ref.fork(np.array([[1, 3]]), np.array([0, 1, 0, 1, 0]), [0, 0, 2, 0], [100, 64, 64, 65], 2, pages)
    assert np.array_equal(table, [[1, 0], [1, -1], [-1, -1], [1, 2]]) and np.array_equal(refs, [1, 4, 1, 1, 0]) and np.array_equal(pages[:, 0], [3, 1, 3, 3, 4]) and missing == 0
    table, refs = ref.free(table, refs, [64, 0, 5, 128])
    assert np.array_equal(table, [[1, -1], [-1, -1], [-1, -1], [1, 2]]) and np.array_equal(refs, [0, 3, 1, 1, 0])
    table, refs, pages, used = ref.compact(np.array([[1, 2], [3, 1]]), np.array([0, 2, 1, 1, 0]), np.arange(5))
    assert used == 3 and np.array_equal(table, [[1, 2], [0, 1]]) and np.array_equal(refs, [1, 2, 1, 0, 0]) and pages[0] == 3


def test_oracle_selection_by_hand():
    codes, step = ref.bounds(np.array([[1.0, -2.0], [127.0, 4.25], [-3.5, 0.0]]))
    assert np.array_equal(codes, [[127, 5], [-4, -2]]) and step == 1
    score = ref.scores(np.array([[127.0, -127.0]]), np.array([codes, codes]), np.array([1.0, 2.0]), np.array([True, True]))
    assert score[0] == 127 * 127 + 127 * 2 and score[1] == 2 * score[0]
    assert np.array_equal(ref.select(np.array([0, 5, 7, 5, 5, 0.0]), 6, 1, 1, 4), [0, 1, 2, 5])  # of equal ones the first
    assert np.array_equal(ref.select(np.zeros(3), 3, 1, 1, 5), [0, 1, 2, -1, -1])


# ---------------------------------------------------------------- pages
def _random_bounds(cache, seed):
    """Bounds of no keys, and their copies on the host."""
    b, rng = B.PageBounds(cache), np.random.default_rng(seed)
    codes, steps = rng.integers(-128, 128, tuple(b.codes.shape), dtype=np.int8), rng.random(tuple(b.steps.shape), dtype=np.float32)
    b.codes.copy_(torch.from_numpy(codes)), b.steps.copy_(torch.from_numpy(steps))
    return b, codes, steps


def _bounds_are(b, codes, steps):
    assert np.array_equal(b.codes.cpu().numpy(), codes) and np.array_equal(b.steps.cpu().numpy(), steps)


class Pool:
    """A cache with references and their copies on the host."""

    def __init__(self, num, h_kv=1, d=64, rng=None):
        self.cache = B.PagedCache(num, h_kv, d)
        self.bytes = 80 * d * h_kv
        self.pages = (rng or np.random.default_rng(3)).integers(0, 256, (num, self.bytes), dtype=np.uint8)
        self.cache.pages.copy_(torch.from_numpy(self.pages.ravel()))

    def now(self):
        return self.cache.pages.cpu().numpy().reshape(-1, self.bytes)

    def space(self, batch):
        n = B.qfc_pages_workspace_size(self.cache, batch)
        w = torch.full((n + 64,), 0xAB, dtype=torch.uint8, device=DEV)
        return w[:n], w[n:]


def _counts(rng, num, share):
    """References of a pool of which a share is in use."""
    return np.where(rng.random(num) < share, rng.integers(1, 4, num), 0).astype(np.int32)


@pytest.fixture(params=["native", "ctypes"])
def either_way(request, monkeypatch):
    """Both ways of passing arguments."""
    B.lib()
    if request.param == "ctypes":
        monkeypatch.setattr(B, "_fast", None)
    elif B._fast is None:
        pytest.skip("_marshal is not built")


@gpu
@pytest.mark.parametrize("num,batch,width,share", [(1, 1, 1, 0.0), (1, 2, 3, 1.0), (64, 3, 7, 0.5), (65, 1, 70, 0.1), (1023, 5, 130, 0.5), (1024, 4, 300, 0.9), (1025, 130, 9, 0.3), (5000, 37, 65, 0.7),
                                                   (70000, 11, 200, 0.99), (4096, 1, 5000, 0.0)])
def test_take_pages(num, batch, width, share):
    rng = np.random.default_rng(num + batch)
    pool, refs = Pool(num), _counts(rng, num, share)
    table = np.where(rng.random((batch, width)) < 0.4, rng.integers(-5, num + 5, (batch, width)), -1).astype(np.int32)
    positions = rng.integers(-3, width * 64 + 100, batch).astype(np.int32)
    positions[0] = width * 64
    want = ref.take(table, refs, positions)
    t, r, missing, (space, behind) = _i(table), _i(refs), _i([77]), pool.space(batch)
    B.qfc_take_pages(pool.cache, r, t, _i(positions), space, missing)
    assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(r.cpu().numpy(), want[1]) and int(missing) == want[2]
    assert np.array_equal(pool.now(), pool.pages) and bool((behind == 0xAB).all())
    t, r = _i(table), _i(refs)
    B.qfc_take_pages(pool.cache, r, t, _i(positions), space)
    assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(r.cpu().numpy(), want[1])


@gpu
@pytest.mark.parametrize("num,parents,children,from_width,width,share,h_kv,d", [(4, 1, 1, 1, 1, 0.5, 1, 64), (70, 3, 5, 4, 6, 0.5, 3, 64), (1500, 20, 64, 30, 20, 0.4, 2, 128),
                                                                                (3000, 7, 300, 9, 9, 0.95, 1, 256), (2100, 2, 3, 600, 700, 0.6, 8, 128)])
def test_fork_pages(num, parents, children, from_width, width, share, h_kv, d):
    rng = np.random.default_rng(num)
    pool, refs = Pool(num, h_kv, d), _counts(rng, num, share)
    used = np.flatnonzero(refs)
    source = rng.choice(used, (parents, from_width)).astype(np.int32) if used.size else np.full((parents, from_width), -1, np.int32)
    source[rng.random(source.shape) < 0.05] = rng.choice([-1, num, -7, 2 ** 30])
    of = rng.integers(0, parents, children).astype(np.int32)
    of[rng.random(children) < 0.1] = rng.choice([-1, parents])
    positions = rng.integers(0, 64 * from_width + 30, children).astype(np.int32)
    positions[rng.random(children) < 0.3] &= ~63
    want = ref.fork(source, refs, of, positions, width, pool.pages)
    f, r, missing, (space, behind) = _i(source), _i(refs), _i([77]), pool.space(children)
    t = torch.full((children, width), 123456, dtype=torch.int32, device=DEV)
    bounds, codes, steps = _random_bounds(pool.cache, 1)
    B.qfc_fork_pages(pool.cache, r, f, _i(of), _i(positions), t, space, missing, bounds)
    assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(r.cpu().numpy(), want[1]) and int(missing) == want[3]
    assert np.array_equal(pool.now(), want[2]) and np.array_equal(f.cpu().numpy(), source) and bool((behind == 0xAB).all())
    for b in range(children):  # a copied page takes its bounds along
        e = positions[b] // 64
        if 0 <= of[b] < parents and positions[b] % 64 and e < min(width, from_width) and 0 <= source[of[b], e] < num and want[0][b, e] >= 0:
            codes[want[0][b, e]], steps[want[0][b, e]] = codes[source[of[b], e]], steps[source[of[b], e]]
    _bounds_are(bounds, codes, steps)


@gpu
@pytest.mark.parametrize("batch", [4096, 4097, 5119, 5120, 5121, 9001])
def test_rows_by_the_thousand(batch):
    """What many rows lack is added up in runs of 1024."""
    test_take_pages(2 * batch, batch, 3, 0.3)
    test_take_pages(batch // 2, batch, 1, 0.1)
    test_fork_pages(batch + 500, 40, batch, 3, 4, 0.3, 1, 64)


@gpu
@pytest.mark.parametrize("num,batch,width", [(3, 1, 1), (100, 7, 33), (5000, 300, 100)])
def test_free_pages(num, batch, width):
    rng = np.random.default_rng(num)
    pool = Pool(num)
    table = np.where(rng.random((batch, width)) < 0.7, rng.integers(-2, num + 2, (batch, width)), -1).astype(np.int32)
    refs = np.bincount(table[(table >= 0) & (table < num)], minlength=num).astype(np.int32)
    keep = rng.integers(-5, 64 * width + 64, batch).astype(np.int32)
    for k in (keep, None):
        want = ref.free(table, refs, k)
        t, r = _i(table), _i(refs)
        B.qfc_free_pages(pool.cache, r, t, None if k is None else _i(k))
        assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(r.cpu().numpy(), want[1])
        assert k is not None or not r.any()


@gpu
@pytest.mark.parametrize("num,batch,width,share,h_kv,d", [(1, 1, 1, 0.0, 1, 64), (1, 1, 1, 1.0, 1, 64), (64, 3, 30, 0.5, 1, 64), (1024, 9, 200, 1.0, 1, 64), (1025, 9, 200, 0.5, 2, 64),
                                                          (3001, 50, 40, 0.03, 1, 128), (2048, 3, 900, 0.5, 1, 256), (5000, 17, 300, 0.9, 3, 64),
                                                          (16384, 30, 400, 0.5, 1, 64), (16385, 30, 400, 0.7, 1, 64), (40000, 5, 900, 0.05, 1, 64)])
def test_compact_pages(num, batch, width, share, h_kv, d):
    rng = np.random.default_rng(num)
    pool = Pool(num, h_kv, d)
    used = np.flatnonzero(rng.random(num) < share)
    table = rng.choice(used, (batch, width)).astype(np.int32) if used.size else np.full((batch, width), -1, np.int32)
    table[rng.random(table.shape) < 0.2] = -1
    table[0, 0] = num  # no page
    refs = np.bincount(table[(table >= 0) & (table < num)], minlength=num).astype(np.int32)
    want = ref.compact(table, refs, pool.pages)
    t, r, count, (space, behind) = _i(table), _i(refs), _i([-1]), pool.space(batch)
    bounds, codes, steps = _random_bounds(pool.cache, 2)
    B.qfc_compact_pages(pool.cache, r, t, space, count, bounds)
    n = want[3]
    for a, b in zip(np.flatnonzero(refs[n:] > 0) + n, np.flatnonzero(refs[:n] <= 0)):
        codes[b], steps[b] = codes[a], steps[a]
    _bounds_are(bounds, codes, steps)
    assert int(count) == n and np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(r.cpu().numpy(), want[1]) and bool((behind == 0xAB).all())
    assert np.array_equal(pool.now(), want[2])
    assert bool((r[:n] > 0).all()) and not r[n:].any()
    B.qfc_compact_pages(pool.cache, r, t, space, None)  # once more: nothing to do
    assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(pool.now(), want[2])


@gpu
@pytest.mark.parametrize("count,h_kv,d", [(1, 1, 64), (5, 3, 64), (333, 2, 128), (40, 8, 256)])
def test_copy_pages(count, h_kv, d):
    rng = np.random.default_rng(count)
    a, b = Pool(count + 7, h_kv, d, rng), Pool(count + 3, h_kv, d, rng)
    source, target = rng.permutation(count + 7)[:count].astype(np.int32), rng.permutation(count + 3)[:count].astype(np.int32)
    if count > 4:
        source[1], target[2], source[3] = -1, count + 3, count + 7
    want = b.pages.copy()
    for x, y in zip(source, target):
        if 0 <= x < count + 7 and 0 <= y < count + 3:
            want[y] = a.pages[x]
    (fb, codes_a, steps_a), (tb, codes_b, steps_b) = _random_bounds(a.cache, 3), _random_bounds(b.cache, 4)
    B.qfc_copy_pages(a.cache, b.cache, _i(source), _i(target), fb, tb)
    for x, y in zip(source, target):
        if 0 <= x < count + 7 and 0 <= y < count + 3:
            codes_b[y], steps_b[y] = codes_a[x], steps_a[x]
    _bounds_are(tb, codes_b, steps_b), _bounds_are(fb, codes_a, steps_a)
    assert np.array_equal(b.now(), want) and np.array_equal(a.now(), a.pages)
    one = a.now()
    B.qfc_copy_pages(a.cache, a.cache, _i([count + 6]), _i([0]))
    one[0] = one[count + 6]
    assert np.array_equal(a.now(), one)
    B.qfc_copy_pages(a.cache, a.cache, _i([]), _i([]))


@gpu
def test_pages_of_a_search_step_by_step(either_way):
    """Forks, frees, new pages and compactions in turn, as a search over continuations makes them; the counts are those of the tables at every step."""
    rng = np.random.default_rng(9)
    num, batch, width = 400, 12, 20
    pool = Pool(num)
    pages, refs, table, positions = pool.pages, np.zeros(num, np.int32), np.full((batch, width), -1, np.int32), rng.integers(1, 300, batch).astype(np.int32)
    r, t, (space, _) = _i(refs), _i(table), pool.space(batch)
    other = torch.empty_like(t)
    for step in range(25):
        B.qfc_take_pages(pool.cache, r, t, _i(positions), space)
        table, refs, missing = ref.take(table, refs, positions)
        assert missing == 0
        of = rng.integers(0, batch, batch).astype(np.int32)
        B.qfc_fork_pages(pool.cache, r, t, _i(of), _i(positions[of]), other, space)
        children, refs, pages, missing = ref.fork(table, refs, of, positions[of], width, pages)
        assert missing == 0
        B.qfc_free_pages(pool.cache, r, t)
        _, refs = ref.free(table, refs)
        t, other, table = other, t, children
        if step % 5 == 4:
            cut = (positions[of] // 2).astype(np.int32)  # tokens that are taken back
            B.qfc_free_pages(pool.cache, r, t, _i(cut))
            table, refs = ref.free(table, refs, cut)
            positions = np.maximum(cut, 1)
            B.qfc_compact_pages(pool.cache, r, t, space)
            table, refs, pages, _ = ref.compact(table, refs, pages)
        else:
            positions = np.minimum(positions[of] + rng.integers(1, 90, batch), width * 64).astype(np.int32)
        assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(r.cpu().numpy(), refs)
        assert np.array_equal(refs, np.bincount(table[table >= 0], minlength=num))
        assert np.array_equal(pool.now(), pages)


@gpu
def test_arguments_out_of_order_are_refused(either_way):
    """Types, shapes, orders and devices that the C calls cannot see."""
    pool = Pool(40)
    space, _ = pool.space(3)
    r, t, p, one = _i(np.zeros(40)), _i(np.full((3, 5), -1)), _i([70, 1, 0]), _i([0])
    calls = {"take": lambda r=r, t=t, p=p, w=space, m=one: B.qfc_take_pages(pool.cache, r, t, p, w, m),
             "fork": lambda r=r, t=t, p=p, w=space, m=one, f=_i(np.full((2, 5), -1)), of=_i([0, 1, 0]): B.qfc_fork_pages(pool.cache, r, f, of, p, t, w, m),
             "free": lambda r=r, t=t, p=p: B.qfc_free_pages(pool.cache, r, t, p),
             "compact": lambda r=r, t=t, w=space, m=one: B.qfc_compact_pages(pool.cache, r, t, w, m)}
    bad_table = [t.long(), t.cpu(), t[0], t.t(), t.repeat(1, 2)[:, ::2], None]
    bad_numbers = [p.long(), p.cpu(), p[:2], p.repeat(2)[::2], p[None], 5]
    bad_pool = [r.long(), r.cpu(), r[:39], r.repeat(2)[::2], None]
    for name, call in calls.items():
        call()
        for x in bad_table:
            with pytest.raises(ValueError):
                call(t=x)
        for x in bad_pool:
            with pytest.raises(ValueError):
                call(r=x)
        if name != "compact":
            for x in bad_numbers:
                with pytest.raises(ValueError):
                    call(p=x)
        if name != "free":
            for x in (space.cpu(), space.float(), None):
                with pytest.raises(ValueError):
                    call(w=x)
            for x in (one.long(), p, one.cpu()):
                with pytest.raises(ValueError):
                    call(m=x)
            with pytest.raises(B.QfcError):
                call(w=space[:16].clone())
    for x in bad_table:
        with pytest.raises(ValueError):
            calls["fork"](f=x)
    with pytest.raises(ValueError):
        calls["take"](p=None)
    other = B.PagedCache(41, 1, 64)
    with pytest.raises(ValueError):
        B.qfc_compact_pages(pool.cache, r, t, space, None, B.PageBounds(other))


@gpu
def test_pages_captured_and_replayed():
    rng = np.random.default_rng(10)
    num, batch, width = 300, 6, 9
    pool, refs = Pool(num), np.zeros(num, np.int32)
    start, refs, _ = ref.take(np.full((batch, width), -1, np.int32), refs, [300, 64, 1, 130, 500, 65])
    space, _ = pool.space(batch)
    r, t, kids = _i(refs), _i(start), _i(np.zeros((batch, width)))
    of, positions, grown = _i(np.zeros(batch)), _i(np.zeros(batch)), _i(np.zeros(batch))
    counts, tables = r.clone(), t.clone()

    def step():
        r.copy_(counts)
        t.copy_(tables)
        B.qfc_fork_pages(pool.cache, r, t, of, positions, kids, space)
        B.qfc_free_pages(pool.cache, r, t)
        B.qfc_take_pages(pool.cache, r, kids, grown, space)
        B.qfc_compact_pages(pool.cache, r, kids, space)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for k in range(4):
        parents = rng.integers(0, batch, batch).astype(np.int32)
        n = np.array([300, 64, 1, 130, 500, 65], np.int32)[parents]
        pool.cache.pages.copy_(torch.from_numpy(pool.pages.ravel()))
        of.copy_(_i(parents)), positions.copy_(_i(n)), grown.copy_(_i(n + k))
        graph.replay()
        torch.cuda.synchronize()
        table, want, pages, _ = ref.fork(start, refs, parents, n, width, pool.pages)
        _, want = ref.free(start, want)
        table, want, _ = ref.take(table, want, n + k)
        table, want, pages, _ = ref.compact(table, want, pages)
        assert np.array_equal(kids.cpu().numpy(), table) and np.array_equal(r.cpu().numpy(), want) and np.array_equal(pool.now(), pages)


@gpu
def test_layers_behind_one_table():
    """Caches of several layers, of heads of their own: the calls on copies of one table and its references give one table, and every cache holds what it names."""
    rng = np.random.default_rng(65)
    num, batch, width, kids = 900, 12, 9, 40
    order = rng.permutation(num)[:batch * 5].reshape(batch, 5)
    table = np.full((batch, width), -1, np.int32)
    table[:, :5] = order
    refs = np.bincount(order.ravel(), minlength=num).astype(np.int32)
    parents, positions = rng.integers(0, batch, kids).astype(np.int32), rng.integers(1, 320, kids).astype(np.int32)
    came_out = []
    for h_kv, d in ((1, 64), (2, 128), (1, 256)):
        pool = Pool(num, h_kv, d, np.random.default_rng(h_kv * d))
        t, r, child, used = _i(table), _i(refs), _i(np.full((kids, width), -1)), _i([0])
        space = pool.space(kids)[0]
        B.qfc_fork_pages(pool.cache, r, t, _i(parents), _i(positions), child, space)
        B.qfc_free_pages(pool.cache, r, t)
        B.qfc_take_pages(pool.cache, r, child, _i(positions + 70), space)
        B.qfc_compact_pages(pool.cache, r, child, space, used)
        kid, want, pages, _ = ref.fork(table, refs, parents, positions, width, pool.pages)
        _, want = ref.free(table, want)
        kid, want, _ = ref.take(kid, want, positions + 70)
        kid, want, pages, count = ref.compact(kid, want, pages)
        assert np.array_equal(pool.now(), pages) and int(used) == count
        came_out.append((child.cpu().numpy(), r.cpu().numpy()))
        assert np.array_equal(came_out[-1][0], kid) and np.array_equal(came_out[-1][1], want)
    assert all(np.array_equal(a, b) for x in came_out[1:] for a, b in zip(came_out[0], x))


@gpu
def test_pages_of_almost_two_gibibytes():
    """The largest page that is not refused: copied, forked and moved whole."""
    h_kv, d = (2 ** 31 - 1) // (80 * 64), 64
    cache = B.PagedCache(3, h_kv, d)
    whole = cache.pages.view(3, -1)
    assert whole.shape[1] > 2 ** 31 - 80 * 64
    words = whole.view(torch.int32)
    words[0] = torch.arange(words.shape[1], dtype=torch.int32, device=DEV) * 7 + 1
    words[1:] = -1
    B.qfc_copy_pages(cache, cache, _i([0]), _i([1]))
    assert torch.equal(words[0], words[1]) and bool((words[2] == -1).all())
    words[0] = -1
    space = _space(B.qfc_pages_workspace_size(cache, 1))
    r, table, child = _i([0, 1, 0]), _i([[1]]), _i([[7]])
    B.qfc_compact_pages(cache, r, table, space)
    assert torch.equal(words[0], words[1]) and bool((words[2] == -1).all()) and r.tolist() == [1, 0, 0] and table.tolist() == [[0]]
    words[1] = -1
    B.qfc_fork_pages(cache, r, table, _i([0]), _i([5]), child, space)
    assert torch.equal(words[0], words[1]) and bool((words[2] == -1).all()) and r.tolist() == [1, 1, 0] and child.tolist() == [[1]]


# ---------------------------------------------------------------- attention behind common pages
def _attend_shared(req, shared, q, h_q, cache, fill=0.0):
    out = torch.full((q.shape[0], h_q * cache.d_head), fill, dtype=torch.float16, device=DEV)
    n = B.qfc_attention_shared_q4_workspace_size(req, shared, h_q, cache)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=DEV)  # (NaN in what is read without having been written)
    B.qfc_attention_shared_q4(_t(q), req, shared, h_q, cache, ws[:n], out)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xFF).all())
    return out.cpu().numpy().astype(np.float64)


def _shared_batch(rng, group, prefix, S, n, h_kv, d):
    """A cache and a table in which the requests of each group share prefix // 64 pages; K, V and V's parts per request."""
    lead = np.arange(len(S))
    whole = np.zeros(len(S), int)
    for i, p in enumerate(prefix):
        first = group[i]
        for b in range(group[i], group[i + 1]):
            lead[b], whole[b] = first, p // 64
    for b in range(len(S)):
        whole[b] = min(whole[b], (n[b] - S[b]) // 64 if S[b] else n[b] // 64, n[lead[b]] // 64)
    table, num = _pages(rng, n)
    k, v = [_normal(rng, x, h_kv, d) for x in n], [_normal(rng, x, h_kv, d) for x in n]
    for b in range(len(S)):
        if lead[b] != b:
            table[b, :whole[b]] = table[lead[b], :whole[b]]
            k[b][:64 * whole[b]], v[b][:64 * whole[b]] = k[lead[b]][:64 * whole[b]], v[lead[b]][:64 * whole[b]]
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num, np.concatenate(k), np.concatenate(v))
    return cache, table, K, V, P


SHARED = [  # group_start, positions, S, n, h_q, h_kv, d
    ([0, 1], [64], [1], [65], 1, 1, 64),
    ([0, 2], [128], [1, 1], [129, 300], 4, 1, 128),
    ([0, 3], [700], [1, 1, 1], [701, 800, 1000], 8, 2, 64),
    ([0, 2, 5], [200, 64], [1, 2, 1, 4, 1], [300, 202, 70, 100, 65], 8, 4, 256),
    ([1, 3], [130], [1, 1, 1, 2], [40, 131, 200, 500], 4, 2, 128),           # requests in front of the groups and behind them
    ([0, 0, 2, 2, 4], [64, 320, 640, 70], [1, 1, 1, 1], [400, 321, 71, 200], 2, 2, 128),  # groups without requests
    ([0, 4], [256], [0, 1, 0, 3], [256, 300, 900, 260], 6, 2, 64),           # a first request without tokens
    ([0, 3], [1000], [1, 1, 1], [1100, 200, 64], 4, 1, 128),                 # more positions than two of the requests have: cut
    ([0, 2], [50], [1, 1], [100, 90], 4, 4, 64),                             # less than a page
    ([0, 40], [2000], [1] * 40, [2001 + 3 * i for i in range(40)], 8, 2, 128),
    ([0, 3], [512], [30, 1, 70], [600, 513, 800], 4, 2, 128),                # prompts
    ([0, 2], [320], [1, 1], [400, 333], 40, 2, 64),                          # 20 heads on one
    ([0, 100], [192], [1] * 100, [193 + i for i in range(100)], 4, 1, 256),
    ([0, 70], [3000], [1] * 70, [3001] * 70, 16, 2, 64),
    ([0, 7, 80, 81], [640, 1300, 70], [1 + i % 3 for i in range(81)], [1310 + i for i in range(81)], 3, 1, 128),
]


@pytest.fixture(params=["few", "many"])
def rows_rule(request):
    """Both paths for common pages, whatever the sizes."""
    B.qfc_tune(16, 1 << 30 if request.param == "few" else 1)
    yield request.param
    B.qfc_tune(16, 0)


@gpu
@pytest.mark.parametrize("group,prefix,S,n,h_q,h_kv,d", SHARED)
def test_attention_shared(group, prefix, S, n, h_q, h_kv, d, rows_rule):
    rng = np.random.default_rng(21)
    cache, table, K, V, P = _shared_batch(rng, group, prefix, S, n, h_kv, d)
    T, behind = sum(S), 3
    q = _normal(rng, T + behind, h_q * d)
    req = _requests(S, n, table, rows=T + behind)
    sizes = np.concatenate([[0], np.cumsum(S)])
    most = max(max(int(sizes[group[i + 1]] - sizes[group[i]]) for i in range(len(prefix))), 1)
    shared = B.SharedPrefixes(_i(group), _i(prefix), most, max(prefix))
    got = _attend_shared(req, shared, q, h_q, cache, fill=7.0)
    assert np.all(got[T:] == 7.0)
    got, at = got.reshape(-1, h_q, d), 0
    for b, s in enumerate(S):
        _close(got[at:at + s], *q4.attention(q.reshape(-1, h_q, d)[at:at + s], K[b], V[b], P[b]))
        at += s
    # limits far above what is there
    loose = B.Requests(req.token_start, req.context, _i(np.pad(table, ((0, 0), (0, 40)), constant_values=-1)), T + behind, max(S) + 5, max(n) + 2000)
    got = _attend_shared(loose, B.SharedPrefixes(_i(group), _i(prefix), most + 100, max(prefix) + 3000), q, h_q, cache, fill=7.0).reshape(-1, h_q, d)
    at = 0
    for b, s in enumerate(S):
        _close(got[at:at + s], *q4.attention(q.reshape(-1, h_q, d)[at:at + s], K[b], V[b], P[b]))
        at += s


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
def test_attention_shared_extremes(rows_rule, d):
    """Pages that are missing, in the common part and behind it; a request that sees nothing; queries that are infinite or no numbers stay their own rows' matter; steps of 2 and more."""
    rng = np.random.default_rng(22)
    group, prefix, S, n, h_q, h_kv = [0, 3], [320], [1, 1, 1, 1], [400, 500, 330, 0], 4, 2
    cache, table, K, V, P = _shared_batch(rng, group, prefix, S[:3], n[:3], h_kv, d)
    table = np.pad(table, ((0, 1), (0, 0)), constant_values=-1)
    table[:3, 2] = -1
    table[1, 6] = 1 << 30
    q = _normal(rng, 4, h_q * d)
    req, shared = _requests(S, n, table), B.SharedPrefixes(_i(group), _i(prefix), 4, 320)
    got = _attend_shared(req, shared, q, h_q, cache).reshape(-1, h_q, d)
    for b in range(3):
        there = np.ones(n[b], bool)
        there[128:192] = False
        if b == 1:
            there[384:448] = False
        _close(got[b:b + 1], *q4.attention(q.reshape(-1, h_q, d)[b:b + 1], K[b], V[b], P[b], there))
    assert np.all(got[3] == 0)
    bad = q.copy()
    bad[0, :d] = np.nan
    bad[2, d:2 * d] = np.inf
    again = _attend_shared(req, shared, bad, h_q, cache).reshape(-1, h_q, d)
    assert np.all(np.isnan(again[0, 0])) and np.all(np.isnan(again[2, 1]))
    for b, h in ((0, 1), (0, 2), (0, 3), (1, 0), (1, 1), (1, 2), (1, 3), (2, 0), (2, 2), (2, 3)):
        assert np.array_equal(again[b, h], got[b, h])
    # values far apart: steps of 2 and more in some pages
    S, n = [1, 1, 1], [400, 500, 330]
    table, num = _pages(rng, n)
    table[1, :5], table[2, :5] = table[0, :5], table[0, :5]
    v = _normal(rng, sum(n), h_kv, d)
    v[::7] *= np.float16(300)
    k = _normal(rng, sum(n), h_kv, d)
    for b, at in ((1, 400), (2, 900)):
        k[at:at + 320], v[at:at + 320] = k[:320], v[:320]
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num, k, v)
    got = _attend_shared(_requests(S, n, table), shared, q[:3], h_q, cache).reshape(-1, h_q, d)
    for b in range(3):
        _close(got[b:b + 1], *q4.attention(q.reshape(-1, h_q, d)[b:b + 1], K[b], V[b], P[b]))


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rise", [0.3, 1.0, 2.0, 2.9, 3.1, -1.0])
def test_attention_shared_maxima_that_move(d, rise, rows_rule):
    """Scores that rise (or fall) from page to page by so many units of log 2, for some rows and not for others: what may lag behind the largest one does so by a bounded amount."""
    rng = np.random.default_rng(24)
    group, prefix, S, h_q, h_kv = [0, 5], [64 * 9], [1] * 5, 2, 1
    n = [64 * 9 + 1 + 7 * i for i in range(5)]
    table, num = _pages(rng, n)
    k, v = _normal(rng, sum(n), h_kv, d) * np.float16(0.25), _normal(rng, sum(n), h_kv, d)
    q = _normal(rng, 5, h_q * d)
    q[:, ::d] = np.array([[0.0, 8.0], [8.0, -8.0], [4.0, 2.0], [8.0, 8.0], [-8.0, 1.0]], dtype=np.float16)
    at = np.cumsum([0] + n[:-1])
    for b in range(5):
        k[at[b]:at[b] + n[b], 0, 0] = (np.arange(n[b]) // 64 * rise * np.log(2.0) * np.sqrt(d) / 8.0).astype(np.float16)
        k[at[b]:at[b] + n[b], 0, 1:32] *= np.float16(0.1)
    for b in range(1, 5):
        table[b, :9] = table[0, :9]
        k[at[b]:at[b] + 576], v[at[b]:at[b] + 576] = k[:576], v[:576]
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num, k, v)
    got = _attend_shared(_requests(S, n, table), B.SharedPrefixes(_i(group), _i(prefix), 5, 576), q, h_q, cache).reshape(-1, h_q, d)
    for b in range(5):
        _close(got[b:b + 1], *q4.attention(q.reshape(-1, h_q, d)[b:b + 1], K[b], V[b], P[b]))


def _check_shared_alike(rng, S, n, d, k, v, q):
    """Requests of n[b] positions, all but the last few of each in common pages that hold k, v (one KV head); q [tokens, heads, d]."""
    whole = len(k) // 64
    table, num = _pages(rng, n)
    table[1:, :whole] = table[0, :whole]
    own = lambda x, b: np.concatenate([x[:64 * whole], _normal(rng, n[b] - 64 * whole, 1, d) * np.float16(2.0 ** -10)])
    cache, K, V, P = _filled(rng, n, 1, d, table, num, np.concatenate([own(k, b) for b in range(len(n))]), np.concatenate([own(v, b) for b in range(len(n))]))
    got = _attend_shared(_requests(S, n, table), B.SharedPrefixes(_i([0, len(S)]), _i([len(k)]), sum(S), len(k)), q.reshape(sum(S), -1), q.shape[1], cache).reshape(q.shape)
    at = 0
    for b, s in enumerate(S):
        _close(got[at:at + s], *q4.attention(q[at:at + s], K[b], V[b], P[b]))
        at += s


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n,where,value,small,gap", [(1000, 100, 40, 0.05, 12), (1000, 100, 40, 0.005, 12), (8000, 100, 30.5, 0.01, 16), (8000, 70, 4000, 0.005, 12), (1000, 64, 60000, 0.01, 14),
                                                     (1000, 950, 60000, 0.01, 14), (448, 0, 300, 0.02, 12), (1000, 100, 20, 0.005, 12)])
def test_attention_shared_large_value_beside_small_ones(n, where, value, small, gap, d, rows_rule):
    """One large value in one group of 32, groups of small ones beside it, and a position with nearly all of P whose values are next to nothing: the others make up the result.  (Products of P and
    a step that are denormals of binary16 are off by 2^-25 of 2^14, times a code of 8: 2^-36 a position, either way, nothing against the bound's 2^-24.)"""
    rng = np.random.default_rng(59)
    base, k, v = _normal(rng, d), _normal(rng, n, 1, d), _normal(rng, n, 1, d)
    k[5, 0] = base * np.float16(gap * np.sqrt(d) / np.sum(base.astype(np.float64) ** 2))
    v[:, :, 32:] *= np.float16(small)
    v[5] *= np.float16(1e-3)
    v[where, 0, 3] = value
    q = np.stack([base * np.float16(x) for x in (1.0, 0.9, 1.1, 1.0, 0.95, 1.05, 0.97, 1.02)]).reshape(4, 2, d)
    _check_shared_alike(rng, [1, 2, 1], [n + 3, n + 70, n + 5], d, k, v, q)


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [0, 3, 8])
@pytest.mark.parametrize("value,far", [(30000, 30), (60000, 24), (60000, 11), (35, 30)])
def test_attention_shared_page_of_large_steps_that_hardly_counts(value, far, page, d, rows_rule):
    """A page with steps of 2 and more and 2^-far of the largest P, and pages of small steps whose positions, all alike, have 2^-10 of it: their products with P round all the same way, once."""
    rng = np.random.default_rng(60)
    n = 640
    unit = np.log(2.0) * np.sqrt(d) / 8.0  # of q . k, with 8 in the query
    k, v = np.zeros((n, 1, d), np.float16), np.zeros((n, 1, d), np.float16)
    k[64 * page:64 * page + 64, 0, 0] = -(far - 10) * unit
    k[5 if page else 300, 0, 0] = 10 * unit
    v[:, 0, :] = np.tile(np.linspace(-2.0 ** -5, 2.0 ** -5, 32).astype(np.float16), d // 32)
    v[5 if page else 300] *= np.float16(2.0 ** -6)
    v[64 * page:64 * page + 64, 0, 1::2] = value
    q = np.zeros((3, 2, d), np.float16)
    q[:, :, 0] = 8
    _check_shared_alike(rng, [1, 1, 1], [n + 1, n + 2, n + 100], d, k, v, q)


@gpu
def test_attention_shared_by_its_own_rule():
    """Sizes at which the rule, and not the tunable, takes the way of many rows: the same result, and large values beside small ones."""
    rng = np.random.default_rng(61)
    requests, h_q, h_kv, d, whole = 64, 32, 8, 128, 620
    n = [64 * whole + 1 + 5 * b for b in range(requests)]
    table = np.full((requests, whole + 6), -1, np.int32)
    table[:, :whole] = rng.permutation(whole)
    at = whole
    for b, x in enumerate(n):
        own = (x + 63) // 64 - whole
        table[b, whole:whole + own] = np.arange(at, at + own)
        at += own
    cache = B.PagedCache(at, h_kv, d)
    k, v = _normal(rng, at * 64, h_kv, d), _normal(rng, at * 64, h_kv, d)
    v[:, :, 32:64] *= np.float16(0.005)
    v[4000, :, 40] = 40
    K, _ = q4.q4_values(*q4.q4(k))
    V, P = q4.q4_values(*q4.q4(v))
    every = _requests([at * 64], [at * 64], np.arange(at, dtype=np.int32)[None])
    B.qfc_append_q4(_t(np.concatenate([k, k, v], 1).reshape(at * 64, -1)), every, h_kv, None, None, cache, torch.empty((at * 64, h_kv * d), dtype=torch.float16, device=DEV))
    q = _normal(rng, requests, h_q * d)
    req = _requests([1] * requests, n, table)
    out = _attend_shared(req, B.SharedPrefixes(_i([0, requests]), _i([64 * whole]), requests, 64 * whole), q, h_q, cache).reshape(requests, h_q, d)
    paged = lambda x, b: x.reshape(at, 64, h_kv, d)[table[b, :(n[b] + 63) // 64]].reshape(-1, h_kv, d)[:n[b]]
    for b in (0, 31, 63):
        _close(out[b:b + 1], *q4.attention(q.reshape(requests, h_q, d)[b:b + 1], paged(K, b), paged(V, b), paged(P, b)))


@gpu
@pytest.mark.parametrize("most", [9, 300, 1 << 20, 2 ** 31 - 1])
def test_attention_shared_limits_far_above_the_call_change_nothing(most):
    """What a group may have is not what the call has: the same way is taken, and the same bits come out."""
    rng = np.random.default_rng(62)
    group, prefix, S, n, h_q, h_kv, d = [0, 8], [1300], [1] * 8, [1301 + 9 * i for i in range(8)], 8, 2, 128
    cache, table, K, V, P = _shared_batch(rng, group, prefix, S, n, h_kv, d)
    q, req = _normal(rng, 8, h_q * d), _requests(S, n, table)
    want = _attend_shared(req, B.SharedPrefixes(_i(group), _i(prefix), 8, 1300), q, h_q, cache)
    assert np.array_equal(_attend_shared(req, B.SharedPrefixes(_i(group), _i(prefix), most, 2 ** 31 - 1), q, h_q, cache), want)
    for b in range(8):
        _close(want.reshape(8, h_q, d)[b:b + 1], *q4.attention(q.reshape(8, h_q, d)[b:b + 1], K[b], V[b], P[b]))


@gpu
def test_attention_shared_arrays_that_break_the_rules_stay_inside(rows_rule):
    rng = np.random.default_rng(23)
    group, prefix, S, n, h_q, h_kv, d = [0, 3], [320], [1, 1, 1], [400, 500, 330], 4, 2, 64
    cache, table, K, V, P = _shared_batch(rng, group, prefix, S, n, h_kv, d)
    q = _normal(rng, 8, h_q * d)
    for g, p in (([5, -3], [1 << 30]), ([0, 1 << 30], [-5]), ([2, 1], [320]), ([-9, 2], [2 ** 31 - 1])):
        for start in ([0, 1, 2, 3], [0, 1 << 30, -4, 2], [3, 2, 1, 0]):
            req = B.Requests(_i(start), _i([2 ** 31 - 1, -5, 330]), _i(table), 8, 2, 500)
            out = torch.full((10, h_q * d), 9.0, dtype=torch.float16, device=DEV)
            shared = B.SharedPrefixes(_i(g), _i(p), 3, 330)
            ws = torch.zeros(B.qfc_attention_shared_q4_workspace_size(req, shared, h_q, cache) + 64, dtype=torch.uint8, device=DEV)
            B.qfc_attention_shared_q4(_t(q), req, shared, h_q, cache, ws[:-64], out[:8])
            assert bool((out[8:] == 9.0).all()) and not ws[-64:].any()


# ---------------------------------------------------------------- bounds and selection
def _bounds_of(K, n, h_kv, d):
    pages = (n + 63) // 64
    codes, steps = np.zeros((pages, h_kv, 2, d), np.int8), np.zeros((pages, h_kv), np.float32)
    for p in range(pages):
        for kv in range(h_kv):
            codes[p, kv], steps[p, kv] = ref.bounds(K[64 * p:min(n, 64 * p + 64), kv])
    return codes, steps


@gpu
@pytest.mark.parametrize("S,n,h_kv,d", [([1], [1], 1, 64), ([1, 1], [64, 65], 2, 128), ([3, 0, 1], [66, 40, 500], 3, 256), ([130, 1, 64], [130, 200, 128], 2, 64), ([66], [129], 1, 128), ([2], [65], 8, 128),
                                        ([300, 7], [1000, 7], 4, 256)])
def test_bound_pages(S, n, h_kv, d):
    rng = np.random.default_rng(31)
    table, num = _pages(rng, n)
    k = _normal(rng, sum(n), h_kv, d)
    k[0] = 0
    k[-1] *= np.float16(100)
    if sum(n) > 300:
        k[100:200] *= np.float16(2.0 ** -12)
    cache, K, _, _ = _filled(rng, n, h_kv, d, table, num, k)
    bounds = B.PageBounds(cache)
    bounds.codes.fill_(99), bounds.steps.fill_(-5.0)
    B.qfc_bound_pages_q4(_requests(S, n, table), cache, bounds)
    codes, steps = bounds.codes.cpu().numpy(), bounds.steps.cpu().numpy()
    touched = set()
    for b in range(len(S)):
        want = _bounds_of(K[b], n[b], h_kv, d)
        for p in range((n[b] - S[b]) // 64, (n[b] - 1) // 64 + 1) if S[b] else ():
            page = table[b, p]
            touched.add(int(page))
            assert np.array_equal(codes[page], want[0][p]) and np.array_equal(steps[page], want[1][p]), (b, p)
    for page in set(range(num)) - touched:
        assert np.all(codes[page] == 99) and np.all(steps[page] == -5.0)


SELECT = [  # S, n, h_q, h_kv, d, first, last, count
    ([1], [1], 1, 1, 64, 0, 1, 1),
    ([1], [640], 4, 1, 128, 1, 1, 4),
    ([1, 1], [641, 100], 8, 2, 64, 0, 0, 3),
    ([3, 1], [400, 1500], 2, 2, 256, 1, 2, 5),
    ([1], [3000], 40, 2, 64, 2, 3, 10),      # 20 heads on one
    ([70, 0, 2], [900, 5, 70], 3, 1, 128, 0, 1, 7),
    ([1], [20000], 4, 4, 64, 1, 1, 100),
    ([1], [64 * 1026], 4, 4, 64, 1, 1, 500),  # 1024 to choose from
    ([2], [64 * 2049], 2, 1, 64, 0, 1, 7),   # 2047 and 2048
    ([1], [64 * 2051], 2, 1, 64, 1, 1, 900),
    ([1], [40000], 2, 1, 64, 0, 1, 600),
    ([1, 1], [1000, 2000], 4, 2, 64, 5, 4, 9),  # nothing left to choose
    ([2], [200], 4, 2, 128, 0, 1, 50),       # fewer pages than asked for
]


def _select(req, q, h_q, cache, bounds, first, last, count, T):
    selected = torch.full((T, cache.h_kv, count), 12345, dtype=torch.int32, device=DEV)
    B.qfc_select_pages_q4(_t(q), req, h_q, cache, bounds, first, last, selected, _space(B.qfc_select_pages_q4_workspace_size(req, h_q, cache)))
    return selected


@gpu
@pytest.mark.parametrize("S,n,h_q,h_kv,d,first,last,count", SELECT)
@pytest.mark.parametrize("alike", [False, True])
def test_select_pages(S, n, h_q, h_kv, d, first, last, count, alike):
    """alike: pages that repeat, so that many scores are equal."""
    rng = np.random.default_rng(41)
    table, num = _pages(rng, n)
    k = _normal(rng, sum(n), h_kv, d)
    if alike:
        k = np.tile(_normal(rng, 192, h_kv, d), (sum(n) // 192 + 1, 1, 1))[:sum(n)]
    cache, K, _, _ = _filled(rng, n, h_kv, d, table, num, k)
    bounds = B.PageBounds(cache)
    B.qfc_bound_pages_q4(_requests(n, n, table), cache, bounds)
    if n[0] > 700:
        table[0, 3] = -1  # an entry without a page
    T = sum(S) + 2
    q = _normal(rng, T, h_q * d)
    q[0, :d] = 0
    req = _requests(S, n, table, rows=T)
    got = _select(req, q, h_q, cache, bounds, first, last, count, T).cpu().numpy()
    # the same with scores in the workspace: limits above what a workgroup has at once, and above what fits the LDS
    for limit in (3000, 33000):
        wide = np.full((len(n), limit), -1, np.int32)
        wide[:, :table.shape[1]] = table
        far = B.Requests(req.token_start, req.context, _i(wide), T, max(S), limit * 64)
        assert np.array_equal(_select(far, q, h_q, cache, bounds, first, last, count, T).cpu().numpy(), got)
    at, g = 0, h_q // h_kv
    for b, s in enumerate(S):
        codes, steps = _bounds_of(K[b], n[b], h_kv, d)
        there = table[b, :len(steps)] >= 0
        for i in range(s):
            sees = (n[b] - s + i) // 64 + 1
            for kv in range(h_kv):
                rows = q[at + i].reshape(h_q, d)[kv * g:(kv + 1) * g]
                want = ref.select(ref.scores(rows, codes[:, kv], steps[:, kv], there), sees, first, last, count)
                assert np.array_equal(got[at + i, kv], want), (b, i, kv)
        at += s
    assert np.all(got[at:] == 12345)


@gpu
@pytest.mark.parametrize("pages,count", [(40, 7), (130, 11), (130, 99), (300, 50), (514, 3), (700, 33), (1030, 600), (2050, 77), (4000, 1234), (16400, 333), (33000, 2000)])
def test_select_pages_whose_scores_are_close(pages, count):
    """Scores that are neighbours among the numbers of 32 bits, or some of them far off: every step of the search for the last one's place decides."""
    d, h = 64, 2
    rng = np.random.default_rng(pages + count)
    cache = B.PagedCache(pages, h, d)
    b = B.PageBounds(cache)
    codes = np.zeros((pages, h, 2, d), np.int8)
    codes[:, :, 0, 0], codes[:, :, 1, 0] = 127, -127
    i = np.stack([rng.permutation(pages), rng.integers(0, max(pages // 3, 2), pages)])
    q = np.zeros((2, d), np.float16)
    q[0, 0], q[1, 0] = 1, 1
    table = rng.permutation(pages).astype(np.int32)[None]
    n = pages * 64
    req = _requests([1], [n], table)
    for far in (0.0, 0.1, 0.9):
        steps = (1.5 + i * 2.0 ** -23).astype(np.float32)
        steps = np.where(rng.random((2, pages)) < far, rng.random((2, pages), dtype=np.float32) * np.float32(4), steps).T
        b.codes.copy_(torch.from_numpy(codes)), b.steps.copy_(torch.from_numpy(np.ascontiguousarray(steps)))
        for limit in sorted({pages, max(pages, 3000), 33000}):  # scores in the LDS, or in the workspace
            wide = np.full((1, limit), -1, np.int32)
            wide[:, :pages] = table
            far_off = B.Requests(req.token_start, req.context, _i(wide), 1, 1, limit * 64)
            got = _select(far_off, q.reshape(1, -1), 2, cache, b, 1, 1, count, 1).cpu().numpy()[0]
            for kv in range(2):
                score = ref.scores(q[kv:kv + 1], codes[table[0], kv], steps[table[0], kv], np.ones(pages, bool))
                assert np.array_equal(got[kv], ref.select(score, pages, 1, 1, count)), (far, limit, kv)


@gpu
def test_a_page_scores_at_least_what_its_keys_do():
    """What the bounds are for: up to the rounding of the query (half a code of each of d components, against bounds of 127 steps) no key scores above its page."""
    rng = np.random.default_rng(42)
    n, h_kv, d = [1500], 2, 128
    table, num = _pages(rng, n)
    cache, K, _, _ = _filled(rng, n, h_kv, d, table, num)
    codes, steps = _bounds_of(K[0], n[0], h_kv, d)
    q = _normal(rng, 1, h_kv * d).reshape(h_kv, d)
    for kv in range(h_kv):
        score = ref.scores(q[kv:kv + 1], codes[:, kv], steps[:, kv], np.ones(len(steps), bool))
        best = np.array([(K[0][64 * p:64 * p + 64, kv] @ q[kv].astype(np.float64)).max() for p in range(len(steps))])
        slack = 0.5 * np.abs(q[kv].astype(np.float64)).max() / 127 * d * 127 * steps[:, kv]
        assert np.all(best <= score + slack)


# ---------------------------------------------------------------- attention over selected pages
def _attend_selected(req, q, h_q, cache, selected, fill=0.0):
    out = torch.full((q.shape[0], h_q * cache.d_head), fill, dtype=torch.float16, device=DEV)
    n = B.qfc_attention_selected_q4_workspace_size(req, h_q, cache, selected.shape[2])
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    B.qfc_attention_selected_q4(_t(q), req, h_q, cache, selected, ws[:n], out)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xFF).all())
    return out.cpu().numpy().astype(np.float64)


SOME = [  # S, n, h_q, h_kv, d, count
    ([1], [1], 1, 1, 64, 1),
    ([1], [640], 4, 1, 128, 3),
    ([1, 1], [641, 100], 8, 2, 64, 5),
    ([3, 1], [400, 1500], 2, 2, 256, 6),
    ([1], [3000], 40, 2, 64, 17),
    ([70, 0, 2], [900, 5, 70], 3, 1, 128, 7),
    ([1], [9000], 32, 8, 128, 70),
    ([1] * 40, [300 + 10 * i for i in range(40)], 8, 4, 256, 4),
    ([130], [600], 4, 2, 64, 8),
    ([1], [900], 32, 8, 128, 8),             # eight wavefronts, a page each
    ([2], [700], 6, 2, 256, 5),
    ([1] * 30, [1300 + i for i in range(30)], 32, 8, 64, 20),  # eight wavefronts, some pages each
    ([1] * 62, [590 + i for i in range(62)], 32, 4, 128, 9),
    ([1] * 62, [590 + i for i in range(62)], 8, 4, 256, 9),
    ([100], [200], 7, 7, 64, 3),             # and three lists one after the other
]


@gpu
@pytest.mark.parametrize("S,n,h_q,h_kv,d,count", SOME)
def test_attention_selected(S, n, h_q, h_kv, d, count):
    rng = np.random.default_rng(51)
    table, num = _pages(rng, n)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num)
    T, behind, g = sum(S), 2, h_q // h_kv
    q = _normal(rng, T + behind, h_q * d)
    req = _requests(S, n, table, rows=T + behind)
    selected = np.full((T + behind, h_kv, count), -1, np.int32)
    at = 0
    for b, s in enumerate(S):
        for i in range(s):
            sees = (n[b] - s + i) // 64 + 1
            for kv in range(h_kv):
                pick = rng.permutation(sees)[:rng.integers(0, min(sees, count) + 1)]
                selected[at + i, kv, rng.permutation(count)[:len(pick)]] = pick  # any order, -1 in between
                if rng.random() < 0.2 and len(pick) < count:
                    selected[at + i, kv, np.flatnonzero(selected[at + i, kv] < 0)[0]] = rng.choice([sees + 1, 2 ** 31 - 1, -2 ** 31])  # pages that it does not see
        at += s
    got = _attend_selected(req, q, h_q, cache, _i(selected), fill=5.0)
    assert np.all(got[T:] == 5.0)
    got, at = got.reshape(-1, h_q, d), 0
    for b, s in enumerate(S):
        for i in range(s):
            m = n[b] - s + i + 1
            for kv in range(h_kv):
                there = np.isin(np.arange(m) // 64, selected[at + i, kv])
                heads = slice(kv * g, (kv + 1) * g)
                rows = q[at + i].reshape(1, h_q, d)[:, heads]
                _close(got[at + i:at + i + 1, heads], *q4.attention(rows, K[b][:m, kv:kv + 1], V[b][:m, kv:kv + 1], P[b][:m, kv:kv + 1], there))
        at += s


@gpu
@pytest.mark.parametrize("h_q,h_kv,d", [(2, 1, 64), (8, 1, 64), (9, 1, 64), (8, 2, 128), (5, 1, 128), (4, 2, 256), (3, 1, 256), (17, 1, 256)])
@pytest.mark.parametrize("values", ["steps of 2 and more", "far from zero", "one of them large", "infinite and no queries"])
def test_attention_selected_extremes(h_q, h_kv, d, values):
    """On both sides of the number of heads that are spread over the groups of values."""
    rng = np.random.default_rng(53)
    S, n, g = [1, 2], [500, 700], h_q // h_kv
    table, num = _pages(rng, n)
    k, v, q = _normal(rng, sum(n), h_kv, d), _normal(rng, sum(n), h_kv, d), _normal(rng, 3, h_q * d)
    if values == "steps of 2 and more":
        v[::3] *= np.float16(300)
        v[::7, :, 32:64] *= np.float16(20)
    elif values == "far from zero":
        v += np.float16(1000)
        k += np.float16(20)
    elif values == "one of them large":
        v[:, :, 5] = 60000
        k[40, :, :] = q.reshape(3, h_q, d)[0, 0]
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num, k, v)
    picks = [np.arange(8), np.array([0, 3, 4, 6, 7, 8, 9, 10]), np.array([10, 2, 1, 0, 5, 6, 7, 8])]
    selected = np.repeat(np.stack(picks)[:, None], h_kv, 1).astype(np.int32)
    if values == "infinite and no queries":
        want = _attend_selected(_requests(S, n, table), q, h_q, cache, _i(selected)).reshape(3, h_q, d)
        bad = q.copy().reshape(3, h_q, d)
        bad[0, 0, 3], bad[1, h_q - 1, d - 1] = np.nan, np.inf
        got = _attend_selected(_requests(S, n, table), bad.reshape(3, -1), h_q, cache, _i(selected)).reshape(3, h_q, d)
        assert np.all(np.isnan(got[0, 0])) and np.all(np.isnan(got[1, h_q - 1]))
        keep = np.ones((3, h_q), bool)
        keep[0, 0] = keep[1, h_q - 1] = False
        assert np.array_equal(got[keep], want[keep])
        return
    got = _attend_selected(_requests(S, n, table), q, h_q, cache, _i(selected)).reshape(3, h_q, d)
    for t, (b, m) in enumerate(((0, 500), (1, 699), (1, 700))):
        there = np.isin(np.arange(m) // 64, picks[t])
        _close(got[t:t + 1], *q4.attention(q.reshape(3, h_q, d)[t:t + 1], K[b][:m], V[b][:m], P[b][:m], there))


BROKEN = [  # token_start, context
    ([0, 1, 2, 3], [2 ** 31 - 1, -5, 330]), ([0, 1 << 30, -4, 2], [400, 500, 330]), ([3, 2, 1, 0], [400, 2 ** 31 - 1, 330]), ([0, 5, 5, 8], [400, 500, 330]), ([0, 8, 8, 8], [3, 2, 1]),
    ([-9, 4, 9, 1 << 30], [-2 ** 31, 500, 500]), ([0, 3, 1, 8], [400, 500, 330]), ([6, 2 ** 31 - 1, 0, 7], [1, 500, 0]),
]


@gpu
@pytest.mark.parametrize("start,context", BROKEN)
@pytest.mark.parametrize("limit", [8, 600])  # pages: scores in one launch, in two
def test_bounds_and_selection_with_arrays_that_break_the_rules_stay_inside(start, context, limit):
    rng = np.random.default_rng(52)
    n, h_q, h_kv, d, T, count = [400, 500, 330], 4, 2, 64, 8, 5
    table, num = _pages(rng, n)
    cache, _, _, _ = _filled(rng, n, h_kv, d, table, num)
    table = np.pad(table, ((0, 0), (0, limit - table.shape[1])), constant_values=-1)
    table[1, 3], table[0, 2] = 2 ** 31 - 1, num
    for longest in (500, 64 * limit):
        req = B.Requests(_i(start), _i(context), _i(table), T, 2, min(longest, 64 * limit))
        b = B.PageBounds(cache)
        codes, steps = torch.full((b.codes.numel() + 512,), 7, dtype=torch.int8, device=DEV), torch.full((b.steps.numel() + 64,), 2.0, device=DEV)
        b.desc.codes, b.desc.steps = codes.data_ptr() + 256, steps.data_ptr() + 128
        B.qfc_bound_pages_q4(req, cache, b)
        lists = torch.full((T + 2, h_kv, count), 99, dtype=torch.int32, device=DEV)
        size = B.qfc_select_pages_q4_workspace_size(req, h_q, cache)
        ws = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        B.qfc_select_pages_q4(_t(_normal(rng, T, h_q * d)), req, h_q, cache, b, 1, 1, lists[1:-1], ws[:size])
        assert bool((codes[:256] == 7).all()) and bool((codes[-256:] == 7).all()) and bool((steps[:32] == 2).all()) and bool((steps[-32:] == 2).all())
        assert bool((lists[0] == 99).all()) and bool((lists[-1] == 99).all()) and bool((ws[size:] == 0xFF).all())
        inside = lists[1:-1][lists[1:-1] != 99]
        assert bool(((inside >= -1) & (inside < limit)).all())


@gpu
@pytest.mark.parametrize("start,context", BROKEN)
@pytest.mark.parametrize("count", [4, 17])  # lists whole, lists cut
def test_attention_selected_with_arrays_that_break_the_rules_stays_inside(start, context, count):
    rng = np.random.default_rng(53)
    n, h_q, h_kv, d, T = [400, 500, 330], 4, 2, 64, 8
    table, num = _pages(rng, n)
    cache, _, _, _ = _filled(rng, n, h_kv, d, table, num)
    table[1, 3], table[0, 2] = 2 ** 31 - 1, num
    selected = rng.integers(-3, 12, (T, h_kv, count)).astype(np.int32)
    selected[:, :, 1], selected[:, :, 2] = 2 ** 31 - 1, -2 ** 31
    req = B.Requests(_i(start), _i(context), _i(table), T, 2, 500)
    size = B.qfc_attention_selected_q4_workspace_size(req, h_q, cache, count)
    ws = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full((T + 2, h_q * d), 9.0, dtype=torch.float16, device=DEV)
    B.qfc_attention_selected_q4(_t(_normal(rng, T, h_q * d)), req, h_q, cache, _i(selected), ws[:size], out[1:-1])
    assert bool((out[0] == 9.0).all()) and bool((out[-1] == 9.0).all()) and bool((ws[size:] == 0xFF).all())


@gpu
@pytest.mark.parametrize("h_q,h_kv,d", [(4, 2, 64), (40, 2, 128), (3, 1, 256)])
@pytest.mark.parametrize("count", [4, 17])  # lists whole, lists cut
def test_attention_selected_leaves_what_is_nobodys(h_q, h_kv, d, count):
    """Tokens that no request has: in front of the first, behind the last, and those of a request that are more than any may have."""
    rng = np.random.default_rng(54)
    n = [400, 1500]
    table, num = _pages(rng, n)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num)
    q = _normal(rng, 10, h_q * d)
    selected = np.tile(np.arange(count, dtype=np.int32), (10, h_kv, 1))
    req = B.Requests(_i([1, 3, 8]), _i(n), _i(table), 10, 2, 1500)
    got = _attend_selected(req, q, h_q, cache, _i(selected), fill=9.0).reshape(10, h_q, d)
    for t in range(10):
        if t in (1, 2, 3, 4):
            b, lim = (0, 399 + t - 1) if t < 3 else (1, 1499 + t - 3)
            lim = min(lim, 64 * count)
            _close(got[t:t + 1], *q4.attention(q.reshape(10, h_q, d)[t:t + 1], K[b][:lim], V[b][:lim], P[b][:lim]))
        else:
            assert np.all(got[t] == 9.0), t


@gpu
def test_a_page_listed_twice_counts_twice():
    rng = np.random.default_rng(52)
    n, h_q, h_kv, d = [400], 2, 1, 64
    table, num = _pages(rng, n)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num)
    q = _normal(rng, 1, h_q * d)
    got = _attend_selected(_requests([1], n, table), q, h_q, cache, _i([[[2, 0, 2, -1]]])).reshape(1, h_q, d)
    rows = np.concatenate([np.arange(128, 192), np.arange(64), np.arange(128, 192)])
    _close(got, *q4.attention(q.reshape(1, h_q, d), K[0][rows], V[0][rows], P[0][rows]))


# ---------------------------------------------------------------- runs of them
@gpu
def test_a_server_that_picks_pages_step_by_step():
    """Append, bound, select, attend, for prompts and then single tokens, pages taken as they are needed; with all pages selected the result is attention's over the cache."""
    rng = np.random.default_rng(61)
    h_q, h_kv, d, width, first, last, count = 8, 2, 64, 12, 1, 1, 5
    S, n = np.array([200, 3, 330]), np.array([200, 3, 330])
    cache = B.PagedCache(3 * width + 5, h_kv, d)
    cache.pages.fill_(0xFF)
    bounds, refs, table = B.PageBounds(cache), _i(np.zeros(cache.num_pages)), _i(np.full((3, width), -1))
    space = _space(B.qfc_pages_workspace_size(cache, 3))
    keys, values = [np.zeros((0, h_kv, d), np.float16) for _ in n], [np.zeros((0, h_kv, d), np.float16) for _ in n]
    for step in range(6):
        B.qfc_take_pages(cache, refs, table, _i(n), space)
        T = int(S.sum())
        qkv = _normal(rng, T, (h_q + 2 * h_kv) * d)
        req = B.Requests(_i(np.concatenate([[0], np.cumsum(S)])), _i(n), table, T, int(S.max()), int(n.max()))
        q = torch.empty((T, h_q * d), dtype=torch.float16, device=DEV)
        B.qfc_append_q4(_t(qkv), req, h_q, None, None, cache, q)
        B.qfc_bound_pages_q4(req, cache, bounds)
        selected = _select(req, q.cpu().numpy(), h_q, cache, bounds, first, last, count, T)
        out = _attend_selected(req, q.cpu().numpy(), h_q, cache, selected).reshape(T, h_q, d)
        whole = _attend_selected(req, q.cpu().numpy(), h_q, cache, _select(req, q.cpu().numpy(), h_q, cache, bounds, 0, 1, width, T)).reshape(T, h_q, d)
        x, at, g, picked = qkv.reshape(T, -1, d), 0, h_q // h_kv, selected.cpu().numpy()
        for b in range(3):
            keys[b] = np.concatenate([keys[b], x[at:at + S[b], h_q:h_q + h_kv]])
            values[b] = np.concatenate([values[b], x[at:at + S[b], h_q + h_kv:]])
            K, (V, P) = q4.q4_values(*q4.q4(keys[b]))[0], q4.q4_values(*q4.q4(values[b]))
            rows = x[at:at + S[b], :h_q]
            _close(whole[at:at + S[b]], *q4.attention(rows, K, V, P))
            codes, steps = _bounds_of(K, n[b], h_kv, d)
            for i in range(0, S[b], 1 if step else 37):
                m = n[b] - S[b] + i + 1
                for kv in range(h_kv):
                    # (a page of a prompt is bounded with all its positions, later ones of the same prompt among them)
                    want = ref.select(ref.scores(rows[i, kv * g:(kv + 1) * g], codes[:, kv], steps[:, kv], np.ones(len(steps), bool)), (m - 1) // 64 + 1, first, last, count)
                    assert np.array_equal(picked[at + i, kv], want)
                    there = np.isin(np.arange(m) // 64, want)
                    _close(out[at + i:at + i + 1, kv * g:(kv + 1) * g], *q4.attention(rows[i:i + 1, kv * g:(kv + 1) * g], K[:m, kv:kv + 1], V[:m, kv:kv + 1], P[:m, kv:kv + 1], there))
            at += S[b]
        S = np.array([1, 1 + step % 2, 1])
        n = n + S


@gpu
def test_a_search_behind_a_prompt_shares_its_pages():
    """One prompt, forked into continuations that grow apart, attention behind the common pages; then the pool is compacted and the same call gives the same bits."""
    rng = np.random.default_rng(62)
    h_q, h_kv, d, width, n0, kids = 8, 2, 128, 8, 300, 6
    cache = B.PagedCache(60, h_kv, d)
    cache.pages.fill_(0xFF)
    refs, root, space = _i(np.zeros(60)), _i(np.full((1, width), -1)), _space(B.qfc_pages_workspace_size(cache, kids))
    holes = _i(np.full((1, 30), -1))
    B.qfc_take_pages(cache, refs, holes, _i([30 * 64]), space)  # pages that are let go below
    B.qfc_take_pages(cache, refs, root, _i([n0]), space)

    def append(S, n, table):
        T = sum(S)
        qkv = _normal(rng, T, (h_q + 2 * h_kv) * d)
        req = B.Requests(_i(np.concatenate([[0], np.cumsum(S)])), _i(n), table, T, max(S), max(n))
        q = torch.empty((T, h_q * d), dtype=torch.float16, device=DEV)
        B.qfc_append_q4(_t(qkv), req, h_q, None, None, cache, q)
        return req, q, qkv.reshape(T, -1, d)

    _, _, x = append([n0], [n0], root)
    keys, values = [x[:, h_q:h_q + h_kv]] * kids, [x[:, h_q + h_kv:]] * kids
    table, n = _i(np.zeros((kids, width))), [n0] * kids
    B.qfc_fork_pages(cache, refs, root, _i([0] * kids), _i(n), table, space)
    B.qfc_free_pages(cache, refs, root)
    assert int(refs[30:34].min()) == kids and int(refs[34]) == 0  # four whole pages are shared, the fifth was copied
    shared = B.SharedPrefixes(_i([0, kids]), _i([n0]), 3 * kids, n0)
    for step in range(5):
        S = [1 + (step * b) % 3 for b in range(kids)]
        n = [a + b for a, b in zip(n, S)]
        B.qfc_take_pages(cache, refs, table, _i(n), space)
        req, q, x = append(S, n, table)
        got, at = _attend_shared(req, shared, q.cpu().numpy(), h_q, cache).reshape(-1, h_q, d), 0
        for b in range(kids):
            keys[b], values[b] = np.concatenate([keys[b], x[at:at + S[b], h_q:h_q + h_kv]]), np.concatenate([values[b], x[at:at + S[b], h_q + h_kv:]])
            K, (V, P) = q4.q4_values(*q4.q4(keys[b]))[0], q4.q4_values(*q4.q4(values[b]))
            _close(got[at:at + S[b]], *q4.attention(x[at:at + S[b], :h_q], K, V, P))
            at += S[b]
    B.qfc_free_pages(cache, refs, holes)
    before = table.clone()
    used = _i([0])
    B.qfc_compact_pages(cache, refs, table, space, used)
    assert int(used) == int((refs > 0).sum()) and not torch.equal(before, table) and int(table.max()) < int(used)
    assert np.array_equal(_attend_shared(req, shared, q.cpu().numpy(), h_q, cache).reshape(-1, h_q, d), got)


@gpu
def test_captured_steps_follow_the_arrays(rows_rule):
    """Attention behind common pages, bounds, selection and attention over it in one graph; lengths, tables and groups change between replays."""
    rng = np.random.default_rng(63)
    h_q, h_kv, d, batch, width, count = 8, 2, 64, 4, 20, 4
    lengths = [[700, 650, 1000, 64], [1200, 1, 300, 900], [80, 1279, 500, 640]]
    cache = B.PagedCache(batch * width, h_kv, d)
    table = np.arange(batch * width, dtype=np.int32).reshape(batch, width)
    table[:2, :6] = table[0, :6]
    every = [width * 64] * batch
    k, v = _normal(rng, width * 64 * batch, h_kv, d), _normal(rng, width * 64 * batch, h_kv, d)
    k[width * 64:width * 64 + 384], v[width * 64:width * 64 + 384] = k[:384], v[:384]
    _, K, V, P = _filled(rng, every, h_kv, d, table, batch * width, k, v, cache=cache)
    context, pages, start, group, prefix = _i(lengths[0]), _i(table), _i(range(batch + 1)), _i([0, 2]), _i([384])
    req, shared, bounds = B.Requests(start, context, pages, batch, 1, width * 64), B.SharedPrefixes(group, prefix, batch, width * 64), B.PageBounds(cache)
    B.qfc_bound_pages_q4(_requests(every, every, table), cache, bounds)
    q = torch.empty((batch, h_q * d), dtype=torch.float16, device=DEV)
    q.copy_(_t(_normal(rng, batch, h_q * d)))
    outs = [torch.zeros_like(q) for _ in range(2)]
    selected = torch.zeros((batch, h_kv, count), dtype=torch.int32, device=DEV)
    ws = [_space(B.qfc_attention_shared_q4_workspace_size(req, shared, h_q, cache)), _space(B.qfc_select_pages_q4_workspace_size(req, h_q, cache)),
          _space(B.qfc_attention_selected_q4_workspace_size(req, h_q, cache, count))]

    def step():
        B.qfc_attention_shared_q4(q, req, shared, h_q, cache, ws[0], outs[0])
        B.qfc_bound_pages_q4(req, cache, bounds)
        B.qfc_select_pages_q4(q, req, h_q, cache, bounds, 0, 1, selected, ws[1])
        B.qfc_attention_selected_q4(q, req, h_q, cache, selected, ws[2], outs[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for n, (g, p) in zip(lengths * 2, [([0, 2], [384]), ([1, 2], [300]), ([0, 2], [64]), ([0, 0], [0]), ([0, 4], [0]), ([0, 2], [2000])]):
        context.copy_(_i(n)), group.copy_(_i(g)), prefix.copy_(_i(p))
        q.copy_(_t(_normal(rng, batch, h_q * d)))
        for o in outs:
            o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        rows = q.cpu().numpy().reshape(batch, h_q, d)
        if p[0] <= 384:
            for b in range(batch):
                _close(got[0][b:b + 1].cpu().numpy().astype(np.float64).reshape(1, h_q, d), *q4.attention(rows[b:b + 1], K[b][:n[b]], V[b][:n[b]], P[b][:n[b]]))
        picked = selected.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], outs[0]) and torch.equal(got[1], outs[1]) and torch.equal(picked, selected)


@gpu
def test_two_streams_with_workspaces_of_their_own(rows_rule):
    rng = np.random.default_rng(64)
    group, prefix, S, n, h_q, h_kv, d = [0, 20], [640], [1] * 20, [641 + 9 * i for i in range(20)], 8, 2, 128
    cache, table, K, V, P = _shared_batch(rng, group, prefix, S, n, h_kv, d)
    req, shared = _requests(S, n, table), B.SharedPrefixes(_i(group), _i(prefix), 20, 640)
    qs = [_t(_normal(rng, 20, h_q * d)) for _ in range(2)]
    picks = [_i(np.tile(np.arange(i, i + 6), (20, h_kv, 1))) for i in range(2)]
    want = [(torch.empty_like(q), torch.empty_like(q)) for q in qs]
    outs = [[(torch.empty_like(q), torch.empty_like(q)) for q in qs] for _ in range(5)]
    sizes = B.qfc_attention_shared_q4_workspace_size(req, shared, h_q, cache), B.qfc_attention_selected_q4_workspace_size(req, h_q, cache, 6)
    ws = [[_space(x) for x in sizes] for _ in range(2)]

    def both(i, out):
        B.qfc_attention_shared_q4(qs[i], req, shared, h_q, cache, ws[i][0], out[0])
        B.qfc_attention_selected_q4(qs[i], req, h_q, cache, picks[i], ws[i][1], out[1])

    for i in range(2):
        both(i, want[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for out in outs:
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                both(i, out[i])
    torch.cuda.synchronize()
    for out in outs:
        for i in range(2):
            assert torch.equal(out[i][0], want[i][0]) and torch.equal(out[i][1], want[i][1])
