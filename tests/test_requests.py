"""Operators that serve a batch of different requests against the oracle: rotation and append into the paged 4-bit cache,
attention over it, low-rank adapters, and the run of them beside quantized layers."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import requests as ref
from paper_2505_00232_amd import binding as B
from paper_2505_00232_amd import synth

DEV = "cuda"
HALF = 2.0 ** -11  # a rounding to binary16, relative
gpu = pytest.mark.gpu


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _pages(rng, context, spare=3, width=None):
    """A page table over shuffled pages, -1 behind a request's last page."""
    used = [(n + 63) // 64 for n in context]
    order = rng.permutation(sum(used) + spare)
    table = np.full((len(context), width or max(max(used), 1)), -1, dtype=np.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    return table, sum(used) + spare


def _requests(S, n, table, rows=None, max_tokens=None, max_context=None):
    start = np.concatenate([[0], np.cumsum(S)]).astype(np.int32)
    return B.Requests(_t(start), _t(np.asarray(n, dtype=np.int32)), _t(table), rows or max(int(start[-1]), 1), max_tokens or max(max(S), 1), max_context or max(max(n), 1))


def _normal(rng, *shape):
    return rng.standard_normal(shape, dtype=np.float32).astype(np.float16)


def _filled(rng, n, h_kv, d, table, num_pages, k=None, v=None, cache=None):
    """A cache that holds n[b] positions of each request, garbage around them; (cache, K values, V values, V's parts) per request."""
    if cache is None:
        cache = B.PagedCache(num_pages, h_kv, d)
        cache.pages.fill_(0xFF)  # (NaN as steps and offsets)
    rows = sum(n)
    k = _normal(rng, rows, h_kv, d) if k is None else k
    v = _normal(rng, rows, h_kv, d) if v is None else v
    if rows:
        qkv = np.concatenate([k.reshape(rows, -1), k.reshape(rows, -1), v.reshape(rows, -1)], 1)
        B.qfc_append_q4(_t(qkv), _requests(n, n, table), h_kv, None, None, cache, torch.empty((rows, h_kv * d), dtype=torch.float16, device=DEV))
    K, _ = ref.q4_values(*ref.q4(k)) if rows else (k, k)
    V, P = ref.q4_values(*ref.q4(v)) if rows else (v, v)
    cut = np.cumsum(n)[:-1]
    return cache, np.split(K, cut), np.split(V, cut), np.split(P, cut)


def _attend(req, q, h_q, cache, fill=0.0):
    out = torch.full((q.shape[0], h_q * cache.d_head), fill, dtype=torch.float16, device=DEV)
    ws = torch.empty(B.qfc_attention_q4_workspace_size(req, h_q, cache), dtype=torch.uint8, device=DEV)
    B.qfc_attention_q4(_t(q), req, h_q, cache, ws, out)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64)


def _close(got, want, spread):
    """Roundings: the output (2^-11 of it), P times a step or P (2^-11 of the parts they multiply), and half as much again for sums and exponentials in 32 bits."""
    worst = np.max(np.abs(got - want) - HALF * np.abs(want) - 1.5 * HALF * spread - 2.0 ** -24, initial=-1.0)
    assert worst <= 0, (worst, float(np.max(np.abs(got - want))))


def _check_attention(rng, S, n, h_q, h_kv, d, **filled):
    table, num = _pages(rng, n)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num, **filled)
    q = _normal(rng, sum(S), h_q * d)
    got = _attend(_requests(S, n, table), q, h_q, cache).reshape(-1, h_q, d)
    at = 0
    for b, s in enumerate(S):
        want = ref.attention(q.reshape(-1, h_q, d)[at:at + s], K[b], V[b], P[b])
        _close(got[at:at + s], *want)
        at += s


# ---------------------------------------------------------------- refusals, without a GPU
def test_refusals_before_any_launch():
    L = B.lib()
    A, odd = 0x1000, 0x1002
    s = ctypes.c_void_p(0)
    size = ctypes.c_size_t(0)
    cache = lambda pages=A, num=4, h=2, d=64: ctypes.byref(B.CacheDesc(pages, num, h, d))
    req = lambda start=A, ctx=A, table=A, batch=2, tokens=2, most=1, longest=128, width=2: ctypes.byref(B.RequestsDesc(start, ctx, table, batch, tokens, most, longest, width))
    rot = lambda dim=64, layout=0, base=1e4, factor=1.0, orig=0, low=1.0, high=4.0, amp=1.0: ctypes.byref(B.Rotary(dim, layout, base, factor, orig, low, high, amp))
    assert L.qfc_q4_cache_size(cache(None), ctypes.byref(size)) == 0 and size.value == 4 * 2 * 80 * 64
    assert L.qfc_q4_cache_size(cache(None, d=96), ctypes.byref(size)) == 2 and L.qfc_q4_cache_size(cache(num=0), ctypes.byref(size)) == 1
    assert L.qfc_q4_cache_size(None, ctypes.byref(size)) == 1 and L.qfc_q4_cache_size(cache(), None) == 1
    # the table
    assert L.qfc_rotary_table(None, 8, A, s) == 1 and L.qfc_rotary_table(rot(), 0, A, s) == 1 and L.qfc_rotary_table(rot(), 8, None, s) == 1
    for bad in (rot(layout=2), rot(base=1.0), rot(base=float("inf")), rot(base=float("nan")), rot(factor=0.5), rot(factor=float("nan")), rot(orig=-1), rot(amp=0.0), rot(dim=0),
                rot(orig=8, low=4.0, high=4.0), rot(orig=8, low=-1.0), rot(orig=8, high=float("nan"))):
        assert L.qfc_rotary_table(bad, 8, A, s) == 1
        assert L.qfc_append_q4(A, req(), 4, bad, A, 128, cache(), A, s) == 1
    assert L.qfc_rotary_table(rot(dim=40), 8, A, s) == 2 and L.qfc_rotary_table(rot(dim=272), 8, A, s) == 2 and L.qfc_rotary_table(rot(), 8, 0x1004, s) == 4
    # batches: the same checks in front of append, read and attention
    calls = [lambda r, c, h=4: L.qfc_append_q4(A, r, h, None, None, 0, c, A, s), lambda r, c, h=4: L.qfc_attention_q4(A, r, h, c, A, 1 << 40, A, s)]
    for call in calls + [lambda r, c, h=None: L.qfc_read_q4(r, c, A, A, s)]:
        for bad in (None, req(start=None), req(ctx=None), req(table=None), req(batch=0), req(tokens=-1), req(most=0), req(longest=0), req(longest=129), req(width=0)):
            assert call(bad, cache()) == 1
        for bad in (None, cache(None), cache(num=0), cache(h=0)):
            assert call(req(), bad) == 1
        assert call(req(), cache(d=80)) == 2 and call(req(), cache(odd)) == 4
        for bad in (req(start=odd), req(ctx=odd), req(table=0x1001)):
            assert call(bad, cache()) == 4
        assert call(req(batch=40000), cache(h=2)) == 2
        assert call(req(tokens=0), cache()) == 0  # nothing to do, nothing launched
    for call in calls:
        assert call(req(), cache(), 3) == 1 and call(req(), cache(), 0) == 1 and call(req(), cache(h=2), 65534) == 2 and call(req(most=1 << 25), cache(), 4) == 2
    assert L.qfc_append_q4(None, req(), 4, None, None, 0, cache(), A, s) == 1 and L.qfc_append_q4(A, req(), 4, None, None, 0, cache(), None, s) == 1
    assert L.qfc_append_q4(odd, req(), 4, None, None, 0, cache(), A, s) == 4
    assert L.qfc_append_q4(A, req(), 4, rot(), A, 127, cache(), A, s) == 1 and L.qfc_append_q4(A, req(), 4, rot(), None, 128, cache(), A, s) == 1
    assert L.qfc_append_q4(A, req(), 4, rot(), 0x1004, 128, cache(), A, s) == 4 and L.qfc_append_q4(A, req(), 4, rot(dim=80), A, 128, cache(), A, s) == 2
    assert L.qfc_read_q4(req(), cache(), None, A, s) == 1 and L.qfc_read_q4(req(), cache(), A, odd, s) == 4
    assert L.qfc_attention_q4(A, req(), 4, cache(), None, 1 << 40, A, s) == 1 and L.qfc_attention_q4(A, req(), 4, cache(), A, 0, A, s) == 3
    assert L.qfc_attention_q4(A, req(), 4, cache(), odd, 1 << 40, A, s) == 4 and L.qfc_attention_q4(None, req(), 4, cache(), A, 1 << 40, A, s) == 1
    assert L.qfc_attention_q4_workspace_size(req(start=None, ctx=None, table=None), 4, cache(None), ctypes.byref(size)) == 0 and size.value > 0
    assert L.qfc_attention_q4_workspace_size(req(), 4, cache(), None) == 1
    # adapters
    ad = lambda a=A, b=A, sc=A, count=2, rank=16, K=64, N=40: ctypes.byref(B.AdaptersDesc(a, b, sc, count, rank, K, N))
    assert L.qfc_adapters_workspace_size(ad(None, None, None), 5, ctypes.byref(size)) == 0 and size.value >= 16 * 16 * 4
    add = lambda d, x=A, M=5, ids=A, y=A, ws=A, n=1 << 40, out=A: L.qfc_add_adapters(x, M, ids, d, y, ws, n, out, s)
    for bad in (None, ad(None), ad(b=None), ad(sc=None), ad(count=0), ad(rank=0), ad(K=0), ad(K=40), ad(N=0)):
        assert add(bad) == 1
    assert add(ad(rank=12)) == 2 and add(ad(rank=136)) == 2 and add(ad(a=odd)) == 4 and add(ad(sc=odd)) == 4 and add(ad(), ids=odd) == 4
    assert add(ad(), x=None) == 1 and add(ad(), M=0) == 1 and add(ad(), ids=None) == 1 and add(ad(), y=None) == 1 and add(ad(), ws=None) == 1 and add(ad(), out=None) == 1
    assert add(ad(), n=16) == 3 and add(ad(), x=0x1008) == 4


def test_refusals_of_the_largest_sizes_and_calls_without_tokens():
    L = B.lib()
    A, s, size = 0x1000, ctypes.c_void_p(0), ctypes.c_size_t(0)
    ad = lambda N: ctypes.byref(B.AdaptersDesc(A, A, A, 2, 16, 64, N))
    for M, N in (((1 << 24) + 1, 8), (1, (1 << 23) + 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert L.qfc_adapters_workspace_size(ad(N), M, ctypes.byref(size)) == 2
        assert L.qfc_add_adapters(A, M, A, ad(N), A, A, 1 << 60, A, s) == 2
    assert L.qfc_adapters_workspace_size(ad(1 << 23), 1 << 24, ctypes.byref(size)) == 0 and size.value >= (1 << 24) * 16 * 4
    cache, none = ctypes.byref(B.CacheDesc(A, 4, 2, 64)), ctypes.byref(B.RequestsDesc(A, A, A, 2, 0, 1, 128, 2))
    assert L.qfc_append_q4(None, none, 4, None, None, 0, cache, None, s) == 0 and L.qfc_read_q4(none, cache, None, None, s) == 0
    assert L.qfc_attention_q4(None, none, 4, cache, None, 0, None, s) == 0
    assert L.qfc_attention_q4(None, none, 3, cache, None, 0, None, s) == 1


def test_refusals_of_batches_above_each_limit():
    """At a limit the workspace's size is given; one more is refused by every call."""
    L = B.lib()
    A, s, size = 0x1000, ctypes.c_void_p(0), ctypes.c_size_t(0)
    pairs = [  # (batch, tokens, max_tokens, max_context, h_q, h_kv, d) at the limit, and above it
        ((2, 2, 1, 128, 65531, 1, 64), None), (None, (2, 2, 1, 128, 65534, 1, 64)), ((65535, 2, 1, 128, 1, 1, 64), (65536, 2, 1, 128, 1, 1, 64)),
        ((2, 2, 1 << 25, 128, 2, 1, 64), (2, 2, (1 << 25) + 1, 128, 2, 1, 64)), ((16, 1 << 22, 1 << 18, 128, 256, 1, 64), (16, (1 << 22) + 1, 1 << 18, 128, 256, 1, 64)),
        ((2, 1 << 28, 1 << 26, 128, 1, 1, 64), (2, (1 << 28) + 1, 1 << 26, 128, 1, 1, 64)), ((2, 1 << 26, 1 << 26, 128, 1, 1, 256), (2, (1 << 26) + 1, 1 << 26, 128, 1, 1, 256)),
        ((2, 2, 1, 1 << 26, 2, 1, 64), (2, 2, 1, (1 << 26) + 1, 2, 1, 64))]
    for case, want in [(c, w) for pair in pairs for c, w in zip(pair, (0, 2)) if c]:
        batch, tokens, most, longest, h_q, h_kv, d = case
        req = ctypes.byref(B.RequestsDesc(A, A, A, batch, tokens, most, longest, 1 << 21))
        cache = ctypes.byref(B.CacheDesc(A, 4, h_kv, d))
        assert L.qfc_attention_q4_workspace_size(req, h_q, cache, ctypes.byref(size)) == want, case
        if want:
            assert L.qfc_append_q4(A, req, h_q, None, None, 0, cache, A, s) == 2 and L.qfc_attention_q4(A, req, h_q, cache, A, 1 << 60, A, s) == 2
            assert h_q != h_kv or L.qfc_read_q4(req, cache, A, A, s) == 2


def test_binding_refuses_host_tensors():
    c = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.Requests(torch.zeros(3, dtype=torch.int32), c, torch.zeros((2, 1), dtype=torch.int32), 2, 1, 64)
    with pytest.raises(ValueError):
        B.Adapters(torch.zeros((1, 8, 32), dtype=torch.float16), torch.zeros((1, 4, 8), dtype=torch.float16), torch.zeros(1))


def test_oracle_q4_by_hand():
    x = np.zeros(32, dtype=np.float16)
    x[:16] = np.arange(16)
    code, step, offset = ref.q4(x[None])
    assert step[0, 0] == 1.0 and offset[0, 0] == 8.0 and np.array_equal(code[0, :16], np.arange(16))
    assert np.array_equal(ref.q4_values(code, step, offset)[0][0], x.astype(np.float64))
    code, step, offset = ref.q4(np.full((1, 32), 65504, dtype=np.float16))
    assert step[0, 0] == 0 and offset[0, 0] == 65504 and np.all(code == 8)


# ---------------------------------------------------------------- rotation and append
@gpu
@pytest.mark.parametrize("rot,extra", [(128, {}), (64, dict(factor=4.0)), (16, dict(factor=8.0, original_positions=8192, low_turns=1.0, high_turns=4.0)),
                                       (256, dict(factor=16.0, original_positions=4096, low_turns=1.0, high_turns=32.0, amplitude=1.277))])
def test_rotary_table(rot, extra):
    positions = 131072
    table = B.qfc_rotary_table(B.make_rotary(rot, 500000.0, **extra), positions).cpu().numpy()
    at = np.unique(np.concatenate([np.arange(64), np.random.default_rng(1).integers(0, positions, 500), [positions - 1]]))
    keys = dict(factor="factor", original_positions="original", low_turns="low", high_turns="high", amplitude="amplitude")
    want = ref.rotary_table(rot, at, np.float32(500000.0), **{keys[k]: float(np.float32(v)) for k, v in extra.items()})
    # the rounding to 32 bits of values up to the amplitude, and 2^17 turns' angle to 2^-50 of it: less than another one
    assert np.max(np.abs(table[at] - want)) <= 2.0 ** -24 * extra.get("amplitude", 1.0)


@gpu
def test_rotary_table_of_more_angles_than_a_launch_has_threads():
    """2^26 positions (the most that a batch may have) of 64 pairs.  Bound: the rounding to 32 bits 2^-25; on either side the frequency's roundings, 3 (1 + x) e^-x 2^-53 <= 3 2^-53
    for f = e^-x, at 2^26 positions 2^-25.4; together less than 2^-23."""
    positions, rotary = 1 << 26, B.make_rotary(128, 500000.0)
    table = B.qfc_rotary_table(rotary, positions)
    few = B.qfc_rotary_table(rotary, 5000)
    assert torch.equal(table[:5000], few)
    at = np.unique(np.concatenate([np.random.default_rng(2).integers(0, positions, 300), np.arange(positions - 3, positions), (1 << 22) + np.arange(-2, 3), (1 << 25) + np.arange(-2, 3)]))
    got = table[torch.from_numpy(at).to(DEV)].cpu().numpy()
    assert np.max(np.abs(got - ref.rotary_table(128, at, 500000.0))) <= 2.0 ** -23


@gpu
def test_rotary_table_is_the_other_one_where_they_meet():
    a = B.qfc_rope_table(B.AttnShape(1, 2, 1, 128, 64), 10000.0, 5000)
    b = B.qfc_rotary_table(B.make_rotary(128, 10000.0), 5000)
    assert float((a - b).abs().max()) <= 2.0 ** -24


APPENDS = [  # S, n, h_q, h_kv, d, rot, interleaved
    ([1], [1], 1, 1, 64, 64, False),
    ([1], [1280], 32, 8, 128, 128, False),
    ([1, 0, 2, 1], [70, 5, 2, 64], 4, 2, 64, 16, True),
    ([65, 3, 130], [65, 200, 193], 6, 2, 128, 96, False),
    ([31, 1, 40], [100, 64, 41], 8, 4, 256, 128, True),
    ([7, 64], [1000, 64], 3, 3, 256, 256, False),
    ([200], [777], 16, 1, 64, 48, True),
    ([1] * 67, list(range(1, 68)), 4, 1, 128, 112, False),
]


@gpu
@pytest.mark.parametrize("S,n,h_q,h_kv,d,rot,interleaved", APPENDS)
def test_append(S, n, h_q, h_kv, d, rot, interleaved):
    """Bit for bit: the rotation is rounded once from exact products, the codes are defined operation by operation."""
    rng = np.random.default_rng(11)
    table, num = _pages(rng, n)
    T, behind = sum(S), 2
    qkv = _normal(rng, T + behind, (h_q + 2 * h_kv) * d)
    req = _requests(S, n, table, rows=T + behind)
    cache = B.PagedCache(num, h_kv, d)
    cache.pages.fill_(0xA5)
    before = cache.pages.clone()
    rotary = B.make_rotary(rot, 10000.0, layout=B.QFC_ROPE_INTERLEAVED if interleaved else B.QFC_ROPE_HALF, factor=4.0, original_positions=512)
    angles = B.qfc_rotary_table(rotary, max(n))
    q = torch.full((T + behind, h_q * d), 77.0, dtype=torch.float16, device=DEV)
    k, v = (torch.full((T + behind, h_kv, d), 55.0, dtype=torch.float16, device=DEV) for _ in range(2))
    B.qfc_append_q4(_t(qkv), req, h_q, rotary, angles, cache, q)
    B.qfc_read_q4(req, cache, k, v)
    torch.cuda.synchronize()
    pos = np.concatenate([np.arange(m - s, m) for s, m in zip(S, n)])
    x = qkv[:T].reshape(T, -1, d)
    turned = ref.rotate(x[:, :h_q + h_kv], angles.cpu().numpy()[pos], interleaved)
    assert np.array_equal(q[:T].cpu().numpy().reshape(T, h_q, d), turned[:, :h_q])
    for got, rows in ((k, turned[:, h_q:]), (v, x[:, h_q + h_kv:])):
        want = ref.q4_values(*ref.q4(rows))[0].astype(np.float32).astype(np.float16)
        assert np.array_equal(got[:T].cpu().numpy(), want)
    for t, fill in ((q, 77.0), (k, 55.0), (v, 55.0)):
        assert bool((t[T:] == fill).all())  # rows behind the last request
    # everything that belongs to no new token is as it was: appending the same rows to a copy of the state before changes the same bytes only
    changed = (cache.pages != before).sum().item()
    assert changed <= T * h_kv * (d + 4 * 2 * (d // 32))
    once = cache.pages.clone()
    B.qfc_append_q4(_t(qkv), req, h_q, rotary, angles, cache, q)
    assert torch.equal(once, cache.pages)


@gpu
def test_append_token_by_token_is_append_at_once():
    rng = np.random.default_rng(12)
    n, h_kv, d = 150, 2, 128
    table, num = _pages(rng, [n])
    qkv = _normal(rng, n, 4 * h_kv * d)
    rotary = B.make_rotary(d, 10000.0)
    angles = B.qfc_rotary_table(rotary, n)
    whole, single = B.PagedCache(num, h_kv, d), B.PagedCache(num, h_kv, d)
    whole.pages.zero_()
    single.pages.zero_()
    q = torch.empty((n, 2 * h_kv * d), dtype=torch.float16, device=DEV)
    B.qfc_append_q4(_t(qkv), _requests([n], [n], table), 2 * h_kv, rotary, angles, whole, q)
    at = 0
    for s in [1, 2, 3, 5, 1, 20, 33, 64, 21]:  # ends inside and at pages, dwords and tiles
        B.qfc_append_q4(_t(qkv[at:at + s]), _requests([s], [at + s], table, max_context=n), 2 * h_kv, rotary, angles, single, torch.empty((s, 2 * h_kv * d), dtype=torch.float16, device=DEV))
        at += s
    assert at == n and torch.equal(whole.pages, single.pages)


@gpu
def test_append_extreme_values():
    rng = np.random.default_rng(13)
    h_kv, d, n = 1, 64, 12
    k, v = (_normal(rng, n, h_kv, d) for _ in range(2))
    k[0], k[1], k[2, 0, ::2], k[2, 0, 1::2] = 0, 65504, 65504, -65504
    k[3], k[4], k[5] = k[3] * np.float16(2.0 ** -14), np.float16(2.0 ** -24), np.float16(-0.0)
    v[0] = k[2]
    v[1] = v[1] * np.float16(2.0 ** -20)
    v[2, 0, 32:] = 1000
    table, num = _pages(rng, [n])
    cache, _, _, _ = _filled(rng, [n], h_kv, d, table, num, k, v)
    got = [torch.empty((n, h_kv, d), dtype=torch.float16, device=DEV) for _ in range(2)]
    B.qfc_read_q4(_requests([n], [n], table), cache, *got)
    for g, rows in zip(got, (k, v)):
        assert np.array_equal(g.cpu().numpy(), ref.q4_values(*ref.q4(rows))[0].astype(np.float32).astype(np.float16))


# ---------------------------------------------------------------- attention
ATTENDS = [  # S, n, h_q, h_kv, d
    ([1], [1], 1, 1, 64),
    ([1], [64], 4, 1, 128),
    ([1], [65], 2, 2, 256),
    ([1], [1280], 32, 8, 128),
    ([1, 1, 1], [3, 500, 129], 8, 2, 64),
    ([1, 1], [700, 63], 8, 4, 256),
    ([1] * 5, [1, 64, 127, 128, 4000], 16, 2, 128),
    ([4, 1, 2], [4, 300, 65], 16, 1, 128),     # 64 query rows of a head
    ([17], [17], 3, 1, 128),                   # rows of one token in two blocks
    ([5, 9], [70, 9], 7, 7, 64),
    ([1], [333], 40, 2, 64),                   # 20 heads on one
    ([130, 1, 0, 33], [130, 257, 9, 1000], 4, 2, 128),
    ([100, 65], [163, 65], 2, 1, 256),
    ([257], [300], 8, 2, 64),
    ([200, 1, 3], [3000, 2000, 70], 8, 2, 64),  # a prompt's walks in pieces, beside single tokens
    ([1, 90, 300, 2], [700, 90, 811, 2], 4, 1, 128),
    ([150, 260], [150, 700], 4, 2, 256),
    ([600, 17], [601, 900], 1, 1, 128),
    ([100] * 5, [100, 163, 164, 500, 228], 6, 2, 64),
]


@gpu
@pytest.mark.parametrize("S,n,h_q,h_kv,d", ATTENDS)
def test_attention(S, n, h_q, h_kv, d):
    _check_attention(np.random.default_rng(21), S, n, h_q, h_kv, d)


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("k_size,v_size", [(1.0, 2000.0), (1.0, 2.0 ** -13), (30.0, 1.0), (0.0, 1.0), (1.0, 0.0)])
def test_attention_sizes_of_values(d, k_size, v_size):
    """Steps of 2 and more, steps that are denormal, sharp and flat maps."""
    rng = np.random.default_rng(22)
    n, h_kv = [300, 70], 2
    k, v = (_normal(rng, sum(n), h_kv, d).astype(np.float32) for _ in range(2))
    v[::7] *= 0.01  # (small steps beside large ones, in pages before and behind them)
    _check_attention(rng, [1, 3], n, 4, h_kv, d, k=(k * k_size).astype(np.float16), v=(v * v_size).astype(np.float16))


@gpu
@pytest.mark.parametrize("least", [0, 5, 300])  # pages a wavefront takes at least: wavefronts with and without large steps, and walks that meet them on the way
@pytest.mark.parametrize("first,last", [(0, 64), (640, 704), (700, 701), (1280, 1399)])
@pytest.mark.parametrize("S,h_q,h_kv,d", [([1, 1], 4, 2, 64), ([3, 1], 2, 1, 256), ([600], 8, 2, 64)])
def test_attention_large_values_in_some_pages(S, h_q, h_kv, d, first, last, least):
    """Steps of 2 and more in one page of a walk that several wavefronts share, in the middle of one wavefront's, and in the last page; other requests without any."""
    rng = np.random.default_rng(58)
    n = [1400, 1000][:len(S)]
    k, v = (_normal(rng, sum(n), h_kv, d) for _ in range(2))
    v[first:last] *= np.float16(100)
    try:
        B.lib().qfc_tune(15, least)
        _check_attention(rng, S, n, h_q, h_kv, d, k=k, v=v)
    finally:
        B.lib().qfc_tune(15, 0)


@gpu
@pytest.mark.parametrize("least", [0, 300])
@pytest.mark.parametrize("S,d,n,where,value,small,gap", [(1, 64, 1000, 100, 40, 0.05, 12), (1, 64, 1000, 100, 40, 0.005, 12), (1, 64, 8000, 100, 30.5, 0.01, 16), (1, 64, 8000, 70, 4000, 0.005, 12),
                                                         (3, 128, 1000, 64, 60000, 0.01, 14), (3, 128, 1000, 999, 60000, 0.01, 14), (1, 256, 1000, 100, 40, 0.005, 12), (20, 256, 400, 0, 300, 0.02, 12)])
def test_attention_large_value_beside_small_ones(S, d, n, where, value, small, gap, least):
    """One large value in one group of 32, a group of small ones beside it, and a position with nearly all of P whose values are next to nothing: the others make up the result, with
    products down to 2^-30 of the large value's.  (Products that are denormals of binary16 are off by 2^-25 of 2^14, times a code of 8: 2^-36, nothing against the bound's 2^-24.)"""
    rng = np.random.default_rng(59)
    q, k, v = _normal(rng, S, d), _normal(rng, n, 1, d), _normal(rng, n, 1, d)
    k[5, 0] = q[0] * np.float16(gap * np.sqrt(d) / np.sum(q[0].astype(np.float64) ** 2))
    v[:, :, 32:] *= np.float16(small)
    v[5] *= np.float16(1e-3)
    v[where, 0, 3] = value
    table, num = _pages(rng, [n])
    try:
        B.lib().qfc_tune(15, least)
        cache, K, V, P = _filled(rng, [n], 1, d, table, num, k=k, v=v)
        got = _attend(_requests([S], [n], table), q, 1, cache).reshape(-1, 1, d)
    finally:
        B.lib().qfc_tune(15, 0)
    _close(got, *ref.attention(q.reshape(-1, 1, d), K[0], V[0], P[0]))


@gpu
def test_attention_far_from_zero():
    """Keys and values with a mean far above their spread: offsets carry the result."""
    rng = np.random.default_rng(23)
    n = [200]
    k, v = _normal(rng, 200, 2, 128) + np.float16(8), _normal(rng, 200, 2, 128) - np.float16(50)
    _check_attention(rng, [2], n, 8, 2, 128, k=k, v=v)


@gpu
@pytest.mark.parametrize("S", [1, 40, 150])
def test_attention_rows_that_see_nothing_and_missing_pages(S):
    rng = np.random.default_rng(24)
    h_q, h_kv, d, n = 4, 2, 128, [300, 0, 200, 130, 64]
    table, num = _pages(rng, n)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num)
    there = [np.ones(x, dtype=bool) for x in n]
    # pages that are none: in the middle, the last, all of them; indexes on either side of the range
    table[0, 1], table[0, 4], table[2, 3] = -1, num, np.iinfo(np.int32).max
    table[3, :] = np.iinfo(np.int32).min
    there[0][64:128], there[0][256:], there[2][192:], there[3][:] = False, False, False, False
    T = S * len(n)
    req = _requests([S] * len(n), n, table, rows=T + 3)
    q = _normal(rng, T + 3, h_q * d)
    got = _attend(req, q, h_q, cache, fill=9.0).reshape(-1, h_q, d)
    for b in range(len(n)):
        rows = slice(b * S, b * S + S)
        # (fewer positions than tokens: the first tokens have none)
        want = ref.attention(q.reshape(-1, h_q, d)[rows], K[b], V[b], P[b], there[b])
        _close(got[rows], *want)
    assert np.all(got[S:2 * S] == 0) and np.all(got[3 * S:4 * S] == 0) and np.all(got[T:] == 9.0)


@gpu
def test_arrays_that_break_the_rules_stay_inside_the_buffers():
    """Starts that descend or pass the rows, contexts and tokens above the limits: no result is defined, and nothing outside the outputs changes."""
    rng = np.random.default_rng(25)
    h_q, h_kv, d = 4, 2, 64
    table, num = _pages(rng, [256, 256, 256])
    cache, _, _, _ = _filled(rng, [256, 256, 256], h_kv, d, table, num)
    q = _normal(rng, 8, h_q * d)
    qkv = _normal(rng, 8, (h_q + 2 * h_kv) * d)
    for start, ctx in (([0, 5, 2, 8], [256, 256, 256]), ([-7, 3, 900, 2 ** 31 - 1], [2 ** 31 - 1, -5, 256]), ([0, 8, 8, 8], [256, 0, 0])):
        req = B.Requests(_t(np.asarray(start, dtype=np.int32)), _t(np.asarray(ctx, dtype=np.int32)), _t(table), 8, 2, 256)
        guard = torch.full((8 + 16, h_q * d), 3.0, dtype=torch.float16, device=DEV)
        for name in ("append", "attention"):
            out = guard[8:16]
            if name == "append":
                B.qfc_append_q4(_t(qkv), req, h_q, None, None, cache, out)
            else:
                ws = torch.empty(B.qfc_attention_q4_workspace_size(req, h_q, cache), dtype=torch.uint8, device=DEV)
                B.qfc_attention_q4(_t(q), req, h_q, cache, ws, out)
            torch.cuda.synchronize()
            assert bool((guard[:8] == 3.0).all()) and bool((guard[16:] == 3.0).all())


@gpu
def test_requests_that_overlap_until_their_places_pass_an_int():
    """Thousands of requests that each claim all rows: the call ends, does no more than its limits allow, and writes nothing outside its rows."""
    T, batch, longest, d = 16384, 4096, 131072, 64
    start = np.zeros(batch + 1, dtype=np.int32)
    start[1::2] = T  # 0, T, 0, T, ...
    cache = B.PagedCache(4, 1, d)
    cache.pages.zero_()
    table = torch.zeros((batch, longest // 64), dtype=torch.int32, device=DEV)
    req = B.Requests(_t(start), torch.full((batch,), longest, dtype=torch.int32, device=DEV), table, T, T, longest)
    guard = torch.full((T + 32, d), 3.0, dtype=torch.float16, device=DEV)
    ws = torch.empty(B.qfc_attention_q4_workspace_size(req, 1, cache) + 1024, dtype=torch.uint8, device=DEV)
    ws[-1024:] = 0x5A
    try:
        for least in (0, 40):
            B.lib().qfc_tune(15, least)
            B.qfc_attention_q4(torch.ones((T, d), dtype=torch.float16, device=DEV), req, 1, cache, ws, guard[16:-16])
            torch.cuda.synchronize()
            assert bool((guard[:16] == 3.0).all()) and bool((guard[-16:] == 3.0).all()) and bool((ws[-1024:] == 0x5A).all())
    finally:
        B.lib().qfc_tune(15, 0)


@gpu
def test_pages_beyond_two_gigabytes():
    rng = np.random.default_rng(26)
    h_q, h_kv, d, n = 16, 8, 128, [130]
    num = 60000  # 4.9 GB
    cache = B.PagedCache(num, h_kv, d)
    table = np.asarray([[num - 1, 1, num - 3]], dtype=np.int32)
    _, K, V, P = _filled(rng, n, h_kv, d, table, num, cache=cache)
    q = _normal(rng, 1, h_q * d)
    got = _attend(_requests([1], n, table), q, h_q, cache).reshape(-1, h_q, d)
    _close(got, *ref.attention(q.reshape(1, h_q, d), K[0], V[0], P[0]))


@gpu
def test_captured_decode_step_follows_its_arrays():
    """A captured append and attention, replayed while lengths and pages change, against eager calls; on a stream of its own."""
    rng = np.random.default_rng(27)
    h_q, h_kv, d, batch, longest = 8, 2, 128, 3, 640
    width = longest // 64
    num = batch * width
    table = _t(rng.permutation(num).reshape(batch, width).astype(np.int32))
    cache, twin = B.PagedCache(num, h_kv, d), B.PagedCache(num, h_kv, d)
    _filled(rng, [200, 63, 512], h_kv, d, table.cpu().numpy(), num, cache=cache)
    twin.pages.copy_(cache.pages)
    context = torch.zeros(batch, dtype=torch.int32, device=DEV)
    req = B.Requests(torch.arange(batch + 1, dtype=torch.int32, device=DEV), context, table, batch, 1, longest)
    rotary = B.make_rotary(d, 10000.0)
    angles = B.qfc_rotary_table(rotary, longest)
    qkv = torch.empty((batch, (h_q + 2 * h_kv) * d), dtype=torch.float16, device=DEV)
    E = lambda: torch.empty((batch, h_q * d), dtype=torch.float16, device=DEV)
    q, out, q2, out2 = E(), E(), E(), E()
    ws, ws2 = (torch.empty(B.qfc_attention_q4_workspace_size(req, h_q, cache), dtype=torch.uint8, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    context.copy_(_t(np.asarray([201, 64, 513], dtype=np.int32)))
    qkv.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.qfc_append_q4(qkv, req, h_q, rotary, angles, cache, q)
        B.qfc_attention_q4(q, req, h_q, cache, ws, out)
    for step in range(5):
        context.copy_(_t(np.asarray([201 + step, 64 + step, 513 + 25 * step], dtype=np.int32)))
        qkv.copy_(_t(_normal(rng, *qkv.shape)))
        graph.replay()
        torch.cuda.synchronize()
        B.qfc_append_q4(qkv, req, h_q, rotary, angles, twin, q2)
        B.qfc_attention_q4(q2, req, h_q, twin, ws2, out2)
        torch.cuda.synchronize()
        assert torch.equal(q, q2) and torch.equal(out, out2) and torch.equal(cache.pages, twin.pages)


@gpu
def test_attention_repeats_bit_for_bit():
    rng = np.random.default_rng(28)
    n, S = [5000, 64, 900], [1, 40, 3]
    table, num = _pages(rng, n)
    cache, _, _, _ = _filled(rng, n, 2, 128, table, num)
    q, req = _normal(rng, sum(S), 8 * 128), _requests(S, n, table)
    first = _attend(req, q, 8, cache)
    assert np.array_equal(first, _attend(req, q, 8, cache))


@gpu
@pytest.mark.parametrize("S,n,h_q,h_kv", [([1, 1, 1], [3000, 700, 40], 4, 1), ([3, 5], [250, 60], 4, 2), ([600], [1400], 8, 2)])
def test_attention_of_queries_that_are_not_finite(S, n, h_q, h_kv):
    """Walked by one wavefront and by several, joined by either kernel: their own row and head is NaN, the others keep their bits."""
    rng = np.random.default_rng(61)
    d = 64
    table, num = _pages(rng, n)
    cache, _, _, _ = _filled(rng, n, h_kv, d, table, num)
    q, req = _normal(rng, sum(S), h_q * d), _requests(S, n, table)
    clean = _attend(req, q, h_q, cache)
    bad = np.zeros((sum(S), h_q), dtype=bool)
    for row, head, value in ((0, 1, np.nan), (sum(S) - 1, 0, np.nan), (sum(S) // 2, 2, np.inf)):
        q.reshape(-1, h_q, d)[row, head, 7], bad[row, head] = value, True
    got = _attend(req, q, h_q, cache).reshape(-1, h_q, d)
    assert np.array_equal(got[~bad], clean.reshape(-1, h_q, d)[~bad]) and np.all(np.isnan(got[bad]))


@gpu
@pytest.mark.parametrize("S,n,h_q,h_kv", [([1, 1], [3000, 700], 4, 1), ([40, 3], [2500, 900], 4, 2), ([600], [1400], 8, 2), ([327, 300], [2000, 1700], 12, 4)])
def test_attention_whatever_the_workspace_holds(S, n, h_q, h_kv):
    """Partial results are read where a wavefront has left some: not in the places of blocks without a partner, of rows behind a block's last, of units that were not cut."""
    rng = np.random.default_rng(60)
    d = 64
    table, num = _pages(rng, n)
    cache, _, _, _ = _filled(rng, n, h_kv, d, table, num)
    q, req = _t(_normal(rng, sum(S), h_q * d)), _requests(S, n, table)
    out = []
    for fill in (0, 0xFF, 0x7C):  # (NaN; large values)
        ws = torch.full((B.qfc_attention_q4_workspace_size(req, h_q, cache),), fill, dtype=torch.uint8, device=DEV)
        out.append(torch.zeros_like(q))
        B.qfc_attention_q4(q, req, h_q, cache, ws, out[-1])
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2]) and bool(torch.isfinite(out[0]).all())


# ---------------------------------------------------------------- adapters
def _adapters(rng, count, rank, K, N):
    a = (_normal(rng, count, rank, K).astype(np.float32) / np.sqrt(K)).astype(np.float16)
    b = (_normal(rng, count, N, rank).astype(np.float32) / np.sqrt(rank)).astype(np.float16)
    return a, b, rng.uniform(0.5, 2.0, count).astype(np.float32)


def _add(x, ids, a, b, scale, y, alias=False):
    ad = B.Adapters(_t(a), _t(b), _t(scale))
    ws = torch.empty(B.qfc_adapters_workspace_size(ad, x.shape[0]), dtype=torch.uint8, device=DEV)
    yd = _t(y)
    out = yd if alias else torch.empty_like(yd)
    B.qfc_add_adapters(_t(x), _t(ids), ad, yd, ws, out)
    torch.cuda.synchronize()
    return out.cpu().numpy()


def _check_adapters(got, x, ids, a, b, scale, y):
    """Roundings: the output, and the low-rank values in binary16 (2^-11 of each product); as much as the latter once more for the sums over K in 32 bits (K 2^-24 <= 2^-12
    of terms some sqrt(K) times the sum) and values far below the row's largest."""
    want, spread = ref.adapters(x, ids, a, b, scale, y)
    low = np.zeros_like(spread)
    for m, i in enumerate(ids):
        if 0 <= i < a.shape[0]:
            low[m] = abs(scale[i]) * np.abs(b[i].astype(np.float64)).sum(-1) * np.abs(a[i].astype(np.float64) @ x[m].astype(np.float64)).max() * 2.0 ** -13
    bound = HALF * np.abs(want) + 2 * HALF * spread + low + 2.0 ** -24
    assert np.max(np.abs(got.astype(np.float64) - want) - bound) <= 0
    none = [m for m, i in enumerate(ids) if not 0 <= i < a.shape[0]]
    assert np.array_equal(got[none].view(np.uint16), y[none].view(np.uint16))


@gpu
@pytest.mark.parametrize("M,K,N,rank,count", [(1, 32, 1, 8, 1), (1, 4096, 6144, 16, 3), (3, 96, 40, 8, 2), (16, 512, 100, 24, 5), (17, 2304, 257, 32, 4),
                                              (40, 1024, 128, 64, 7), (64, 4096, 1000, 16, 40), (130, 160, 33, 128, 3), (300, 288, 264, 72, 2), (33, 14336, 72, 16, 33)])
def test_adapters(M, K, N, rank, count):
    rng = np.random.default_rng(31)
    a, b, scale = _adapters(rng, count, rank, K, N)
    x, y = _normal(rng, M, K), _normal(rng, M, N)
    ids = rng.integers(-1, count + 1, M).astype(np.int32)
    for alias in (False, True):
        _check_adapters(_add(x, ids, a, b, scale, y, alias), x, ids, a, b, scale, y)
    ids = np.sort(ids)  # requests one behind the other
    _check_adapters(_add(x, ids, a, b, scale, y), x, ids, a, b, scale, y)


@gpu
def test_adapters_do_not_reach_other_rows():
    """An adapter, a row of x and a row of y that are not finite change their own rows only."""
    rng = np.random.default_rng(32)
    M, K, N, rank, count = 20, 256, 72, 16, 4
    a, b, scale = _adapters(rng, count, rank, K, N)
    x, y = _normal(rng, M, K), _normal(rng, M, N)
    ids = (np.arange(M) % (count + 1) - 1).astype(np.int32)
    clean = _add(x, ids, a, b, scale, y)
    a[2], b[1, 5], scale[3] = np.inf, np.nan, np.inf
    x[4], y[9] = np.nan, np.inf
    got = _add(x, ids, a, b, scale, y)
    for m in range(M):
        if m in (4, 9) or ids[m] in (2, 3):
            continue
        same = np.ones(N, dtype=bool)
        if ids[m] == 1:
            same[5] = False
        assert np.array_equal(got[m, same].view(np.uint16), clean[m, same].view(np.uint16)), m


@gpu
def test_adapters_extreme_ids_and_sizes_of_values():
    rng = np.random.default_rng(33)
    M, K, N, rank, count = 24, 128, 64, 8, 2
    a, b, scale = _adapters(rng, count, rank, K, N)
    ids = np.asarray([np.iinfo(np.int32).min, np.iinfo(np.int32).max, -1, 2, 0, 1] * 4, dtype=np.int32)
    # low-rank values beyond binary16's range, brought back by a small scale; and tiny ones
    x, y = (_normal(rng, M, K).astype(np.float32) * 3000).astype(np.float16), _normal(rng, M, N)
    a[0] = (a[0].astype(np.float32) * 500).astype(np.float16)
    a[1] = (a[1].astype(np.float32) * 2.0 ** -9).astype(np.float16)
    scale[0] = 1e-6
    _check_adapters(_add(x, ids, a, b, scale, y), x, ids, a, b, scale, y)


# ---------------------------------------------------------------- the run of them
@gpu
@pytest.mark.parametrize("S,n", [([1, 1, 1, 1], [40, 129, 1, 700]), ([20, 1, 70], [20, 300, 100])])
def test_layer_of_a_batch_of_requests(S, n):
    """QKV layer and adapters, rotation and append, attention, O layer and adapters: each step against the oracle on the step before's own result."""
    rng = np.random.default_rng(41)
    h_q, h_kv, d, hidden = 8, 2, 64, 512
    T, batch = sum(S), len(S)
    fcs = [synth.FC("qkv", hidden, (h_q + 2 * h_kv) * d, "w4g32"), synth.FC("o", h_q * d, hidden, "w8c")]
    layers = [B.QuantLinear(*synth.weights(9300, 0, i, fc), fc.fmt, max_m=T) for i, fc in enumerate(fcs)]
    ads = [_adapters(rng, 3, 16, fc.K, fc.N) for fc in fcs]
    ids = np.repeat(np.arange(batch) % 4 - 1, S).astype(np.int32)
    table, num = _pages(rng, n)
    past = [m - s for s, m in zip(S, n)]
    rotary = B.make_rotary(d, 10000.0)
    angles = B.qfc_rotary_table(rotary, max(n))
    cache, K, V, P = _filled(rng, past, h_kv, d, table, num)
    req = _requests(S, n, table)
    x = _normal(rng, T, hidden)

    def layer(i, x):
        y = layers[i].forward(_t(x))
        torch.cuda.synchronize()
        y = y.cpu().numpy()
        out = _add(x, ids, *ads[i], y)
        _check_adapters(out, x, ids, *ads[i], y)
        return out

    qkv = layer(0, x)
    q = torch.empty((T, h_q * d), dtype=torch.float16, device=DEV)
    B.qfc_append_q4(_t(qkv), req, h_q, rotary, angles, cache, q)
    q = q.cpu().numpy()
    got = _attend(req, q, h_q, cache)
    heads = qkv.reshape(T, -1, d)
    pos = np.concatenate([np.arange(a, b) for a, b in zip(past, n)])
    turned = ref.rotate(heads[:, :h_q + h_kv], angles.cpu().numpy()[pos], False)
    assert np.array_equal(q.reshape(T, h_q, d), turned[:, :h_q])
    k_new, (v_new, p_new) = ref.q4_values(*ref.q4(turned[:, h_q:]))[0], ref.q4_values(*ref.q4(heads[:, h_q + h_kv:]))
    at = 0
    for b, s in enumerate(S):
        rows = slice(at, at + s)
        join = lambda old, new: np.concatenate([old[b], new[rows]])
        want = ref.attention(q.reshape(T, h_q, d)[rows], join(K, k_new), join(V, v_new), join(P, p_new))
        _close(got[rows].reshape(s, h_q, d), *want)
        at += s
    out = layer(1, got.astype(np.float16))
    assert out.shape == (T, hidden) and np.all(np.isfinite(out))
    for l in layers:
        l.close()


@gpu
def test_prompts_in_a_replayed_graph():
    """Which requests have many rows, and how long their walks are, may change from replay to replay."""
    rng = np.random.default_rng(29)
    h_q, h_kv, d, T, longest = 8, 2, 64, 400, 1024
    table, num = _pages(rng, [longest] * 3)
    cache, _, _, _ = _filled(rng, [longest] * 3, h_kv, d, table, num)
    start, context = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    req = B.Requests(start, context, _t(table), T, T, longest)
    q = _t(_normal(rng, T, h_q * d))
    ws, ws2 = (torch.empty(B.qfc_attention_q4_workspace_size(req, h_q, cache), dtype=torch.uint8, device=DEV) for _ in range(2))
    out, out2 = torch.zeros_like(q), torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    B.qfc_attention_q4(q, req, h_q, cache, ws2, out2)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.qfc_attention_q4(q, req, h_q, cache, ws, out)
    for cuts, n in (([0, 300, 301, 400], [1000, 5, 1024]), ([0, 1, 2, 3], [64, 65, 1]), ([0, 65, 400, 400], [65, 1023, 0]), ([0, 0, 200, 399], [9, 200, 1024])):
        start.copy_(torch.tensor(cuts, dtype=torch.int32))
        context.copy_(torch.tensor(n, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        out2.zero_()
        B.qfc_attention_q4(q, req, h_q, cache, ws2, out2)
        torch.cuda.synchronize()
        assert torch.equal(out[:cuts[-1]], out2[:cuts[-1]]) and bool(torch.isfinite(out2).all())


def _check_some(req, got, q, S, n, h_q, K, V, P, which):
    """Requests `which` of an attention's result."""
    first, d = np.concatenate([[0], np.cumsum(S)]), K[0].shape[-1]
    for b in which:
        rows = slice(first[b], first[b + 1])
        want = ref.attention(q.reshape(-1, h_q, d)[rows], K[b], V[b], P[b])
        _close(got.reshape(-1, h_q, d)[rows], *want)


@gpu
@pytest.mark.parametrize("batch,longest,h_q,h_kv,d", [(130, 700, 4, 2, 64), (300, 200, 4, 1, 128), (100, 1500, 16, 8, 128), (90, 1900, 8, 8, 64)])
def test_attention_of_more_requests_than_a_wavefront_has_lanes(batch, longest, h_q, h_kv, d):
    """Single tokens, chunks and empty requests among them, few pages per wavefront and more than four; every request against the oracle."""
    rng = np.random.default_rng(51)
    n = [int(x) for x in rng.integers(1, longest + 1, batch)]
    S = [int(min(rng.choice([1, 1, 1, 0, 3]), m)) for m in n]
    S[5], n[5], n[64], S[64] = 1, 1, 1, 1
    table, num = _pages(rng, n)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num)
    q, req = _normal(rng, sum(S), h_q * d), _requests(S, n, table)
    got = _attend(req, q, h_q, cache)
    _check_some(req, got, q, S, n, h_q, K, V, P, range(batch))


@gpu
def test_prompts_among_many_requests():
    """More requests than the first kernel's threads, prompts before and behind the 256th."""
    rng = np.random.default_rng(52)
    batch, h_q, h_kv, d = 270, 4, 1, 64
    n = [int(x) for x in rng.integers(1, 90, batch)]
    S = [1] * batch
    for b, s in ((0, 140), (3, 90), (200, 33), (255, 129), (256, 150), (269, 100)):
        S[b], n[b] = s, s + b % 70
    table, num = _pages(rng, n)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num)
    q, req = _normal(rng, sum(S), h_q * d), _requests(S, n, table)
    _check_some(req, _attend(req, q, h_q, cache), q, S, n, h_q, K, V, P, range(batch))


@gpu
@pytest.mark.parametrize("least", [7, 70, 300])
def test_attention_of_long_walks(least):
    """Wavefronts that take more pages than a wavefront holds page numbers; the limits above the real lengths."""
    rng = np.random.default_rng(53)
    h_q, h_kv, d, n, S = 4, 1, 64, [9000, 4470, 64], [1, 2, 1]
    table, num = _pages(rng, n, width=200)
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num)
    q, req = _normal(rng, sum(S), h_q * d), _requests(S, n, table, max_tokens=4, max_context=200 * 64)
    try:
        B.lib().qfc_tune(15, least)
        got = _attend(req, q, h_q, cache)
    finally:
        B.lib().qfc_tune(15, 0)
    _check_some(req, got, q, S, n, h_q, K, V, P, range(3))


@gpu
def test_requests_that_share_pages():
    """A common beginning held once: pages in several requests' rows of the table."""
    rng = np.random.default_rng(54)
    h_q, h_kv, d, common, n = 8, 2, 128, 256, [300, 420, 257]
    table, num = _pages(rng, n)
    table[:, :common // 64] = table[0, :common // 64]
    k, v = _normal(rng, sum(n), h_kv, d), _normal(rng, sum(n), h_kv, d)
    at = np.concatenate([[0], np.cumsum(n)])
    for x in (k, v):
        for b in (1, 2):
            x[at[b]:at[b] + common] = x[:common]
    cache, K, V, P = _filled(rng, n, h_kv, d, table, num, k, v)
    q, req = _normal(rng, 3, h_q * d), _requests([1] * 3, n, table)
    _check_some(req, _attend(req, q, h_q, cache), q, [1] * 3, n, h_q, K, V, P, range(3))


@gpu
def test_single_tokens_on_two_streams_at_once():
    rng = np.random.default_rng(55)
    h_q, h_kv, d, n = 8, 2, 128, [2000, 1500, 900]
    table, num = _pages(rng, n)
    cache, _, _, _ = _filled(rng, n, h_kv, d, table, num)
    q, req = [_normal(rng, 3, h_q * d) for _ in range(2)], _requests([1] * 3, n, table)
    alone = [_attend(req, x, h_q, cache) for x in q]
    size = B.qfc_attention_q4_workspace_size(req, h_q, cache)
    dev = [_t(x) for x in q]
    out, ws, streams = [torch.zeros_like(x) for x in dev], [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in q], [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                B.qfc_attention_q4(dev[i], req, h_q, cache, ws[i], out[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert np.array_equal(out[i].cpu().numpy().astype(np.float64), alone[i])


@gpu
def test_calls_without_tokens_and_with_wrong_tensors():
    rng = np.random.default_rng(56)
    table, num = _pages(rng, [64])
    cache = B.PagedCache(num, 1, 64)
    half = lambda *shape: torch.zeros(shape, dtype=torch.float16, device=DEV)
    none = B.Requests(_t(np.zeros(2, dtype=np.int32)), _t(np.asarray([64], dtype=np.int32)), _t(table), 0, 1, 64)
    B.qfc_append_q4(half(0, 4 * 64), none, 2, None, None, cache, half(0, 2 * 64))
    B.qfc_read_q4(none, cache, half(0, 1, 64), half(0, 1, 64))
    ws = torch.empty(max(B.qfc_attention_q4_workspace_size(none, 2, cache), 1), dtype=torch.uint8, device=DEV)
    B.qfc_attention_q4(half(0, 2 * 64), none, 2, cache, ws, half(0, 2 * 64))
    req = _requests([1], [64], table)
    size = B.qfc_attention_q4_workspace_size(req, 2, cache)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    for q, w, out in ((half(1, 64), ws, half(1, 128)), (half(1, 128).float(), ws, half(1, 128)), (half(1, 128), ws, half(2, 128)), (half(1, 256)[:, ::2], ws, half(1, 128)),
                      (torch.zeros((1, 128), dtype=torch.float16), ws, half(1, 128))):
        with pytest.raises(ValueError):
            B.qfc_attention_q4(q, req, 2, cache, w, out)
    with pytest.raises(B.QfcError):
        B.qfc_attention_q4(half(1, 128), req, 2, cache, ws[:size - 1], half(1, 128))
    rotary = B.make_rotary(64, 10000.0)
    with pytest.raises(B.QfcError):  # angles for fewer positions than the requests may have
        B.qfc_append_q4(half(1, 4 * 64), req, 2, rotary, B.qfc_rotary_table(rotary, 63), cache, half(1, 128))
    with pytest.raises(ValueError):
        B.PagedCache(2, 1, 64, pages=torch.zeros(100, dtype=torch.uint8, device=DEV))


@gpu
@pytest.mark.parametrize("M,K,N,rank,count", [(513, 128, 1000, 16, 6), (700, 160, 257, 64, 3), (640, 64, 6144, 8, 2), (1030, 96, 520, 128, 40), (2048, 256, 8200, 32, 5), (576, 64, 32, 40, 1)])
def test_adapters_of_many_rows(M, K, N, rank, count):
    """Blocks of many rows: whole and cut ones, one adapter and many in a block, none in some, tiles that the columns end inside of."""
    rng = np.random.default_rng(34)
    a, b, scale = _adapters(rng, count, rank, K, N)
    x, y = _normal(rng, M, K), _normal(rng, M, N)
    for ids in (np.full(M, count - 1), np.sort(rng.integers(-1, count, M)), rng.integers(0, count, M), rng.integers(-1, count + 1, M), np.repeat([0, -1, count - 1], [300, 100, M - 400])):
        ids = ids.astype(np.int32)
        got = _add(x, ids, a, b, scale, y)
        _check_adapters(got, x, ids, a, b, scale, y)
        assert np.array_equal(got, _add(x, ids, a, b, scale, y, alias=True))


@gpu
@pytest.mark.parametrize("M,N", [(700, 512), (700, 1000)])
def test_adapters_of_many_rows_do_not_reach_other_rows(M, N):
    rng = np.random.default_rng(35)
    K, rank, count = 64, 16, 4
    a, b, scale = _adapters(rng, count, rank, K, N)
    x, y = _normal(rng, M, K), _normal(rng, M, N)
    ids = (np.arange(M) // 7 % count).astype(np.int32)
    clean = _add(x, ids, a, b, scale, y)
    a[2], b[1, 5], scale[3] = np.inf, np.nan, np.inf
    x[4], y[9] = np.nan, np.inf
    got = _add(x, ids, a, b, scale, y)
    same = (ids < 2)[:, None] & ~((ids == 1)[:, None] & (np.arange(N) == 5))
    same[[4, 9]] = False
    assert np.array_equal(got.view(np.uint16)[same], clean.view(np.uint16)[same])


@gpu
@pytest.mark.parametrize("M", [1, 48, 600])
def test_adapters_in_a_replayed_graph(M):
    """Rows and adapters that change from replay to replay; the output in place of the layer's."""
    rng = np.random.default_rng(36)
    K, N, rank, count = 512, 264, 16, 5
    ad = B.Adapters(*(_t(t) for t in _adapters(rng, count, rank, K, N)))
    x, y, ids = torch.zeros((M, K), dtype=torch.float16, device=DEV), torch.zeros((M, N), dtype=torch.float16, device=DEV), torch.zeros(M, dtype=torch.int32, device=DEV)
    ws, ws2 = (torch.empty(B.qfc_adapters_workspace_size(ad, M), dtype=torch.uint8, device=DEV) for _ in range(2))
    out = torch.empty_like(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.qfc_add_adapters(x, ids, ad, y, ws2, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.qfc_add_adapters(x, ids, ad, y, ws, y)
    for _ in range(4):
        x.copy_(_t(_normal(rng, M, K)))
        y.copy_(_t(_normal(rng, M, N)))
        ids.copy_(_t(rng.integers(-1, count + 1, M).astype(np.int32)))
        B.qfc_add_adapters(x, ids, ad, y, ws2, out)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), y.view(torch.int16))


@gpu
def test_append_of_a_batch_is_append_one_by_one():
    """Requests whose rows begin inside a tile, positions that begin inside a dword."""
    rng = np.random.default_rng(57)
    h_q, h_kv, d, S = 2, 1, 128, [5, 6, 1, 70]
    n = [5, 70, 64, 133]
    table, num = _pages(rng, n)
    qkv = _normal(rng, sum(S), (h_q + 2 * h_kv) * d)
    caches = [B.PagedCache(num, h_kv, d) for _ in range(2)]
    for c in caches:
        c.pages.fill_(0x5A)
    out = torch.empty((sum(S), h_q * d), dtype=torch.float16, device=DEV)
    B.qfc_append_q4(_t(qkv), _requests(S, n, table), h_q, None, None, caches[0], out)
    at = 0
    for b, s in enumerate(S):  # one request at a time
        B.qfc_append_q4(_t(qkv[at:at + s]), _requests([s], [n[b]], table[b:b + 1]), h_q, None, None, caches[1], torch.empty((s, h_q * d), dtype=torch.float16, device=DEV))
        at += s
    assert torch.equal(caches[0].pages, caches[1].pages) and np.array_equal(out.cpu().numpy(), qkv[:, :h_q * d])
