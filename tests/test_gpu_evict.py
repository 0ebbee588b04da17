"""patchkv_evict_select and patchkv_cache_gather against plain references; a cache that is filled, weighed, cut down and used on."""
import ctypes as C

import numpy as np
import pytest
import torch

from live_common import BF16, F16, Case, Layout, attention64, build_tables, device_batch, random_rows
from rotary_common import HALF, INTERLEAVED, frequencies, rotate64, rotation_tolerance

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pk():
    from paper_2609_26219_b200 import build, binding
    build.build()
    return binding


@pytest.fixture(scope="module")
def ctx(pk):
    c = pk.Context(device=0)
    yield c
    c.close()


def chosen(mass, n, budget, recent, sinks):
    """The definition, by sorting."""
    if n <= budget:
        return list(range(n))
    last = min(recent, budget)
    first = min(sinks, budget - last)
    w = np.where(np.isfinite(mass) & (mass > 0), mass, 0.0)
    middle = sorted(range(first, n - last), key=lambda i: (-w[i], i))[:budget - last - first]
    return sorted(list(range(first)) + middle + list(range(n - last, n)))


def select(pk, ctx, mass, lengths, max_keep, recent, sinks, budget=None, status=0):
    n = len(lengths)
    m = torch.from_numpy(mass).to(DEV)
    keep = torch.full((n, max_keep), 77, dtype=torch.int32, device=DEV)
    kept = torch.full((n,), 77, dtype=torch.int32, device=DEV)
    out = torch.full((n, max_keep), -5.0, device=DEV)
    kv = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    b = None if budget is None else torch.tensor(budget, dtype=torch.int32, device=DEV)
    ctx.evict_select(m, kv, keep, kept, sinks=sinks, recent=recent, budget=b, mass_out=out)
    assert ctx.query_status() == status
    keep, kept, out = keep.cpu().numpy(), kept.cpu().numpy(), out.cpu().numpy()
    for s, t in enumerate(lengths):
        t = max(0, min(t, mass.shape[1]))
        have = max(0, min(max_keep if budget is None else budget[s], max_keep))
        want = chosen(mass[s], t, have, recent, sinks)
        assert kept[s] == len(want)
        assert keep[s, :len(want)].tolist() == want and np.all(keep[s, len(want):] == -1), s
        w = mass[s, want]
        assert np.array_equal(out[s, :len(want)], np.where(np.isfinite(w) & (w > 0), w, 0.0)) and np.all(out[s, len(want):] == -5.0)


@pytest.mark.parametrize("length", [1, 2, 31, 33, 1000, 1024, 1025, 4097, 8200, 20000, 70001])
@pytest.mark.parametrize("kind", ["tail", "ties", "equal", "zeros", "close"])
def test_select(pk, ctx, length, kind):
    rng = np.random.default_rng(length)
    lengths = [length, max(1, length // 2), length - 1, 0]
    m = np.exp(2 * rng.standard_normal((4, length + 3))).astype(np.float32)
    if kind == "ties":
        m = np.floor(m)
    if kind == "equal":
        m[:] = 0.75
    if kind == "zeros":
        m[:] = 0
        m[:, ::7] = -0.0
    if kind == "close":                                 # keys that differ in their last bits alone
        m = (1.0 + rng.integers(0, 64, m.shape) * 2.0 ** -23).astype(np.float32)
    for keep, recent, sinks in ((max(1, length // 3), 0, 0), (max(1, length - 1), 2, 1), (max(1, length // 2), length // 8, 4), (1, 5, 5), (length + 2, 3, 3),
                                (min(10, length), 6, 17)):
        select(pk, ctx, m, lengths, keep, recent, sinks)


def test_select_longer_than_what_shared_memory_holds(pk, ctx):
    n = 8 * 32768 + 5000
    rng = np.random.default_rng(0)
    m = np.floor(np.exp(3 * rng.standard_normal((1, n)))).astype(np.float32)
    select(pk, ctx, m, [n], n // 3, 1000, 4)
    select(pk, ctx, m, [n - 4321], 20, 0, 0)


def test_budgets_of_their_own(pk, ctx):
    rng = np.random.default_rng(3)
    m = rng.random((5, 3000)).astype(np.float32)
    select(pk, ctx, m, [3000, 2000, 10, 0, 999], 1500, 7, 3, budget=[1500, 1, 5, 4, 0])
    select(pk, ctx, m, [3000, 2000, 10, 0, 999], 1500, 7, 3, budget=[1501, -2, 5, 4, 8], status=pk.E_BOUNDS)


def test_lengths_out_of_range_and_bad_masses_are_latched(pk, ctx):
    rng = np.random.default_rng(4)
    m = rng.random((2, 500)).astype(np.float32)
    select(pk, ctx, m, [501, -3], 100, 7, 3, status=pk.E_BOUNDS)
    m[0, 100], m[0, 200], m[0, 300], m[0, 400] = np.nan, np.inf, -1.0, -0.0
    select(pk, ctx, m, [500, 500], 499, 0, 0, status=pk.E_BADINPUT)
    select(pk, ctx, m, [500, 500], 50, 0, 0, status=pk.E_BADINPUT)


def test_select_of_views_and_in_a_graph(pk, ctx):
    rng = np.random.default_rng(6)
    m = torch.from_numpy(rng.random((3, 700)).astype(np.float32)).to(DEV)
    wide = torch.zeros((3, 900), device=DEV)
    wide[:, :700] = m
    keep = torch.zeros((3, 300), dtype=torch.int32, device=DEV)
    kept, kv = torch.zeros(3, dtype=torch.int32, device=DEV), torch.tensor([700, 300, 5], dtype=torch.int32, device=DEV)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        ctx.evict_select(wide[:, :700], kv, keep[:, :200], kept, sinks=2, recent=3, stream=torch.cuda.current_stream())
    kv.copy_(torch.tensor([600, 700, 200], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    for s, n in enumerate((600, 700, 200)):
        assert keep[s, :200].tolist() == chosen(m[s].cpu().numpy(), n, 200, 3, 2)
    assert torch.all(keep[:, 200:] == 0) and ctx.query_status() == 0


def test_select_refusals(pk, ctx):
    m, kv = torch.zeros((2, 50), device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    keep, kept = torch.zeros((2, 10), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    for args, more in (((m, kv, keep, kv), {}), ((m, kv, keep, kept), dict(recent=-1)), ((m, kv, keep, kept), dict(sinks=-1)), ((m, kv, keep, kept), dict(mass_out=m)),
                       ((m, kv, keep, kept), dict(budget=kept))):
        with pytest.raises(pk.PatchKVError) as e:
            ctx.evict_select(*args, **more)
        assert e.value.code == pk.E_INVALID
    for args in ((m.double(), kv, keep, kept), (m, kv.long(), keep, kept), (m, kv, keep.long(), kept), (m.t(), kv, keep, kept), (m, kv, keep, kept[:1])):
        with pytest.raises(ValueError):
            ctx.evict_select(*args)
    a = pk.EvictArgs(C.sizeof(pk.EvictArgs), 1, (1 << 24) + 1, 1)
    a.mass_stride, a.keep_stride = 1 << 25, 1
    assert pk.lib().patchkv_evict_select(ctx._h, a, None) == pk.E_UNSUPPORTED
    assert pk.lib().patchkv_evict_select(ctx._h, None, None) == pk.E_INVALID


# ---------------------------------------------------------------- rows
GEOMETRIES = [(8, 128, 128, 16, 32), (4, 64, 64, 16, 32), (1, 256, 64, 32, 256), (3, 32, 32, 64, 16), (40, 128, 128, 16, 32), (2, 80, 80, 16, 16),
              (3, 10, 6, 5, 5), (1, 2, 2, 1, 1), (2, 64, 36, 16, 8)]


def gather(pk, ctx, tag, geometry, lengths, keeps, rotate=False, style=HALF, layer=0, layers=1, status=0, spoil=None):
    H, D, Dr, P, G = geometry
    rng = np.random.default_rng(8)
    most = max(1, max(-(-t // P) for t in lengths))
    cap = max(len(k) for k in keeps)
    to = max(1, -(-cap // P))
    n = len(lengths)
    n_pages = n * (most + to) + 2
    pages = rng.permutation(n_pages).astype(np.int32)
    src, dst = pages[:n * most].reshape(n, most).copy(), pages[n * most:n * (most + to)].reshape(n, to).copy()
    keep = np.full((n, cap + 1), -1, np.int32)
    for s, k in enumerate(keeps):
        keep[s, :len(k)] = k
    skipped = set()
    if spoil:
        spoil(src, dst, keep, skipped)
    geom = pk.make_geom(layers, H, D, Dr, style, 1e4, 16, P, G)
    if tag == 0:
        host = [torch.from_numpy(rng.standard_normal((layers, n_pages, P, H, D))).to(BF16) for _ in range(2)]
        dev = [x.to(DEV) for x in host]
        cache = pk.make_pool(dev[0], dev[1], n_pages, (n_pages * P * H * D, P * H * D, H * D, D))
    else:
        lay = Layout(tag, H, D, P, G)
        host = rng.integers(0, 256, (layers, n_pages, lay.page_bytes() + 16), dtype=np.uint8)
        dev = torch.from_numpy(host).to(DEV)
        cache = pk.make_qpool(dev, tag, n_pages)
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    ctx.cache_gather(geom, cache, layer, t(keep)[:, :cap], torch.tensor([len(k) for k in keeps], dtype=torch.int32, device=DEV),
                     torch.tensor(lengths, dtype=torch.int32, device=DEV), t(src), t(dst), rotate=rotate)
    assert ctx.query_status() == status
    theta = frequencies(Dr, 1e4)
    got = [x.cpu() for x in dev] if tag == 0 else dev.cpu().numpy()
    before = None if tag == 0 else host.copy()
    for s, k in enumerate(keeps):
        for i in range(len(k)):
            if (s, i) in skipped:
                continue
            old = int(keep[s, i])
            a, b = (src[s, old // P], old % P), (dst[s, i // P], i % P)
            if tag == 0:
                k0 = host[0][layer][a].double().numpy()[None]
                want = rotate64(k0, [i - old], theta, style)[0] if rotate else k0[0]
                tol = rotation_tolerance(k0, theta, style, 1.0, BF16)[0] if rotate and i != old else 0.0
                k1 = got[0][layer][b]
                assert np.all(np.abs(k1.double().numpy() - want) <= tol), (s, i)
                assert torch.equal(got[1][layer][b], host[1][layer][a])
                got[0][layer][b], got[1][layer][b] = host[0][layer][b], host[1][layer][b]      # then nothing else has changed
            else:
                off = 0
                for size in lay.sections():
                    row = size // P
                    host[layer, b[0], off + b[1] * row:off + (b[1] + 1) * row] = before[layer, a[0], off + a[1] * row:off + (a[1] + 1) * row]
                    off += size
    if tag == 0:
        assert torch.equal(got[0], host[0]) and torch.equal(got[1], host[1])
    else:
        assert np.array_equal(got, host)


def some(rng, n, k):
    return sorted(rng.permutation(n)[:k].tolist())


@pytest.mark.parametrize("tag", [0, 1, 2, 3])
@pytest.mark.parametrize("geometry", GEOMETRIES, ids=str)
def test_gather(pk, ctx, tag, geometry):
    rng = np.random.default_rng(1)
    lengths = [130, 1, 77, 40]
    keeps = [some(rng, 130, 61), [0], [], list(range(40))]
    for style in (HALF, INTERLEAVED):
        for rotate in ((False, True) if tag == 0 else (False,)):
            gather(pk, ctx, tag, geometry, lengths, keeps, rotate, style)
    gather(pk, ctx, tag, geometry, [300], [some(rng, 300, 3)], tag == 0, layer=1, layers=3)


def test_gather_many_rows(pk, ctx):
    rng = np.random.default_rng(2)
    for tag in (0, 3):
        gather(pk, ctx, tag, (8, 128, 128, 16, 32), [3000, 2500], [some(rng, 3000, 1100), some(rng, 2500, 999)], tag == 0)


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("geometry", [(8, 128, 128, 16, 32), (2, 80, 80, 16, 16)], ids=str)
def test_rows_out_of_range_are_skipped(pk, ctx, tag, geometry):
    def position(src, dst, keep, skipped):
        keep[0, 3], keep[1, 0] = 60, -4
        skipped.update([(0, 3), (1, 0)])

    def page(src, dst, keep, skipped):
        src[0, 1], dst[1, 0] = -1, 10 ** 6
        skipped.update([(0, i) for i in range(20) if 16 <= keep[0, i] < 32] + [(1, i) for i in range(5)])

    for spoil in (position, page):
        gather(pk, ctx, tag, geometry, [60, 20], [list(range(0, 60, 3)), [1, 4, 8, 9, 19]], status=pk.E_BOUNDS, spoil=spoil)


def test_rows_that_stay_where_they_are(pk, ctx):
    """The first pages, which nothing has been taken out of, may be the destination's own."""
    H, D, P = 2, 64, 16
    rng = np.random.default_rng(3)
    k, v = (torch.from_numpy(rng.standard_normal((8, P, H, D))).to(BF16).to(DEV) for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    keep = list(range(32)) + [40, 41, 50]
    geom = pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, 32)
    ctx.cache_gather(geom, pk.make_pool(k, v, 8, (0, P * H * D, H * D, D)), 0, t([keep]), t([35]), t([60]), t([[5, 2, 7, 0]]), t([[5, 2, 4]]), rotate=True)
    assert ctx.query_status() == 0
    assert torch.equal(k[[5, 2, 7, 0]], k0[[5, 2, 7, 0]]) and torch.equal(v[4, :3], torch.stack([v0[7, 8], v0[7, 9], v0[0, 2]]))
    want = rotate64(k0[7, 8:9].double().cpu().numpy(), [32 - 40], frequencies(D, 1e4), HALF)
    assert np.all(np.abs(k[4, 0:1].double().cpu().numpy() - want) <= rotation_tolerance(k0[7, 8:9].double().cpu().numpy(), frequencies(D, 1e4), HALF, 1.0, BF16))


def test_kept_above_the_bound_is_cut(pk, ctx):
    H, D, P = 2, 64, 16
    k, v = (torch.randn((4, P, H, D), device=DEV).to(BF16) for _ in range(2))
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    geom = pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, 32)
    v0 = v.clone()
    ctx.cache_gather(geom, pk.make_pool(k, v, 4, (0, P * H * D, H * D, D)), 0, t([[3, 5]]), t([3]), t([30]), t([[0, 1]]), t([[2]]))
    assert ctx.query_status() == pk.E_BOUNDS
    assert torch.equal(v[2, :2], v0[0, [3, 5]]) and torch.equal(v[2, 2:], v0[2, 2:])


def test_gather_refusals(pk, ctx):
    lay = Layout(3, 2, 64, 16, 32)
    geom = pk.make_geom(1, 2, 64, 64, HALF, 1e4, 16, 16, 32)
    cache = pk.make_qpool(torch.zeros((4, lay.page_bytes()), dtype=torch.uint8, device=DEV), 3, 4)
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    args = (t([[3, 5]]), t([2]), t([30]), t([[0, 1]]), t([[2]]))
    with pytest.raises(pk.PatchKVError) as e:
        ctx.cache_gather(geom, cache, 0, *args, rotate=True)
    assert e.value.code == pk.E_UNSUPPORTED
    with pytest.raises(pk.PatchKVError) as e:
        ctx.cache_gather(geom, cache, 1, *args)
    assert e.value.code == pk.E_INVALID
    with pytest.raises(ValueError):
        ctx.cache_gather(geom, cache, 0, args[0].long(), *args[1:])
    with pytest.raises(ValueError):
        ctx.cache_gather(geom, cache, 0, args[0], args[1].long(), *args[2:])
    x = torch.zeros((4, 16, 2, 64), dtype=BF16, device=DEV)
    for v, strides in ((x, (0, 2048, 128, 64)), (x.clone(), (0, 2048, 64, 64)), (x.clone(), (0, 128, 128, 64))):
        with pytest.raises(pk.PatchKVError) as e:
            ctx.cache_gather(geom, pk.make_pool(x, v, 4, strides), 0, *args)
        assert e.value.code == pk.E_INVALID
    a = pk.GatherArgs(C.sizeof(pk.GatherArgs), 1, 1, 0, 1, 1, None, 1)
    assert pk.lib().patchkv_cache_gather(ctx._h, geom, None, cache, 0, a, None) == pk.E_INVALID
    assert pk.lib().patchkv_cache_gather(ctx._h, geom, None, None, 0, a, None) == pk.E_INVALID


# ---------------------------------------------------------------- all of it in turn
@pytest.mark.parametrize("tag", [0, 1, 3])
def test_a_cache_is_filled_weighed_cut_down_and_used_on(pk, ctx, tag):
    """Prompt rows in, their attention and the weight it gives, the tokens that stay, their rows into spare pages, one more token
    over what is left: against attention over the kept tokens' rows, in 64 bits.  Over the pool the keys move to their new positions,
    over quantised pages they stay at the old ones and the new token is rotated to where it stands in the text."""
    H, Hq, D, P, G, n, budget = 2, 8, 64, 16, 32, 200, 90
    rng = np.random.default_rng(12)
    geom = pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, G)
    theta = frequencies(D, 1e4)
    case = Case([n], [n])
    most = -(-n // P)
    n_pages = 2 * most + 2
    pages = rng.permutation(n_pages).astype(np.int32)
    table, spare = pages[:most].reshape(1, -1), pages[most:2 * most].reshape(1, -1)
    batch, held = device_batch(pk, case, table, DEV)
    if tag == 0:
        kp, vp = (torch.zeros((n_pages, P, H, D), dtype=BF16, device=DEV) for _ in range(2))
        cache = pk.make_pool(kp, vp, n_pages, (0, P * H * D, H * D, D))
    else:
        lay = Layout(tag, H, D, P, G)
        store = torch.zeros((n_pages, lay.page_bytes()), dtype=torch.uint8, device=DEV)
        cache = pk.make_qpool(store, tag, n_pages)
    k, v, q = (random_rows(rng, n, h, D, BF16).to(DEV) for h in (H, H, Hq))
    out = torch.empty_like(q)
    need = lambda b: torch.empty(max(16, pk.attention_workspace_bytes(geom, cache, b, Hq), pk.attention_mass_workspace_bytes(geom, cache, b, Hq)), dtype=torch.uint8, device=DEV)
    ctx.rotary_append(geom, cache, 0, batch, k, v, q=q)
    ctx.attention(geom, cache, 0, batch, q, out, workspace=need(batch))
    mass = torch.full((1, n), -1.0, device=DEV)
    ctx.attention_mass(geom, cache, 0, batch, q, mass, workspace=need(batch))
    keep, kept = torch.zeros((1, budget), dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ctx.evict_select(mass, held["kv"], keep, kept, sinks=2, recent=16)
    to = torch.from_numpy(spare).to(DEV)
    ctx.cache_gather(geom, cache, 0, keep, kept, held["kv"], torch.from_numpy(table).to(DEV), to, rotate=tag == 0)
    step = Case([budget + 1], [1])
    b1, held1 = device_batch(pk, step, spare, DEV)
    k1, v1, q1 = (random_rows(rng, 1, h, D, BF16).to(DEV) for h in (H, H, Hq))
    q0 = q1.clone()
    rope = torch.tensor([budget if tag == 0 else n], dtype=torch.int32, device=DEV)
    ctx.rotary_append(geom, cache, 0, b1, k1, v1, q=q1, rope_pos=rope)
    out1 = torch.empty_like(q1)
    ctx.attention(geom, cache, 0, b1, q1, out1, workspace=need(b1))
    assert ctx.query_status() == 0 and int(kept[0]) == budget

    # the masses, from the rows as they stand in the cache
    def rows(tb, count):
        if tag == 0:
            return [torch.cat([x[int(p)] for p in tb[0]])[:count].double().cpu().numpy() for x in (kp, vp)]
        host = store.cpu().numpy()
        both = [lay.values(host[p]) for p in tb[0]]
        return [np.concatenate([x[i] for x in both])[:count] for i in (0, 1)]

    K, V = rows(table, n)
    qd = q.double().cpu().numpy()
    want = np.zeros(n)
    for h in range(Hq):
        x = qd[:, h] @ K[:, h // (Hq // H)].T * D ** -0.5
        x[np.triu_indices(n, 1)] = -np.inf
        w = np.exp(x - x.max(1, keepdims=True))
        want += (w / w.sum(1, keepdims=True)).sum(0)
    got = mass[0].double().cpu().numpy()
    assert np.linalg.norm(got - want) <= 2e-5 * np.linalg.norm(want)
    assert keep[0].tolist() == chosen(mass[0].cpu().numpy(), n, budget, 16, 2)
    # the kept rows with the new one behind them
    kk, vv = rows(spare, budget + 1)
    idx = keep[0].cpu().numpy()
    assert np.array_equal(vv[:budget], V[idx])
    moved = rotate64(K[idx], np.arange(budget) - idx, theta, HALF) if tag == 0 else K[idx]
    assert np.all(np.abs(kk[:budget] - moved) <= (rotation_tolerance(K[idx], theta, HALF, 1.0, BF16) if tag == 0 else 0.0))
    turned = rotate64(q0.double().cpu().numpy(), [int(rope[0])], theta, HALF)
    assert np.all(np.abs(q1.double().cpu().numpy() - turned) <= rotation_tolerance(q0.double().cpu().numpy(), theta, HALF, 1.0, BF16))
    o, tol = attention64(q1.double().cpu().numpy(), lambda b: kk, lambda b: vv, step, Hq // H, D ** -0.5, 0, 0, BF16, tag == 0)
    assert np.all(np.abs(out1.double().cpu().numpy() - o) <= tol)
