"""patchkv_rotary_append against a plain 64-bit reference: queries, bytes of whole pools, refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from live_common import BF16, F16, Case, Layout, build_tables, device_batch, random_rows
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


BATCHES = {
    "one_row": Case([1000], [1]),
    "ragged": Case([40, 17, 1, 90], [13, 17, 1, 2]),
    "empty_sequences": Case([5, 0, 33], [0, 0, 33]),
    "scattered": Case([70, 33], [4, 3], [[0, 15, 16, 69], [1, 2, 32]]),
}
# KV heads, query heads, D, rotary channels, page, group: those of the fast kernel, and others
GEOMETRIES = [(8, 32, 128, 128, 16, 32), (4, 8, 64, 64, 16, 32), (4, 28, 128, 64, 32, 64), (1, 5, 256, 96, 16, 256), (3, 3, 32, 32, 16, 16),
              (2, 6, 128, 0, 64, 128), (2, 2, 16, 16, 32, 16), (2, 4, 80, 80, 16, 16), (3, 1, 10, 6, 5, 5), (1, 2, 2, 2, 1, 1), (5, 7, 64, 36, 16, 8)]


def check(pk, ctx, tag, style, geometry, dtype, case, base=1e4, inv_freq=None, factor=1.0, far=None, q_in_place=False, with_q=True):
    H, Hq, D, Dr, P, G = geometry
    rng = np.random.default_rng(5)
    theta = frequencies(Dr, base) if inv_freq is None else inv_freq.double().numpy()
    table, n_pages = build_tables(case, P, rng)
    n, extra = sum(case.rows), 2
    batch, held = device_batch(pk, case, table, DEV, n_rows=n + extra)
    k, v, q = random_rows(rng, n + extra, H, D, dtype), random_rows(rng, n + extra, H, D, dtype, False), random_rows(rng, n + extra, Hq, D, dtype, False)
    flat = np.array([p for s in case.positions() for p in s], np.int64)
    turn = flat if far is None else far + np.arange(n) * 3 - 7
    rope = None if far is None else torch.tensor(np.concatenate([turn, [1] * extra]), dtype=torch.int32, device=DEV)
    geom = pk.make_geom(1, H, D, Dr, style, base, 16, P, G, inv_freq)
    kd, vd, qd = k[:n].double().numpy(), v[:n].double().numpy(), q[:n].double().numpy()
    turned = rotate64(kd, turn, theta, style, factor)
    if tag == 0:
        pools = [torch.from_numpy(rng.standard_normal((n_pages, P, H, D))).to(BF16) for _ in range(2)]
        dev = [x.to(DEV) for x in pools]
        cache = pk.make_pool(dev[0], dev[1], n_pages, (n_pages * P * H * D, P * H * D, H * D, D))
    else:
        lay = Layout(tag, H, D, P, G)
        pages = rng.integers(0, 256, (n_pages, lay.page_bytes()), dtype=np.uint8)
        dev = torch.from_numpy(pages).to(DEV)
        cache = pk.make_qpool(dev, tag, n_pages)
    q_dev = q.to(DEV)
    out = q_dev if q_in_place else torch.full_like(q_dev, 7.0)
    ctx.rotary_append(geom, cache, 0, batch, k.to(DEV), v.to(DEV), q=q_dev if with_q else None, q_out=out if with_q else None, rope_pos=rope, rope_factor=factor)
    assert ctx.query_status() == 0
    if with_q:
        want, tol = rotate64(qd, turn, theta, style, factor), rotation_tolerance(qd, theta, style, factor, dtype)
        got = out.cpu()
        assert np.all(np.abs(got[:n].double().numpy() - want) <= tol)
        assert torch.equal(got[n:], q[n:] if q_in_place else torch.full_like(q[n:], 7.0))
    r = 0
    if tag == 0:
        tol = rotation_tolerance(kd, theta, style, factor, BF16)
        got = [x.cpu() for x in dev]
        for b, positions in enumerate(case.positions()):
            for pos in positions:
                at = (table[b, pos // P], pos % P)
                assert np.all(np.abs(got[0][at].double().numpy() - turned[r]) <= tol[r])
                assert torch.equal(got[1][at], v[r])
                pools[0][at], pools[1][at] = got[0][at], v[r]
                r += 1
        assert torch.equal(got[0], pools[0]) and torch.equal(got[1], pools[1])          # all other slots
    else:
        for b, positions in enumerate(case.positions()):
            for pos in positions:
                lay.put(pages[table[b, pos // P]], pos % P, turned[r], vd[r])
                r += 1
        assert np.array_equal(dev.cpu().numpy(), pages)


@pytest.mark.parametrize("tag", [0, 1, 2, 3])
@pytest.mark.parametrize("style", [HALF, INTERLEAVED], ids=["half", "interleaved"])
@pytest.mark.parametrize("geometry", GEOMETRIES, ids=str)
@pytest.mark.parametrize("name", list(BATCHES))
def test_rows(pk, ctx, tag, style, geometry, name):
    for dtype in (BF16, F16):
        if tag or dtype is BF16:
            check(pk, ctx, tag, style, geometry, dtype, BATCHES[name])


@pytest.mark.parametrize("tag", [0, 1, 3])
@pytest.mark.parametrize("style", [HALF, INTERLEAVED], ids=["half", "interleaved"])
def test_far_positions_given_frequencies_and_a_factor(pk, ctx, tag, style):
    for D, Dr in ((128, 128), (128, 64), (80, 40)):
        inv = torch.from_numpy(frequencies(Dr, 5e5) / np.linspace(1, 8, Dr // 2)).float()
        for far in (100000, 2 ** 30, -50):
            check(pk, ctx, tag, style, (2, 4, D, Dr, 16, 16), BF16, BATCHES["ragged"], inv_freq=inv, factor=1.3, far=far)


def test_queries_in_place_and_without(pk, ctx):
    for tag in (0, 3):
        for geometry in ((8, 32, 128, 128, 16, 32), (2, 4, 80, 80, 16, 16)):
            check(pk, ctx, tag, HALF, geometry, BF16, BATCHES["ragged"], q_in_place=True)
            check(pk, ctx, tag, INTERLEAVED, geometry, BF16, BATCHES["ragged"], with_q=False)


def test_many_rows(pk, ctx):
    for tag in (0, 2):
        check(pk, ctx, tag, HALF, (8, 8, 128, 128, 16, 32), BF16, Case([700, 333], [650, 333]))


def test_strided_rows_of_one_projection(pk, ctx):
    """q, k and v as slices of one projection's output, and heads first."""
    H, Hq, D, n = 2, 6, 64, 21
    rng = np.random.default_rng(2)
    case = Case([30], [n])
    table, n_pages = build_tables(case, 16, rng)
    batch, held = device_batch(pk, case, table, DEV)
    wide = torch.from_numpy(rng.standard_normal((n, Hq + 2 * H, D))).to(BF16).to(DEV)
    geom = pk.make_geom(1, H, D, D, HALF, 1e4, 16, 16, 32)
    results = []
    for make in (lambda x: x, lambda x: x.contiguous(), lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)):
        q, k, v = make(wide[:, :Hq]), make(wide[:, Hq:Hq + H]), make(wide[:, Hq + H:])
        kp, vp = (torch.zeros((n_pages, 16, H, D), dtype=BF16, device=DEV) for _ in range(2))
        out = torch.empty((Hq, n, D + 8), dtype=BF16, device=DEV).transpose(0, 1)[..., :D]
        ctx.rotary_append(geom, pk.make_pool(kp, vp, n_pages, (0, 16 * H * D, H * D, D)), 0, batch, k, v, q=q, q_out=out)
        assert ctx.query_status() == 0
        results.append((out.cpu().clone(), kp.cpu(), vp.cpu()))
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[0]))


def test_skipped_rows_are_latched_and_left(pk, ctx):
    H, Hq, D, P = 2, 4, 64, 16
    geom = pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, 32)
    rng = np.random.default_rng(9)
    for what in ("page", "position", "descending", "row_start"):
        case = Case([40, 20], [3, 2], [[1, 20, 39], [0, 19]])
        table, n_pages = build_tables(case, P, rng)
        if what == "page":
            table[0, 1] = n_pages
        if what == "position":
            case.pos[0][1] = 40
        if what == "descending":
            case.pos[0] = [1, 39, 20]
        batch, held = device_batch(pk, case, table, DEV)
        if what == "row_start":
            held["start"][1] = -1
        n = 5
        k, v, q = (random_rows(rng, n, h, D, BF16).to(DEV) for h in (H, H, Hq))
        kp, vp = (torch.full((n_pages, P, H, D), 3.0, dtype=BF16, device=DEV) for _ in range(2))
        out = torch.full_like(q, 7.0)
        ctx.rotary_append(geom, pk.make_pool(kp, vp, n_pages, (0, P * H * D, H * D, D)), 0, batch, k, v, q=q, q_out=out)
        assert ctx.query_status() == pk.E_BOUNDS
        # (behind a row at position 40, which the cache does not have, one at 39 descends)
        left = {"page": [1], "position": [1, 2], "descending": [2], "row_start": [0, 1, 2, 3, 4]}[what]
        got = (out == 7.0).all(-1).all(-1).cpu()
        if what != "row_start":
            assert got.tolist() == [i in left for i in range(n)], what
        assert (vp != 3.0).any(-1).any(-1).sum() == (~got).sum()


def test_replay_with_other_rows_and_two_streams(pk, ctx):
    H, Hq, D, P = 8, 32, 128, 16
    geom = pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, 32)
    rng = np.random.default_rng(1)
    case = Case([100, 90], [4, 1])
    table, n_pages = build_tables(case, P, rng)
    batch, held = device_batch(pk, case, table, DEV)
    k, v, q = (random_rows(rng, 5, h, D, BF16).to(DEV) for h in (H, H, Hq))
    kp, vp = (torch.zeros((n_pages, P, H, D), dtype=BF16, device=DEV) for _ in range(2))
    pool = pk.make_pool(kp, vp, n_pages, (0, P * H * D, H * D, D))
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            ctx.rotary_append(geom, pool, 0, batch, k, v, q=q, q_out=out, stream=torch.cuda.current_stream())
    q.copy_(random_rows(rng, 5, Hq, D, BF16))
    held["kv"].copy_(torch.tensor([77, 60], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    want = rotate64(q.cpu().double().numpy(), [73, 74, 75, 76, 59], frequencies(D, 1e4), HALF)
    tol = rotation_tolerance(q.cpu().double().numpy(), frequencies(D, 1e4), HALF, 1.0, BF16)
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= tol)
    assert torch.equal(vp[int(table[1, 59 // P]), 59 % P], v[4]) and ctx.query_status() == 0


def test_refusals(pk, ctx):
    H, D, P = 2, 64, 16
    case = Case([10], [2])
    table, n_pages = build_tables(case, P, np.random.default_rng(0))
    batch, held = device_batch(pk, case, table, DEV)
    k, q = torch.zeros((2, H, D), dtype=BF16, device=DEV), torch.zeros((2, 4, D), dtype=BF16, device=DEV)
    kp = torch.zeros((n_pages, P, H, D), dtype=BF16, device=DEV)
    pool = pk.make_pool(kp, kp.clone(), n_pages, (0, P * H * D, H * D, D))
    ok = lambda **m: pk.make_geom(1, H, D, m.get("Dr", D), m.get("style", HALF), m.get("base", 1e4), 16, P, 32, m.get("inv"))

    def refused(code, geom, *args, **more):
        with pytest.raises(pk.PatchKVError) as e:
            ctx.rotary_append(geom, *args, **more)
        assert e.value.code == code, e.value

    refused(pk.E_INVALID, ok(Dr=D + 2), pool, 0, batch, k, k)
    refused(pk.E_INVALID, ok(Dr=3), pool, 0, batch, k, k)
    refused(pk.E_INVALID, ok(style=2), pool, 0, batch, k, k)
    refused(pk.E_INVALID, ok(base=0.0), pool, 0, batch, k, k)
    refused(pk.E_INVALID, ok(inv=torch.full((D // 2,), float("nan"))), pool, 0, batch, k, k)
    refused(pk.E_INVALID, ok(), pool, 1, batch, k, k)
    refused(pk.E_INVALID, ok(), pool, 0, batch, k.half(), k.half())
    refused(pk.E_INVALID, ok(), pool, 0, batch, k, k, rope_factor=float("inf"))
    refused(pk.E_INVALID, ok(), pool, 0, batch, k, k, q=q, q_out=q[:1].expand(2, 4, D))
    refused(pk.E_INVALID, ok(), pool, 0, batch, k, k, q=q, q_out=q.as_strided((2, 4, D), (D, 2 * D, 1)))
    for bad in (dict(q=q.half()), dict(q=q, q_out=q[:, :2]), dict(q_out=q), dict(q=q, rope_pos=torch.zeros(1, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            ctx.rotary_append(ok(), pool, 0, batch, k, k, **bad)
    for strides in ((0, P * H * D, H * D, 0), (0, P * H * D, D, D), (0, H * D, H * D, D), (0, 0, H * D, D), (0, P * H * D - 8, H * D, D), (0, D, H * D, 2 * D)):
        refused(pk.E_INVALID, ok(), pk.make_pool(kp, kp.clone(), n_pages, strides), 0, batch, k, k)
    refused(pk.E_INVALID, ok(), pk.make_pool(kp, kp, n_pages, (0, P * H * D, H * D, D)), 0, batch, k, k)
    lib = pk.lib()
    a = pk.RotaryArgs(C.sizeof(pk.RotaryArgs))
    assert lib.patchkv_rotary_append(ctx._h, ok(), None, None, 0, batch, a, None) == pk.E_INVALID
    assert lib.patchkv_rotary_append(ctx._h, ok(), pool, None, 0, batch, a, None) == pk.E_INVALID       # null k and v
    a.struct_size = 8
    assert lib.patchkv_rotary_append(ctx._h, ok(), pool, None, 0, batch, a, None) == pk.E_INVALID
    empty, held = device_batch(pk, Case([10], [0]), table, DEV)
    none = torch.zeros((0, H, D), dtype=BF16, device=DEV)
    assert ctx.rotary_append(ok(), pool, 0, empty, none, none) == 0
