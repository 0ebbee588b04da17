"""Pools that patchkv_rotary_append and patchkv_cache_gather write: K and V that share places are refused, K and V side by side in one
tensor are taken."""
import numpy as np
import pytest
import torch

from live_common import BF16, Case, build_tables, device_batch, random_rows
from rotary_common import HALF

pytestmark = pytest.mark.gpu
DEV, H, D, P, PAGES = "cuda:0", 2, 64, 16, 6


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


def layouts():
    """Name -> [K's offset, V's offset, strides of page, token, head]: K and V in one tensor, none of it shared."""
    return {"by_page": (0, P * H * D, 2 * P * H * D, H * D, D), "by_token": (0, H * D, 2 * P * H * D, 2 * H * D, D), "by_head": (0, D, 2 * P * H * D, 2 * H * D, 2 * D),
            "v_first": (P * H * D, 0, 2 * P * H * D, H * D, D), "heads_first": (0, P * D, 2 * P * H * D, D, 2 * P * D), "apart": (0, PAGES * P * H * D, P * H * D, H * D, D),
            "pages_inside": (0, D, 2 * D, 2 * PAGES * D, 2 * PAGES * P * D)}


def shared():
    """The same with some of V's places K's."""
    return {"same": (0, 0, P * H * D, H * D, D), "a_page_on": (0, P * H * D, P * H * D, H * D, D), "a_page_back": (P * H * D, 0, P * H * D, H * D, D),
            "a_head_on": (0, D, P * H * D, H * D, D), "half_a_row_on": (0, D // 2, 2 * P * H * D, 2 * H * D, 2 * D), "into_the_last_token": (0, P * H * D - 8, 2 * P * H * D, H * D, D),
            "two_tokens_on": (0, 4 * H * D, 2 * P * H * D, 2 * H * D, D), "into_the_next_page": (0, 2 * P * H * D - 8, 2 * P * H * D, H * D, D)}


def append(pk, ctx, store, k_at, v_at, strides):
    case = Case([40, 17], [9, 17])
    rng = np.random.default_rng(3)
    table, n_pages = build_tables(case, P, rng, spare=0)
    assert n_pages == PAGES
    batch, held = device_batch(pk, case, table, DEV)
    k, v = (random_rows(rng, 26, H, D, BF16).to(DEV) for _ in range(2))
    pool = pk.make_pool(store[k_at:], store[v_at:], PAGES, (0, *strides))
    ctx.rotary_append(pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, 32), pool, 0, batch, k, v)
    assert ctx.query_status() == 0
    return [store[at:].as_strided((PAGES, P, H, D), (*strides, 1)).cpu() for at in (k_at, v_at)]


def gather(pk, ctx, store, k_at, v_at, strides):
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    pool = pk.make_pool(store[k_at:], store[v_at:], PAGES, (0, *strides))
    ctx.cache_gather(pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, 32), pool, 0, t([[3, 20, 31]]), t([3]), t([40]), t([[0, 4, 2]]), t([[5]]), rotate=True)
    assert ctx.query_status() == 0
    return [store[at:].as_strided((PAGES, P, H, D), (*strides, 1)).cpu() for at in (k_at, v_at)]


def fresh():
    return torch.zeros(4 * PAGES * P * H * D, dtype=BF16, device=DEV)


@pytest.mark.parametrize("name", list(layouts()))
def test_side_by_side(pk, ctx, name):
    k_at, v_at, *strides = layouts()[name]
    plain = layouts()["apart"]
    for a, b in zip(append(pk, ctx, fresh(), k_at, v_at, strides), append(pk, ctx, fresh(), plain[0], plain[1], plain[2:])):
        assert torch.equal(a, b)
    gather(pk, ctx, fresh(), k_at, v_at, strides)


@pytest.mark.parametrize("name", list(shared()))
def test_shared_places_are_refused(pk, ctx, name):
    k_at, v_at, *strides = shared()[name]
    for call in (append, gather):
        with pytest.raises(pk.PatchKVError) as e:
            call(pk, ctx, fresh(), k_at, v_at, strides)
        assert e.value.code == pk.E_INVALID


def test_the_tables_against_sets_of_places():
    """Both tables above, by writing all places down."""
    for table, want in ((layouts(), False), (shared(), True)):
        for name, (k_at, v_at, *strides) in table.items():
            grid = sum(i * s for i, s in zip(np.ogrid[:PAGES, :P, :H, :D], (*strides, 1))).ravel()
            assert len(np.unique(grid)) == grid.size and bool(np.intersect1d(grid + k_at, grid + v_at).size) == want, name
            assert max(k_at, v_at) + grid.max() < 4 * PAGES * P * H * D
