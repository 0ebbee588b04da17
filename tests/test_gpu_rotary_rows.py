"""patchkv_rotary_append with entries of row_start out of order: which rows are left, over the pool and over quantised pages."""
import numpy as np
import pytest
import torch

from live_common import BF16, Case, Layout, build_tables, device_batch, random_rows
from rotary_common import HALF

pytestmark = pytest.mark.gpu
DEV, H, Hq, P = "cuda:0", 2, 4, 16


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


# row_start of two sequences over five rows -> rows that are left (of entries that descend: at least; they may take others with them).
STARTS = {"negative": ([0, -1, 5], [0, 1, 2, 3, 4]), "descending": ([0, 4, 2], [4]), "behind_the_rows": ([0, 3, 6], [3, 4]), "first_behind_zero": ([1, 3, 5], [0])}


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("D", [64, 80])
@pytest.mark.parametrize("name", list(STARTS))
def test_rows_of_bad_entries_are_left(pk, ctx, tag, D, name):
    start, left = STARTS[name]
    case = Case([40, 20], [3, 2], [[1, 20, 39], [10, 19]])
    rng = np.random.default_rng(9)
    table, n_pages = build_tables(case, P, rng)
    batch, held = device_batch(pk, case, table, DEV)
    held["start"].copy_(torch.tensor(start, dtype=torch.int32))
    held["pos"].copy_(torch.arange(5, dtype=torch.int32) + 3)
    geom = pk.make_geom(1, H, D, D, HALF, 1e4, 16, P, 16)
    k, v, q = (random_rows(rng, 5, h, D, BF16).to(DEV) for h in (H, H, Hq))
    out = torch.full_like(q, 7.0)
    if tag == 0:
        store = [torch.full((n_pages, P, H, D), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
        cache = pk.make_pool(store[0], store[1], n_pages, (0, P * H * D, H * D, D))
    else:
        pages = torch.zeros((n_pages, Layout(tag, H, D, P, 16).page_bytes()), dtype=torch.uint8, device=DEV)
        cache = pk.make_qpool(pages, tag, n_pages)
    ctx.rotary_append(geom, cache, 0, batch, k, v, q=q, q_out=out)
    assert ctx.query_status() == (0 if name == "first_behind_zero" else pk.E_BOUNDS)
    got = (out == 7.0).all(-1).all(-1).cpu()
    assert torch.equal((out == 7.0).any(-1).any(-1).cpu(), got)
    if name == "descending":
        assert got[left].all()
        left = got.nonzero()[:, 0].tolist()
    assert got.tolist() == [i in left for i in range(5)]
    if tag == 0:
        for x in store:
            assert int((x != 3.0).any(-1).any(-1).sum()) == 5 - len(left)
    else:
        lay = Layout(tag, H, D, P, 16)
        written = sum(int(np.frombuffer(lay.split(p)[1].tobytes(), np.uint16).reshape(P, -1).any(1).sum()) for p in pages.cpu().numpy())
        assert written == 5 - len(left)
