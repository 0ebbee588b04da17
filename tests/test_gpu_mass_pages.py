"""patchkv_attention_mass with pages out of range, by the kernels of many query vectors: tokens that a row sees on such a page are left out of
its sum, get no weight, and latch PATCHKV_E_BOUNDS; all others have the weights of the 64-bit formula."""
import numpy as np
import pytest
import torch

from live_common import BF16, Case
from test_gpu_mass import DEV, Run

pytestmark = pytest.mark.gpu


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


def lose(run, pages):
    """Takes pages (sequence, logical page) out of the block table; the keys of their tokens are not there then."""
    table = run.held["table"].cpu().numpy()
    for s, page in pages:
        table[s, page] = -1 if (s + page) & 1 else 2 ** 30
    run.held["table"].copy_(torch.from_numpy(table))
    run.lost = set(pages)


def check(run, ctx, window=0, sinks=0, status=0, sequences=None, tokens=None):
    """Tolerance: as mass64's."""
    got = run.call(ctx, window, sinks, status=status, tokens=tokens).double().cpu().numpy()
    q, share, scale, D, r = run.q.double().cpu().numpy(), run.Hq // run.H, run.D ** -0.5, run.D, 0
    for s, (t, positions) in enumerate(zip(run.case.kv, run.case.positions())):
        R = len(positions)
        assert np.all(got[s, t:] == -9.0)
        if sequences is None or s in sequences:
            K, gone = run.keys(s), np.array([(s, j // run.P) in run.lost for j in range(t)])
            j, p = np.arange(t)[None], np.array(positions).reshape(-1, 1)
            see = (j <= p) & ((window == 0) | (p - j < window) | (j < sinks)) & ~gone
            K = np.where((see.any(0))[:, None, None], K, 0.0)
            live, want, tol = see.any(1), np.zeros(t), np.zeros(t)
            for h in range(run.Hq):
                kk, qq = K[:, h // share], q[r:r + R, h]
                x = np.where(see, qq @ kk.T * scale, -np.inf)
                w = np.where(see, np.exp(x - np.where(live, x.max(1), 0.0)[:, None]), 0.0)
                w /= np.where(live, w.sum(1), 1.0)[:, None]
                big = scale * np.where(see, np.abs(qq) @ np.abs(kk).T, 0.0).max(1)[:, None]
                want += w.sum(0)
                tol += (w * (np.expm1(2 * (D + 64) * 2.0 ** -23 * big) + 2.0 ** -19)).sum(0)
            tol += want * (R * run.Hq / 64 + 64) * 2.0 ** -24 + R * run.Hq * 2.0 ** -120
            assert np.all(np.abs(got[s, :t] - want) <= tol), (s, np.flatnonzero(np.abs(got[s, :t] - want) > tol))
            assert np.all(got[s, :t][gone] == 0)
        r += R


@pytest.mark.parametrize("tag", [0, 3])
def test_one_tile_behind_two(pk, ctx, tag):
    """More sequences than SMs, so that a CTA takes those of two tiles of vectors first and then those of one, each with other pages missing."""
    n = 300
    case = Case([1400] * n, [200] * 148 + [60] * (n - 148))
    run = Run(pk, tag, 1, 1, 64, 16, 32, case, BF16)
    lose(run, [(s, page) for s in range(n) for page in ((73, 70, 3) if s < 148 else (0, 20 + s % 40))])
    check(run, ctx, status=pk.E_BOUNDS, sequences={0, 1, 70, 147, 148, 149, 222, 295, 296, 299})


# More than eight tiles of 256 vectors over quantised keys: operands come as images.
MANY = (1, 4, 64, 16, 32), Case([700, 650], [600, 600])


@pytest.mark.parametrize("tag", [0, 1, 3])
def test_many_tiles_of_vectors(pk, ctx, tag):
    geometry, case = MANY
    run = Run(pk, tag, *geometry, case, BF16)
    lose(run, [(0, 2), (0, 40), (1, 0), (1, 17)])
    check(run, ctx, status=pk.E_BOUNDS)
    check(run, ctx, window=30, sinks=5, status=pk.E_BOUNDS)


@pytest.mark.parametrize("tag", [0, 1, 3])
def test_many_tiles_of_vectors_do_not_ask_for_pages_that_none_sees(pk, ctx, tag):
    """Behind the window, between windows that lie apart, and behind the last position."""
    geometry, case = MANY
    run = Run(pk, tag, *geometry, case, BF16)
    lose(run, [(0, 2), (0, 4), (1, 1)])
    check(run, ctx, window=10, sinks=3)
    case = Case([700, 650], [600, 600], [[100 + i % 50 if i < 300 else 400 + i % 70 for i in range(600)], [200 + i % 90 for i in range(600)]])
    run = Run(pk, tag, *geometry, case, BF16)                 # seen: tokens 61 to 149 and 361 to 469, 161 to 289, and the first two
    lose(run, [(0, 2), (0, 14), (0, 21), (0, 40), (1, 3), (1, 20), (1, 39)])
    check(run, ctx, window=40, sinks=2)
    lose(run, [(0, 5), (0, 26), (1, 12)])
    run.lost |= {(0, 2), (0, 14), (0, 21), (0, 40), (1, 3), (1, 20), (1, 39)}
    check(run, ctx, window=40, sinks=2, status=pk.E_BOUNDS)


@pytest.mark.parametrize("tag", [1, 3])
def test_many_tiles_of_vectors_and_scales_that_are_not_numbers_where_none_sees(pk, ctx, tag):
    def spoil(run):
        for s, t, end in ((0, 700, 704), (1, 650, 656), (0, 20, 90)):
            for j in range(t, end):
                ks = run.lay.split(run.pages[run.table[s, j // 16]])[1].view(np.uint16)
                n = len(ks) // 16
                ks[j % 16 * n:(j % 16 + 1) * n] = (0x7E00, 0x7C00, 0xFC00)[j % 3]

    geometry, case = MANY
    run = Run(pk, tag, *geometry, case, BF16, k_edit=spoil)
    run.lost = set()
    check(run, ctx, window=10, sinks=3)


@pytest.mark.parametrize("tag", [1, 3])
@pytest.mark.parametrize("images", [False, True])
def test_many_tiles_in_several_launches_of_quantised_keys(pk, ctx, tag, images):
    """The tiles' sums do not fit the workspace's 256 MiB at once: by the bound on the tokens 100 MiB a tile, so that two go at a time, without images
    (they would take more than their share), and 22.5 MiB a tile with them, eleven at a time of thirteen."""
    n, rows = (90, 50) if images else (400, 460)
    case = Case([500] + [20] * (n - 1), [rows] + [1] * (n - 1))
    run = Run(pk, tag, 1, 64, 64, 16, 32, case, BF16)
    run.held["table"] = run.held["table"].repeat(1, 65536 // (16 * run.table.shape[1]))
    total = rows + n - 1
    run.batch = pk.make_batch(row_start=run.held["start"], kv_len=run.held["kv"], block_table=run.held["table"], n_rows=total, max_rows=rows, max_kv_len=65536)
    assert (pk.attention_mass_workspace_bytes(run.geom, run.cache, run.batch, 64) > 1 << 30) == images
    run.lost = set()
    check(run, ctx, sequences={0, 1, n - 1}, tokens=65536)
    lose(run, [(0, 3), (1, 0)])
    check(run, ctx, status=pk.E_BOUNDS, sequences={0, 1, n - 1}, tokens=65536)


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("D", [64, 80])
def test_batches_without_rows(pk, ctx, tag, D):
    """Their sums are empty; entries of row_start that are out of order are an error in them, too."""
    run = Run(pk, tag, 2, 4, D, 16, 16 if D == 80 else 32, Case([40, 33, 0], [0, 0, 0]), BF16)
    run.q = torch.empty((0, 2, D), dtype=BF16, device=DEV)
    before = torch.rand((3, 43), device=DEV)
    got = run.call(ctx, mass_in=before, decay=0.5)
    for s, t in enumerate(run.case.kv):
        assert torch.equal(got[s, :t], 0.5 * before[s, :t]) and torch.all(got[s, t:] == -9)
    run.held["start"].copy_(torch.tensor([0, 0, 2, 1], dtype=torch.int32))
    got = run.call(ctx, mass_in=before, decay=0.5, status=pk.E_BOUNDS)
    assert torch.equal(got[0, :40], 0.5 * before[0, :40]) and torch.all(got[1:] == -9)
