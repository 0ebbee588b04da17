"""The element-wise kernels at the largest length there is, 2^31 - 1 tokens: a block table that names one page of 2^28 tokens eight times, and
a window, so that few tokens count."""
import numpy as np
import pytest
import torch

from live_common import BF16

pytestmark = pytest.mark.gpu
DEV, D, P, KV, WINDOW = "cuda:0", 2, 1 << 28, 2 ** 31 - 1, 100


@pytest.fixture(scope="module")
def pk():
    from paper_2609_26219_b200 import build, binding
    build.build()
    return binding


def test_attention_and_its_weight(pk):
    ctx = pk.Context(device=0)
    rng = np.random.default_rng(4)
    k = torch.zeros(P * D, dtype=BF16, device=DEV)
    rows = torch.from_numpy(rng.standard_normal((WINDOW, D))).to(BF16)
    k.view(P, D)[P - 1 - WINDOW:P - 1] = rows.to(DEV)         # the last position is slot P - 2 of its page
    q = torch.from_numpy(rng.standard_normal((1, 1, D))).to(BF16).to(DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    held = [i32(0, 1), i32(KV), torch.zeros((1, 8), dtype=torch.int32, device=DEV)]
    batch = pk.make_batch(row_start=held[0], kv_len=held[1], block_table=held[2], n_rows=1, max_rows=1, max_kv_len=KV)
    geom, pool = pk.make_geom(1, 1, D, D, pk.ROPE_HALF, 1e4, 16, P, D), pk.make_pool(k, k, 1, (0, P * D, D, D))
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    out, mass = torch.empty_like(q), torch.full((1, KV), -9.0, device=DEV)
    ctx.attention(geom, pool, 0, batch, q, out, window=WINDOW, workspace=ws)
    ctx.attention_mass(geom, pool, 0, batch, q, mass, window=WINDOW, workspace=ws)
    assert ctx.query_status() == 0
    x, kk = q.double().cpu().numpy()[0, 0], rows.double().numpy()
    w = np.exp(kk @ x * D ** -0.5)
    w /= w.sum()
    d = (D + 64) * 2.0 ** -23 * (np.abs(kk) @ np.abs(x)).max()                    # of a logit; 2^x and its argument 2^-19; 64 sums
    weight_tol = w * (np.expm1(2 * d) + 2.0 ** -19 + 64 * 2.0 ** -24)
    assert np.all(np.abs(mass[0, KV - WINDOW:].double().cpu().numpy() - w) <= weight_tol)
    assert int(torch.count_nonzero(mass)) == WINDOW
    want = w @ kk
    assert np.all(np.abs(out.double().cpu().numpy()[0, 0] - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * (weight_tol @ np.abs(kk) + 64 * 2.0 ** -24 * (w @ np.abs(kk))))
    ctx.close()
