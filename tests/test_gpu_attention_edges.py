"""patchkv_attention where it is easy to get wrong: what unseen slots hold, rows that see nothing or lie far apart, batches
whose entries are out of order, values of very different size.  Bounds as in test_gpu_attention."""
import numpy as np
import pytest
import torch

from live_common import BF16, F16, Case, attention64, random_rows
from test_gpu_attention import DEV, TAGS, Setup, ctx, pk  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2, 60, 300])
@pytest.mark.parametrize("window", [0, 24])
def test_huge_values_in_unseen_pool_tokens(pk, ctx, rows, window):
    """A finite value of 3e38 in a token that a row does not see, later than the row or behind its window, is not part of its result: a weight
    of zero is zero, not a small number.  Two neighbouring tokens at every place of eight."""
    huge_values(pk, ctx, 400, rows, window)


@pytest.mark.parametrize("window", [0, 24])
def test_huge_values_in_unseen_pool_tokens_with_images(pk, ctx, window):
    """The same from images of the pool's tokens, which enough rows get."""
    huge_values(pk, ctx, 1300, 1200, window)


def huge_values(pk, ctx, total, rows, window):
    s = Setup(pk, 0, 2, 4, 64, 16, 32, Case([total], [rows]))
    first, clean = total - rows, max(1, rows // 2)          # rows [clean, ...) see the later tokens
    at = list(range(first + clean, total)) + list(range(0, first - window) if window else [])
    at = [t for t in at if t % 8 in (0, 1)] or [first + clean]
    s.v = s.v.clone()
    for t in at:
        s.v[s.table[0, t // 16], t % 16] = 3.0e38
        s.host[1][s.table[0, t // 16], t % 16] = 0.0
    s.cache = pk.make_pool(s.k, s.v, s.n_pages, (0, 2048, 128, 64))
    out = s.run(ctx, window)
    assert ctx.query_status() == 0
    seen = Case([total], [clean], [list(range(first, first + clean))])
    s.q = s.q[:clean]
    want, tol = s.reference(window, case=seen)
    assert np.all(np.abs(out[:clean].double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [2, 30, 200])
def test_rows_that_see_nothing_do_not_widen_the_window(pk, ctx, tag, rows):
    """Rows at negative positions (padding) beside windowed ones: pages that only they could have seen may be gone."""
    pos = list(range(900 - rows + 1, 900))
    pos.insert(rows // 2, -1)
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([900], [rows], [pos]))
    first = (pos[0] - 99) // 16                             # page of the first token in the earliest row's window
    s.keep["table"][0, 1:first] = torch.arange(first - 1, dtype=torch.int32, device=DEV) * -7 - 1
    out = s.check(ctx, 100, 5)
    assert (out[rows // 2] == 0).all()


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("near", [1, 20, 80, 200])
@pytest.mark.parametrize("splits", [False, True])
def test_pages_between_rows_may_be_gone(pk, ctx, tag, near, splits):
    """Rows further apart than the window: pages between their windows may be gone; one that a row sees may not."""
    total = 4000 if splits else 1400
    pos = list(range(100, 100 + near)) + list(range(total - near, total))
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([total], [2 * near], [pos]))
    a, b = (100 + near - 1) // 16 + 1, (total - near - 63) // 16
    s.keep["table"][0, a:b] = s.n_pages + 5
    s.check(ctx, 64, 3)
    s.keep["table"][0, b] = -1
    s.run(ctx, 64, 3)
    assert ctx.query_status() == pk.E_BOUNDS


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 3, 40, 300])
@pytest.mark.parametrize("window", [1, 4, 20])
def test_rows_behind_the_cache(pk, ctx, tag, rows, window):
    """Positions at and behind kv_len: a window that ends behind the last token shows nothing, and asks for no page."""
    pos = [405 + window - 1 + i for i in range(rows)]       # kv_len 405 ends inside a tile and a page; the windows start at 405 and later
    s = Setup(pk, tag, 2, 4, 64, 32, 32, Case([405], [rows], [pos]))
    s.keep["table"][0] = -1
    out = s.check(ctx, window)
    assert (out[:rows] == 0).all()


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_a_sequence_before_descending_entries_keeps_its_rows(pk, ctx, tag, rows):
    """row_start that descends leaves out the sequence whose entries those are and no other, also where the tokens are split."""
    s = Setup(pk, tag, 1, 2, 64, 16, 32, Case([3000, 50], [rows, rows]))
    s.keep["start"][2] = 0
    out = s.run(ctx)
    assert ctx.query_status() == pk.E_BOUNDS
    assert (out[rows:] == 5).all()
    s.q = s.q[:rows]
    want, tol = s.reference(case=Case([3000], [rows]))
    assert np.all(np.abs(out[:rows].double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 40, 130, 300])
def test_a_loose_bound_on_the_lengths(pk, ctx, tag, rows):
    """max_kv_len of 2^31 - 1: the same results.  Images of that many steps would pass what they may take, so 300 rows run as several CTAs
    that convert the codes themselves."""
    case = Case([700, 350], [rows, max(1, rows // 3)])
    Setup(pk, tag, 2, 8, 64, 16, 32, case, max_kv=2 ** 31 - 1).check(ctx, 300, 4)
    Setup(pk, tag, 1, 4, 128, 16, 32, case, dtype=F16 if tag else BF16, max_kv=2 ** 31 - 1).check(ctx)


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("rows", [1, 40])
def test_long_caches(pk, ctx, tag, rows):
    """Tens of thousands of tokens: many tiles a piece, and look-ups past the first 32 of a warp."""
    s = Setup(pk, tag, 1, 2, 64, 16, 32, Case([40001], [rows]))
    s.check(ctx)
    s.check(ctx, 20000, 5000)


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("rows", [1, 8])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("scale", [0.125, 1.0, 5.0])
def test_few_columns_see_whole_keys(pk, ctx, tag, rows, dtype, scale):
    """Up to 16 columns the logits are those of code * scale, of any size: the bound has no term for a rounding of K."""
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([300], [rows]), dtype=dtype)
    got = s.check(ctx, scale=scale)[:rows].double().cpu().numpy()
    want, tol = attention64(s.q[:rows].double().numpy(), lambda b: s.kv(b)[0], lambda b: s.kv(b)[1], s.case, 2, scale, 0, 0, dtype,
                            False, k_rounding=0.0)
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 4])
@pytest.mark.parametrize("at", [0, 37])
@pytest.mark.parametrize("size", [300.0, 2.0e4])
def test_a_token_of_large_values_and_no_weight(pk, ctx, tag, dtype, rows, at, size):
    """One token's values are far larger than all others and its weight is zero (its logit 150 and more below the others, in
    powers of two): the others keep their bits.  The bound is that of the batch without the token."""
    n, D = 200, 64
    s = Setup(pk, tag, 1, 2, D, 16, 32, Case([n], [rows], [[n - 1] * rows]), dtype=dtype)
    s.q = (s.q.abs() + 0.5).to(dtype)
    rng = np.random.default_rng(8)
    for j in range(n):
        k, v = (random_rows(rng, 1, 1, D, BF16, outliers=False).double().numpy()[0] for _ in range(2))
        if j == at:
            k, v = np.full((1, D), -40.0), np.full((1, D), size)
        s.lay.put(s.pages[s.table[0, j // 16]], j % 16, k, v)
    s.dev.copy_(torch.from_numpy(s.pages))
    got = s.run(ctx)[:rows].double().cpu().numpy()
    assert ctx.query_status() == 0
    rest = [j for j in range(n) if j != at]
    K, V = (x[rest] for x in s.kv(0))
    x = s.q[:rows].double().numpy() @ s.kv(0)[0][at, 0] * D ** -0.5
    assert (x < -104 - 40).all()                            # e^-104 is below 2^-150; logits of the others are above -40
    want, tol = attention64(s.q[:rows].double().numpy(), lambda b: K, lambda b: V, Case([n - 1], [rows], [[n - 2] * rows]), 2,
                            D ** -0.5, 0, 0, dtype, False, k_rounding=0.0)
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)


@pytest.mark.parametrize("tag", [2, 3])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D,G", [(64, 32), (128, 64)])
@pytest.mark.parametrize("size", [2.0 ** -10, 2.0 ** -15])
def test_groups_of_small_values_keep_their_bits(pk, ctx, tag, dtype, D, G, size):
    """The values of one scale group are far smaller than the other's, in every token: bounded group by group."""
    n = 100
    s = Setup(pk, tag, 1, 2, D, 16, G, Case([n], [2]), dtype=dtype)
    rng = np.random.default_rng(8)
    for j in range(n):
        k, v = (random_rows(rng, 1, 1, D, BF16, outliers=False).double().numpy()[0] for _ in range(2))
        v *= 16
        v[:, G:] *= size
        s.lay.put(s.pages[s.table[0, j // 16]], j % 16, k, v)
    s.dev.copy_(torch.from_numpy(s.pages))
    got = s.run(ctx).double().cpu().numpy()
    assert ctx.query_status() == 0
    K, V = s.kv(0)
    for c in (slice(0, G), slice(G, D)):
        only = np.zeros_like(V)
        only[..., c] = V[..., c]
        want, tol = attention64(s.q.double().numpy(), lambda b: K, lambda b: only, s.case, 2, D ** -0.5, 0, 0, dtype, False, k_rounding=0.0)
        err = np.abs(got - want)[..., c]
        assert np.all(err <= tol[..., c]), np.max(err / tol[..., c])


@pytest.mark.parametrize("rows", [500, 1100])
@pytest.mark.parametrize("name", ["causal", "window", "scattered", "gone"])
def test_pool_rows_without_and_with_images(pk, ctx, rows, name):
    """4 and 9 CTAs of vectors over the bf16 pool: fewer than eight read the pages themselves, more get images of them."""
    total = 1500
    pos = [[(i * 37) % total for i in range(rows)]] if name == "scattered" else None
    s = Setup(pk, 0, 1, 2, 64, 16, 32, Case([total], [rows], pos))
    if name == "gone":
        s.keep["table"][0, 1:(total - rows - 100) // 16] = -1
    s.check(ctx, *{"window": (70, 0), "gone": (100, 3)}.get(name, (0, 0)))


@pytest.mark.parametrize("rows", [1, 4, 8])
@pytest.mark.parametrize("scale", [0.125, 0.25])
def test_few_columns_over_the_pool_keep_their_weights(pk, ctx, rows, scale):
    """Up to 16 columns the weights over bf16 pages are sums of two bf16 numbers.  What is left is half a step of the result and,
    of sum p|v|: 2^-16 for the weights (two roundings of 2^-9, the second of what the first left, doubled), 2^-18 for exp2 and the
    sums, and what fp32 dot products of D = 64 put the logits off."""
    s = Setup(pk, 0, 2, 4, 64, 16, 32, Case([300], [rows]))
    got = s.check(ctx, scale=scale)[:rows].double().cpu().numpy()
    q, K, V = s.q[:rows].double().numpy(), s.kv(0)[0], s.kv(0)[1]
    want, _ = attention64(q, lambda b: K, lambda b: V, s.case, 2, scale, 0, 0, BF16, True)
    mass, _ = attention64(q, lambda b: K, lambda b: np.abs(V), s.case, 2, scale, 0, 0, BF16, True)
    big = scale * np.einsum("rhd,khd->rhk", np.abs(q), np.abs(K).repeat(2, 1)).max(2)[..., None]
    half_step = 2.0 ** (np.floor(np.log2(np.abs(want))) - 8)
    tol = half_step + (2.0 ** -16 + 2.0 ** -18 + np.expm1(2 * (64 + 64) * 2.0 ** -23 * big)) * mass
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)
