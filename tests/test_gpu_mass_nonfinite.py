"""patchkv_attention_mass with queries and keys that are not finite, against the formula in 64 bits: where it gives NaN the masses are NaN,
where it gives a number they are that number."""
import numpy as np
import pytest
import torch

from live_common import BF16, F16, Case
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


def formula(run, window=0, sinks=0):
    """Masses of the batch and what fp32 may be off, as mass64 has it, with the terms that are not finite left out of the bound.  A logit of
    minus infinity has the weight 0 beside others, and NaN (0 / 0) where the row has no other."""
    q = run.q[:sum(run.case.rows)].cpu().double().numpy()
    Hq, D, share, scale = q.shape[1], run.D, run.Hq // run.H, run.D ** -0.5
    out, tol, r = [], [], 0
    for b, (t, positions) in enumerate(zip(run.case.kv, run.case.positions())):
        K, R = run.keys(b) if t else np.zeros((0, run.H, D)), len(positions)
        m, e = np.zeros(t), np.zeros(t)
        j, p = np.arange(t)[None], np.array(positions, np.int64).reshape(-1, 1)
        see = (j <= p) & ((window == 0) | (p - j < window) | (j < sinks))
        with np.errstate(invalid="ignore", over="ignore"):
            for h in range(Hq if R and t else 0):
                kk, qq = K[:, h // share], q[r:r + R, h]
                x = np.where(see, (qq[:, None] * kk[None]).sum(-1) * scale, -np.inf)
                w = np.where(see, np.exp(x - x.max(1, keepdims=True)), 0.0)
                w = np.where(see, w / w.sum(1, keepdims=True), 0.0)
                kf, qf = np.where(np.isfinite(kk), kk, 0.0), np.where(np.isfinite(qq), qq, 0.0)
                big = scale * np.where(see, np.abs(qf) @ np.abs(kf).T, 0.0).max(1)[:, None]
                m += w.sum(0)
                e += (w * (np.expm1(2 * (D + 64) * 2.0 ** -23 * big) + 2.0 ** -19)).sum(0)
        out.append(m)
        tol.append(e + m * (R * Hq / 64 + 64) * 2.0 ** -24 + R * Hq * 2.0 ** -120)
        r += R
    return out, tol


def check(run, ctx, window=0, sinks=0, nan_too=False, q=None):
    """nan_too: a NaN will do where the formula has a number."""
    got = run.call(ctx, window, sinks, q=q).double().cpu().numpy()
    want, tol = formula(run, window, sinks)
    for b, t in enumerate(run.case.kv):
        x, nan = got[b, :t], np.isnan(want[b])
        assert np.all(np.isnan(x[nan])), (b, np.flatnonzero(nan & ~np.isnan(x)))
        if not nan_too:
            assert not np.any(np.isnan(x[~nan])), (b, np.flatnonzero(~nan & np.isnan(x)))
        with np.errstate(invalid="ignore"):
            ok = nan | (np.abs(x - want[b]) <= tol[b]) | (nan_too & np.isnan(x))
        assert np.all(ok), (b, np.flatnonzero(~ok))
        assert np.all(got[b, t:] == -9.0)
    return want


# KV heads, query heads, D, page, group: the fast kernels' and the element-wise kernel's
GEOMETRIES = {"fast_64": (1, 4, 64, 16, 32), "fast_128": (2, 8, 128, 16, 32), "any_80": (1, 4, 80, 16, 16)}
# few columns, one tile of vectors, two tiles
ROWS = [1, 3, 30, 50]


def one_sign(run):
    """Every key below zero in every channel, so that an infinite query has logits of minus infinity (or of plus infinity) alone."""
    if run.tag == 0:
        run.kp[:] = -run.kp.abs() - 0.25
    else:
        for page in run.pages:
            run.lay.split(page)[0][:] = 0xFF                # code -1


@pytest.mark.parametrize("tag", [0, 1, 3])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("geometry", list(GEOMETRIES))
@pytest.mark.parametrize("value", ["inf", "-inf", "nan"])
def test_queries(pk, ctx, tag, rows, geometry, value):
    for dtype in (BF16, F16) if tag else (BF16,):
        for edit in (None, one_sign):
            run = Run(pk, tag, *GEOMETRIES[geometry], Case([300, 80], [rows, rows]), dtype, k_edit=edit)
            run.q[rows - 1, 2, 5] = float(value)
            want = check(run, ctx)
            assert np.isnan(want[0]).all() and not np.isnan(want[1]).any()


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("geometry", list(GEOMETRIES))
def test_rows_that_see_one_token(pk, ctx, tag, geometry):
    """All logits of such a row have one sign."""
    for case in (Case([1], [1]), Case([1], [30], [[0] * 30]), Case([60, 2], [60, 1], [list(range(60)), [0]])):
        for sign in (1.0, -1.0):
            run = Run(pk, tag, *GEOMETRIES[geometry], case, BF16)
            run.q[0, :, 3] = sign * float("inf")
            want = check(run, ctx)
            assert np.isnan(want[0][0]) and not np.isnan(want[0][1:]).any()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("geometry", list(GEOMETRIES))
@pytest.mark.parametrize("token", [3, 130, 299])
@pytest.mark.parametrize("value", ["inf", "-inf", "nan"])
def test_keys_of_the_pool(pk, ctx, rows, geometry, token, value):
    """Queries above zero in the channel: plus infinity gives NaN to all that the row sees, minus infinity takes the token's weight away."""
    def spoil(run):
        run.kp[run.table[0, token // run.P], token % run.P, 0, 7] = float(value)

    run = Run(pk, 0, *GEOMETRIES[geometry], Case([300, 80], [rows, rows]), BF16, k_edit=spoil)
    run.q[:, :, 7] = run.q[:, :, 7].abs() + 0.5
    want = check(run, ctx)
    if value == "-inf" and run.H == 1:
        assert want[0][token] == 0 and not np.isnan(want[0]).any()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("geometry", list(GEOMETRIES))
def test_keys_of_the_pool_that_leave_a_row_nothing(pk, ctx, rows, geometry):
    """Minus infinity for every token, and for all but one."""
    for but in (None, 17):
        def spoil(run):
            keep = None if but is None else run.kp[run.table[0, but // run.P], but % run.P].clone()
            run.kp[run.table[0].astype(np.int64), :, :, 7] = float("-inf")
            if but is not None:
                run.kp[run.table[0, but // run.P], but % run.P] = keep

        run = Run(pk, 0, *GEOMETRIES[geometry], Case([300, 80], [rows, rows]), BF16, k_edit=spoil)
        run.q[:, :, 7] = run.q[:, :, 7].abs() + 0.5
        want = check(run, ctx)
        assert np.isnan(want[0]).all() == (but is None) and not np.isnan(want[1]).any()


@pytest.mark.parametrize("tag", [1, 3])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("geometry", list(GEOMETRIES))
@pytest.mark.parametrize("token", [3, 130])
def test_scales_of_keys(pk, ctx, tag, rows, geometry, token):
    """NaN scales, and infinite ones: the masses that the formula has, or NaN (an infinity has no two fp16 parts)."""
    for bits in (0x7E00, 0x7C00):
        def spoil(run):
            ks = run.lay.split(run.pages[run.table[0, token // run.P]])[1].view(np.uint16)
            ks[token % run.P * (len(ks) // run.P)] = bits

        run = Run(pk, tag, *GEOMETRIES[geometry], Case([300, 80], [rows, rows]), BF16, k_edit=spoil)
        want = check(run, ctx, nan_too=bits == 0x7C00)
        assert not np.isnan(want[1]).any()
        check(run, ctx, window=8, sinks=2, nan_too=bits == 0x7C00)


@pytest.mark.parametrize("rows", ROWS)
def test_unaligned_queries_give_the_same(pk, ctx, rows):
    """Calls of a fast geometry whose queries the element-wise kernel takes."""
    def spoil(run):
        run.kp[run.table[0, 0], 3, 0, 7] = float("nan")

    for edit, value in ((one_sign, float("inf")), (spoil, 1.0)):
        run = Run(pk, 0, 1, 4, 64, 16, 32, Case([300, 80], [rows, rows]), BF16, k_edit=edit)
        run.q[rows - 1, 2, 5] = value
        odd = torch.zeros(run.q.numel() + 1, dtype=BF16, device=DEV)[1:].view(run.q.shape)
        odd.copy_(run.q)
        assert np.isnan(check(run, ctx, q=odd)[0]).all()


@pytest.mark.parametrize("rows", [1, 50])
def test_whole_masses_of_broken_rows_are_zero_and_latched(pk, ctx, rows):
    run = Run(pk, 0, 1, 4, 64, 16, 32, Case([300, 80], [rows, rows]), BF16, k_edit=one_sign)
    base = run.call(ctx, dtype=torch.int64)
    run.q[rows - 1, 2, 5] = float("inf")
    got = run.call(ctx, dtype=torch.int64, status=pk.E_BADINPUT)
    assert torch.all(got[0, :300] == 0) and torch.equal(got[1], base[1])


@pytest.mark.parametrize("rows", ROWS)
def test_rows_that_see_nothing_still_add_nothing(pk, ctx, rows):
    """Beside rows that do: at negative positions, and behind the cache's end by more than the window."""
    pos = [[-1] * (rows - 1) + [99], [200] * rows]
    run = Run(pk, 0, 1, 4, 64, 16, 32, Case([100, 80], [rows, rows], pos), BF16)
    run.q[:rows - 1] = float("inf")
    want = check(run, ctx, window=20)
    assert np.all(want[1] == 0) and want[0].sum() == pytest.approx(4.0)
