"""patchkv_attention_mass against a plain 64-bit reference: masks, lengths, types, masses of both kinds, refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from live_common import BF16, F16, Case, Layout, build_tables, device_batch, random_rows

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


def mass64(q, k_of, case, share, scale, window, sinks, n_tokens):
    """q float64 [n][Hq][D], k_of(b) float64 [kv][H][D].  Returns (masses [seqs][n_tokens], tol): tol bounds what fp32 may be off.
      a logit: its D products summed in fp32 (keys of quantised pages to 22 bits), (D + 64) 2^-23 of sum |q||k| scale: d; a weight e^(x - sum)
      is then off by a factor within e^(2d); 2^x itself and the difference in its exponent by 2^-19;
      n weights summed one by one: n 2^-24 of the sum, at most 2^-23 (sqrt is what happens) for each of the levels of a sum: (n / 64 + 64) 2^-24."""
    Hq, D = q.shape[1:]
    out, tol = np.zeros((len(case.kv), n_tokens)), np.zeros((len(case.kv), n_tokens))
    r = 0
    for b, (t, positions) in enumerate(zip(case.kv, case.positions())):
        R = len(positions)
        if R and t:
            K = k_of(b)
            j, p = np.arange(t)[None], np.array(positions)[:, None]
            see = (j <= p) & ((window == 0) | (p - j < window) | (j < sinks))
            some = see.any(0)
            K = np.where(some[:, None, None], K, 0.0)       # what no row sees may hold anything
            live = see.any(1)
            for h in range(Hq):
                kk, qq = K[:, h // share], q[r:r + R, h]
                with np.errstate(invalid="ignore", over="ignore"):
                    x = np.where(see, qq @ kk.T * scale, -np.inf)
                    w = np.where(see, np.exp(x - np.where(live, x.max(1), 0.0)[:, None]), 0.0)
                    w /= np.where(live, w.sum(1), 1.0)[:, None]
                    big = np.abs(scale) * np.where(see, np.abs(qq) @ np.abs(kk).T, 0.0).max(1)[:, None]
                d = (D + 64) * 2.0 ** -23 * big
                out[b, :t] += w.sum(0)
                tol[b, :t] += (w * (np.expm1(2 * d) + 2.0 ** -19)).sum(0)
            tol[b, :t] += out[b, :t] * (R * Hq / 64 + 64) * 2.0 ** -24 + R * Hq * 2.0 ** -120
        r += R
    return out, tol


class Run:
    """A cache with random rows, and a batch over it."""

    def __init__(self, pk, tag, H, Hq, D, P, G, case, dtype, seed=7, layers=1, outliers=True, n_rows=None, k_edit=None):
        rng = np.random.default_rng(seed)
        self.pk, self.tag, self.case, self.H, self.Hq, self.D, self.P = pk, tag, case, H, Hq, D, P
        self.table, n_pages = build_tables(case, P, rng)
        self.batch, self.held = device_batch(pk, case, self.table, DEV, n_rows=n_rows)
        self.geom = pk.make_geom(layers, H, D, D, pk.ROPE_HALF, 1e4, 16, P, G)
        n = self.batch.n_rows
        self.q = random_rows(rng, n, Hq, D, dtype, False).to(DEV)
        if tag == 0:
            self.kp = random_rows(rng, n_pages * P, H, D, BF16, outliers).view(n_pages, P, H, D)
            if k_edit:
                k_edit(self)
            self.dev = self.kp.to(DEV)
            self.cache = pk.make_pool(self.dev, self.dev, n_pages, (0, P * H * D, H * D, D))
        else:
            self.lay = Layout(tag, H, D, P, G)
            self.pages = rng.integers(0, 256, (n_pages, self.lay.page_bytes()), dtype=np.uint8)
            for p in self.pages:                            # scales as normal rows give them
                for _, s in (self.lay.split(p)[:2][::1],):
                    s[:] = np.frombuffer((0.3 * np.exp(0.4 * rng.standard_normal(len(s) // 2))).astype(np.float16).tobytes(), np.uint8)
            if k_edit:
                k_edit(self)
            self.dev = torch.from_numpy(self.pages).to(DEV)
            self.cache = pk.make_qpool(self.dev, tag, n_pages)

    def keys(self, b):
        t = self.case.kv[b]
        ids = self.table[b, :-(-t // self.P)]
        if self.tag == 0:
            return self.kp[ids].flatten(0, 1)[:t].double().numpy()
        out = []
        for i in ids:
            kc, ks = self.lay.split(self.pages[i])[:2]
            from live_common import BITS, unpack
            s = np.frombuffer(ks.tobytes(), np.float16).astype(np.float64)
            with np.errstate(invalid="ignore"):
                out.append((unpack(kc, BITS[self.tag][0]).reshape(-1, self.lay.G) * s[:, None]).reshape(self.P, self.H, self.D))
        return np.concatenate(out)[:t]

    def call(self, ctx, window=0, sinks=0, scale=None, mass_in=None, decay=1.0, dtype=torch.float32, status=0, q=None, workspace=None, tokens=None, out=None):
        tokens = (max(self.case.kv + [0]) + 3) if tokens is None else tokens
        mass = torch.full((len(self.case.kv), tokens), -9, dtype=dtype, device=DEV) if out is None else out
        need = self.pk.attention_mass_workspace_bytes(self.geom, self.cache, self.batch, self.Hq, window, sinks)
        ws = torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device=DEV) if workspace is None else workspace
        ctx.attention_mass(self.geom, self.cache, 0, self.batch, self.q if q is None else q, mass, mass_in=mass_in, decay=decay, scale=scale, window=window,
                           sinks=sinks, workspace=ws)
        assert ctx.query_status() == status
        return mass

    def want(self, window=0, sinks=0, scale=None, tokens=None):
        tokens = (max(self.case.kv + [0]) + 3) if tokens is None else tokens
        n = sum(self.case.rows)
        return mass64(self.q[:n].cpu().double().numpy(), self.keys, self.case, self.Hq // self.H, self.D ** -0.5 if scale is None else scale, window, sinks, tokens)

    def check(self, ctx, window=0, sinks=0, scale=None, status=0):
        got = self.call(ctx, window, sinks, scale, status=status).double().cpu().numpy()
        want, tol = self.want(window, sinks, scale)
        for b, t in enumerate(self.case.kv):
            assert np.all(np.abs(got[b, :t] - want[b, :t]) <= tol[b, :t]), (b, np.max(np.abs(got[b, :t] - want[b, :t]) / np.maximum(tol[b, :t], 1e-300)))
            assert np.all(got[b, t:] == -9.0)
        return got, want


BATCHES = {
    "one_token": Case([1], [1]),
    "decode": Case([1000], [1]),
    "decode_ragged": Case([40, 333, 1, 129, 700], [1, 1, 1, 1, 1]),
    "few_rows": Case([90, 300], [3, 2]),
    "rows_and_none": Case([130, 0, 17, 64, 50], [130, 0, 5, 1, 0]),
    "prompt": Case([333, 100], [333, 61]),
    "scattered": Case([700, 33], [9, 3], [[0, 15, 16, 300, 301, 302, 555, 698, 699], [1, 2, 32]]),
}
GEOMETRIES = [(8, 32, 128, 16, 32), (4, 8, 64, 16, 32), (4, 28, 128, 32, 64), (1, 8, 64, 64, 64), (2, 2, 128, 16, 128), (3, 3, 64, 16, 32), (5, 20, 128, 16, 32),
              (2, 6, 80, 16, 16), (1, 1, 6, 5, 3), (2, 4, 256, 8, 64)]


@pytest.mark.parametrize("tag", [0, 1, 2, 3])
@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("geometry", GEOMETRIES, ids=str)
def test_masses(pk, ctx, tag, name, geometry):
    H, Hq, D, P, G = geometry
    for dtype in (BF16, F16):
        if tag or dtype is BF16:
            Run(pk, tag, H, Hq, D, P, G, BATCHES[name], dtype).check(ctx)


@pytest.mark.parametrize("tag", [0, 1, 3])
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 2), (100, 4), (128, 17), (5000, 1)])
@pytest.mark.parametrize("name", ["decode_ragged", "few_rows", "prompt", "scattered", "rows_and_none"])
def test_windows(pk, ctx, tag, window, sinks, name):
    for geometry in ((8, 32, 128, 16, 32), (2, 14, 64, 32, 32), (2, 6, 80, 16, 16)):
        H, Hq, D, P, G = geometry
        Run(pk, tag, H, Hq, D, P, G, BATCHES[name], BF16).check(ctx, window, sinks)


@pytest.mark.parametrize("tag", [0, 2, 3])
def test_longer_ones(pk, ctx, tag):
    """Lengths over which the work is split; 2-norm errors as fp32 gives them: each logit is some 2^-22 of itself off."""
    for case, geo in ((Case([5000, 3111], [1, 1]), (8, 64, 128, 16, 32)), (Case([4097], [40]), (2, 8, 128, 16, 32)), (Case([2100, 1300], [1500, 700]), (2, 8, 64, 16, 32)),
                      (Case([20000], [5]), (1, 3, 128, 64, 128))):
        got, want = Run(pk, tag, *geo, case, BF16).check(ctx)
        for b, t in enumerate(case.kv):
            assert np.linalg.norm(got[b, :t] - want[b, :t]) <= 1e-5 * np.linalg.norm(want[b, :t])


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("name", ["decode_ragged", "prompt"])
def test_scales_and_large_logits(pk, ctx, tag, name):
    """Weights of one token alone, equal weights, turned signs."""
    for scale in (0.0, -0.3, 8.0, 1e-6):
        Run(pk, tag, 2, 8, 64, 16, 32, BATCHES[name], BF16).check(ctx, scale=scale)


@pytest.mark.parametrize("tag", [0, 1])
@pytest.mark.parametrize("name", ["decode_ragged", "prompt"])
def test_decay_and_the_masses_before(pk, ctx, tag, name):
    run = Run(pk, tag, 2, 8, 64, 16, 32, BATCHES[name], BF16)
    base = run.call(ctx)
    before = torch.rand_like(base)
    for decay in (1.0, 0.5, -2.0):
        got = run.call(ctx, mass_in=before, decay=decay)
        same = before.clone()
        run.call(ctx, mass_in=same, decay=decay, out=same)                 # in place
        for b, t in enumerate(run.case.kv):
            want = base[b, :t].double() + decay * before[b, :t].double()
            assert torch.all((got[b, :t].double() - want).abs() <= 2.0 ** -23 * (want.abs() + abs(decay)))
            assert torch.equal(same[b, :t], got[b, :t]) and torch.equal(same[b, t:], before[b, t:])
    before[:] = float("nan")
    assert torch.equal(run.call(ctx, mass_in=before, decay=0.0), base)     # not read


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("name", ["decode_ragged", "prompt", "rows_and_none"])
def test_whole_masses(pk, ctx, tag, name):
    """Units of 2^-24, the fp32 sum rounded once; what select_repair_tokens ranks by."""
    run = Run(pk, tag, 2, 8, 64, 16, 32, BATCHES[name], BF16)
    base = run.call(ctx)
    units = run.call(ctx, dtype=torch.int64)
    before = torch.full_like(units, 2 ** 40 + 3)
    more = run.call(ctx, dtype=torch.int64, mass_in=before)
    for b, t in enumerate(run.case.kv):
        assert torch.equal(units[b, :t], (base[b, :t].double() * 2 ** 24).round().long())
        assert torch.equal(more[b, :t], units[b, :t] + 2 ** 40 + 3) and torch.all(units[b, t:] == -9)
    with pytest.raises(pk.PatchKVError):
        run.call(ctx, dtype=torch.int64, mass_in=before, decay=0.5)


def test_whole_masses_pick_repair_blocks(pk, ctx):
    run = Run(pk, 0, 2, 8, 64, 16, 32, Case([512], [4]), BF16)
    units = run.call(ctx, dtype=torch.int64, tokens=512)
    nb = 32
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device=DEV)
    out = dict(repair_mask=z(1, nb, t=torch.uint8), repair_idx=z(1, nb), repair_cnt=z(1), reuse_idx=z(1, nb), reuse_cnt=z(1))
    ctx.select_repair_tokens(pk.select_args(kind=pk.SCORE_TOKEN_MASS, n_layers=1, n_suffix_tokens=512, block_tokens=16, dirty_tokens=16, top_k=20,
                                            layer_mode=pk.LAYERS_INDEPENDENT, mass=units, **out))
    assert ctx.query_status() == 0
    m = units[0].cpu().numpy()
    top = sorted(range(16, 512), key=lambda i: (-m[i], i))[:20]
    want = sorted({0} | {i // 16 for i in top})
    assert out["repair_idx"][0, :len(want)].tolist() == want and int(out["repair_cnt"][0]) == len(want)


@pytest.mark.parametrize("tag", [0, 1, 2, 3])
@pytest.mark.parametrize("name", ["decode_ragged", "few_rows", "prompt"])
def test_equal_calls_give_equal_bits(pk, ctx, tag, name):
    run = Run(pk, tag, 4, 16, 128, 16, 32, BATCHES[name], BF16)
    first = run.call(ctx)
    for _ in range(3):
        assert torch.equal(run.call(ctx), first)


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("rows", [1, 40])
def test_what_no_row_sees_may_hold_anything(pk, ctx, tag, rows):
    """NaN and infinities in slots behind the cache's end and behind the window."""
    case = Case([150], [rows])

    def spoil(run):
        for t in list(range(150, 160)) + list(range(20, 150 - rows - 9)):
            page, slot = run.table[0, t // 16], t % 16
            if tag == 0:
                run.kp[page, slot] = float("nan") if t & 1 else float("inf")
            else:
                ks = run.lay.split(run.pages[page])[1]
                n = len(ks) // 16
                ks[slot * n:(slot + 1) * n] = 0xFF if t & 1 else np.frombuffer(np.array([0x7C00] * (n // 2), np.uint16).tobytes(), np.uint8)

    Run(pk, tag, 2, 8, 64, 16, 32, case, BF16, k_edit=spoil).check(ctx, window=10, sinks=3)


@pytest.mark.parametrize("tag", [0, 1, 3])
@pytest.mark.parametrize("rows", [2, 40])
def test_broken_queries_and_keys(pk, ctx, tag, rows):
    """A query with a NaN gives NaN to what it sees and to nothing else; a key that is not finite does so for the rows that see it."""
    run = Run(pk, tag, 1, 4, 64, 16, 32, Case([100, 80], [rows, rows]), BF16)
    base = run.call(ctx)
    run.q[rows - 1, 2, 5] = float("nan")
    got = run.call(ctx)
    assert torch.isnan(got[0, :100]).all() and torch.equal(got[1], base[1])
    run.q[rows - 1, 2, 5] = float("inf")
    got = run.call(ctx)
    assert torch.isnan(got[0, :100]).all() and torch.equal(got[1], base[1])
    run.q[:] = 0.0                                              # equal weights, whatever the sign of the zeros
    got = run.call(ctx)
    want, tol = run.want()
    assert np.all(np.abs(got[0, :100].double().cpu().numpy() - want[0, :100]) <= tol[0, :100])


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("rows", [1, 50])
def test_pages_and_lengths_out_of_range(pk, ctx, tag, rows):
    case = Case([100, 90], [rows, rows])
    run = Run(pk, tag, 2, 8, 64, 16, 32, case, BF16)
    base = run.call(ctx)
    gone = int(run.table[0, 2])
    run.held["table"][0, 2] = -1
    got = run.call(ctx, status=pk.E_BOUNDS)
    assert torch.equal(got[1], base[1])
    assert torch.all(got[0, 32:48] == 0) and torch.allclose(got[0, :100].sum(), torch.tensor(8.0 * rows, device=DEV), rtol=1e-5)
    # behind the window nobody asks for it
    got = run.call(ctx, window=8 if rows == 1 else 2, status=0)
    if rows == 1:
        assert torch.all(got[0, :92] == 0)
    run.held["table"][0, 2] = gone
    run.held["kv"][0] = 200                                     # more than max_kv_len: the first 100 count; rows stand behind them
    got = run.call(ctx, status=pk.E_BOUNDS)
    assert torch.equal(got[1], base[1]) and torch.all(got[0, 100:] == -9)
    run.held["kv"][0] = 0
    got = run.call(ctx, status=0)
    assert torch.equal(got[1], base[1]) and torch.all(got[0] == -9)
    run.held["kv"][0] = 100
    run.held["start"][1] = 2 * rows + 5
    got = run.call(ctx, status=pk.E_BOUNDS)
    assert torch.all(got == -9)                                 # both sequences' entries are out of order or range


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("rows", [1, 40])
def test_loose_bounds(pk, ctx, tag, rows):
    """Bounds far above what there is: tokens up to 2^31 - 1, and packed rows that no sequence has, with aligned and unaligned queries."""
    run = Run(pk, tag, 2, 8, 64, 16, 32, Case([150, 130], [rows, rows]), BF16, n_rows=2 * rows + 5000)
    base = run.call(ctx, tokens=160)
    run.batch.max_kv_len = 2 ** 31 - 1
    assert torch.equal(run.call(ctx, tokens=160), base)
    odd = torch.zeros(run.q.numel() + 1, dtype=BF16, device=DEV)[1:].view(run.q.shape)
    odd.copy_(run.q)
    got, (want, tol) = run.call(ctx, q=odd, tokens=160).double().cpu().numpy(), run.want(tokens=160)
    for b, t in enumerate(run.case.kv):
        assert np.all(np.abs(got[b, :t] - want[b, :t]) <= tol[b, :t]) and np.all(got[b, t:] == -9.0)


def test_many_tiles_in_several_launches(pk, ctx):
    """So many tiles of vectors, sequences and (by the bound) tokens that what the tiles give to the tokens does not fit the workspace's 256 MiB at
    once: 100 MiB a tile, so two at a time."""
    case = Case([500] + [20] * 399, [460] + [1] * 399)
    run = Run(pk, 0, 1, 64, 64, 16, 32, case, BF16)
    want, tol = run.want(tokens=500)
    run.held["wide"] = run.held["table"].repeat(1, 65536 // (16 * run.table.shape[1]))
    run.batch = pk.make_batch(row_start=run.held["start"], kv_len=run.held["kv"], block_table=run.held["wide"], n_rows=859, max_rows=460, max_kv_len=65536)
    before = torch.rand((400, 65536), device=DEV)
    got = run.call(ctx, tokens=65536, mass_in=before, decay=0.5)
    for b, t in ((0, 500), (1, 20), (399, 20)):
        x = got[b, :t].double().cpu().numpy() - 0.5 * before[b, :t].double().cpu().numpy()
        assert np.all(np.abs(x - want[b, :t]) <= tol[b, :t] + 2.0 ** -23 * (np.abs(want[b, :t]) + 1)) and torch.all(got[b, t:] == -9)


@pytest.mark.parametrize("tag", [0, 3])
def test_a_million_tokens(pk, ctx, tag):
    """A block table that names the same eight pages over and over, seen by 38400 vectors: more CTAs along the vectors than SMs, and yet the tokens
    are split.  Every token of a page then has the same mass each time.  Tolerance: as mass64's, and a row's sum is added up by 64 columns
    and then step by step (12000 of them), so it is off by at most (64 + 12000) 2^-24."""
    pages, times, D, share = 8, 2500, 64, 32
    rows, period = 1200, 8 * 64
    kv = period * times
    run = Run(pk, tag, 1, share, D, 64, 32, Case([period], [1]), BF16)
    q = random_rows(np.random.default_rng(5), rows, share, D, BF16, False).to(DEV)
    ids = torch.from_numpy(run.table[:1, :pages].astype(np.int32)).to(DEV)
    held = [torch.tensor([0, rows], dtype=torch.int32, device=DEV), torch.tensor([kv], dtype=torch.int32, device=DEV),
            torch.full((rows,), kv - 1, dtype=torch.int32, device=DEV), ids.repeat(1, times).contiguous()]
    run.batch = pk.make_batch(row_start=held[0], kv_len=held[1], block_table=held[3], pos=held[2], n_rows=rows, max_rows=rows, max_kv_len=kv)
    run.case = Case([kv], [rows])
    got = run.call(ctx, q=q, tokens=kv)[0].double().view(times, period)
    run.case = Case([period], [1])
    K, qq = torch.from_numpy(run.keys(0)[:, 0]).to(DEV), q.double().flatten(0, 1)
    x = qq @ K.T * D ** -0.5
    w = torch.softmax(x, 1) / times
    d = (D + 64) * 2.0 ** -23 * (qq.abs() @ K.abs().T).amax(1, keepdim=True) * D ** -0.5
    want = w.sum(0)
    tol = (w * (torch.expm1(2 * d) + 2.0 ** -19)).sum(0) + want * ((rows * share / 64 + 64) + 64 + kv / 128) * 2.0 ** -24
    assert torch.all((got - want).abs() <= tol)


def test_rows_above_the_bound_are_left_out(pk, ctx):
    for rows in (3, 60):
        run = Run(pk, 0, 2, 4, 64, 16, 32, Case([100, 90], [rows, 2]), BF16)
        base = run.call(ctx)
        run.batch.max_rows = rows - 1
        got = run.call(ctx, status=pk.E_BOUNDS)
        assert torch.equal(got[1], base[1])
        assert torch.allclose(got[0, :100].sum(), torch.tensor(4.0 * (rows - 1), device=DEV), rtol=1e-5)


def test_strided_queries_and_other_layers(pk, ctx):
    for rows in (1, 70):
        run = Run(pk, 0, 2, 8, 64, 16, 32, Case([200], [rows]), BF16)
        base = run.call(ctx)
        wide = torch.zeros((rows, 12, 64), dtype=BF16, device=DEV)
        wide[:, 2:10] = run.q
        assert torch.equal(run.call(ctx, q=wide[:, 2:10]), base)
        flip = run.q.transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(run.call(ctx, q=flip), base)
        odd = torch.zeros(rows * 512 + 1, dtype=BF16, device=DEV)[1:].view(rows, 8, 64)
        odd.copy_(run.q)
        got, (want, tol) = run.call(ctx, q=odd)[0, :200].double().cpu().numpy(), run.want()
        assert np.all(np.abs(got - want[0, :200]) <= tol[0, :200])


def test_replay_with_other_contents(pk, ctx):
    for tag, rows in ((0, 1), (3, 1), (1, 50)):
        run = Run(pk, tag, 2, 8, 64, 16, 32, Case([300, 200], [rows, rows]), BF16)
        need = pk.attention_mass_workspace_bytes(run.geom, run.cache, run.batch, 8)
        ws, mass = torch.zeros(max(need, 16), dtype=torch.uint8, device=DEV), torch.zeros((2, 300), device=DEV)
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            ctx.attention_mass(run.geom, run.cache, 0, run.batch, run.q, mass, workspace=ws, stream=torch.cuda.current_stream())
        run.q.mul_(-1.0)
        run.held["kv"].copy_(torch.tensor([277, 123], dtype=torch.int32))
        run.case = Case([277, 123], [rows, rows])
        graph.replay()
        torch.cuda.synchronize()
        want, tol = run.want(tokens=300)
        got = mass.double().cpu().numpy()
        for b, t in enumerate(run.case.kv):
            assert np.all(np.abs(got[b, :t] - want[b, :t]) <= tol[b, :t]) and np.all(got[b, t:] == 0)
        assert ctx.query_status() == 0


def test_refusals(pk, ctx):
    run = Run(pk, 0, 2, 8, 64, 16, 32, Case([100], [3]), BF16)
    mass = torch.zeros((1, 100), device=DEV)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)

    def refused(code, **m):
        with pytest.raises(pk.PatchKVError) as e:
            ctx.attention_mass(run.geom, run.cache, m.pop("layer", 0), run.batch, m.pop("q", run.q), m.pop("mass", mass), workspace=m.pop("ws", ws), **m)
        assert e.value.code == code

    refused(pk.E_INVALID, layer=1)
    refused(pk.E_INVALID, q=run.q.half())
    refused(pk.E_INVALID, q=run.q[:, :7])
    refused(pk.E_INVALID, window=-1)
    refused(pk.E_INVALID, sinks=-1)
    refused(pk.E_INVALID, scale=float("nan"))
    refused(pk.E_INVALID, decay=float("inf"))
    refused(pk.E_INVALID, ws=None)
    refused(pk.E_INVALID, ws=ws[:8])
    refused(pk.E_INVALID, ws=ws[4:])
    for bad in (dict(mass=mass[:, :50]), dict(mass=mass.double()), dict(mass=mass.t()), dict(mass_in=mass.long()), dict(q=run.q[:2])):
        with pytest.raises(ValueError):
            ctx.attention_mass(run.geom, run.cache, 0, run.batch, bad.pop("q", run.q), bad.pop("mass", mass), workspace=ws, **bad)
    a = pk.MassArgs(C.sizeof(pk.MassArgs), 0, 8)
    assert pk.lib().patchkv_attention_mass(ctx._h, run.geom, None, None, 0, run.batch, a, None) == pk.E_INVALID
    assert pk.lib().patchkv_attention_mass(ctx._h, run.geom, run.cache, None, 0, run.batch, a, None) == pk.E_INVALID
    big = pk.make_geom(1, 2, 512, 64, 0, 1e4, 16, 16, 32)
    assert pk.attention_mass_workspace_bytes(big, run.cache, run.batch, 8) == 0
