"""patchkv_attention against a plain 64-bit reference: every tag and type, ragged batches, windows with sinks, scattered
rows, poisoned slots, strides, refusals, capture, streams.  The bound on each element is derived in live_common."""
import ctypes as C

import numpy as np
import pytest
import torch

from live_common import BF16, F16, Case, Layout, attention64, build_tables, device_batch, random_rows

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


class Setup:
    """A cache (tag 0: the bf16 pool) filled with random tokens for a batch, and its queries."""

    def __init__(self, pk, tag, H, Hq, D, P, G, case: Case, dtype=BF16, seed=1, poison=True, n_rows=None, max_rows=None, max_kv=None):
        rng = np.random.default_rng(seed)
        self.pk, self.case, self.tag, self.share, self.dtype = pk, case, tag, Hq // H, dtype
        self.table, self.n_pages = build_tables(case, P, rng)
        self.geom = pk.make_geom(1, H, D, D, pk.ROPE_HALF, 1e4, 16, P, G)
        self.batch, self.keep = device_batch(pk, case, self.table, DEV, n_rows=n_rows, max_rows=max_rows, max_kv=max_kv)
        n = max(int(self.batch.n_rows), 1)
        self.q = random_rows(rng, n, Hq, D, dtype, outliers=False)
        self.D, self.P = D, P
        shape = (self.n_pages, P, H, D)
        if tag == 0:
            nan = torch.full(shape, float("nan") if poison else 0.0, dtype=BF16)
            k, v = nan.clone(), nan.clone()
            for b, t in enumerate(case.kv):
                kk, vv = random_rows(rng, t, H, D, BF16), random_rows(rng, t, H, D, BF16, outliers=False)
                for j in range(t):
                    k[self.table[b, j // P], j % P], v[self.table[b, j // P], j % P] = kk[j], vv[j]
            self.host = (k, v)
            self.k, self.v = k.to(DEV), v.to(DEV)
            self.cache = pk.make_pool(self.k, self.v, self.n_pages, (0, P * H * D, H * D, D))
        else:
            lay = self.lay = Layout(tag, H, D, P, G)
            # unwritten slots: every byte 0x7E / 0xFF makes the scales NaN
            pages = np.full((self.n_pages, lay.page_bytes()), 0x7F if poison else 0, dtype=np.uint8)
            for b, t in enumerate(case.kv):
                kk = random_rows(rng, t, H, D, BF16).double().numpy()
                vv = random_rows(rng, t, H, D, BF16, outliers=False).double().numpy()
                for j in range(t):
                    lay.put(pages[self.table[b, j // P]], j % P, kk[j], vv[j])
            self.pages = pages
            self.dev = torch.from_numpy(pages).to(DEV)
            self.cache = pk.make_qpool(self.dev, tag, self.n_pages)

    def kv(self, b):
        pages = [int(x) for x in self.table[b, :-(-self.case.kv[b] // self.P)]]
        if not pages:
            z = np.zeros((0, int(self.geom.n_kv_heads), self.D))
            return z, z
        if self.tag == 0:
            return [torch.cat([x[p] for p in pages]).double().numpy()[:self.case.kv[b]] for x in self.host]
        parts = [self.lay.values(self.pages[p]) for p in pages]
        return [np.concatenate([x[i] for x in parts])[:self.case.kv[b]] for i in (0, 1)]

    def workspace(self, window=0, sinks=0):
        n = self.pk.attention_workspace_bytes(self.geom, self.cache, self.batch, self.q.shape[1], window, sinks)
        whole = torch.randint(0, 256, (max(n, 16) + 4096,), dtype=torch.uint8, device=DEV)
        whole[max(n, 16):] = 0xA5
        self.behind = whole[max(n, 16):]
        return whole[:max(n, 16)]

    def run(self, ctx, window=0, sinks=0, scale=None, q=None, out=None, **kw):
        q = self.q.to(DEV) if q is None else q
        out = torch.full_like(q, 5.0) if out is None else out
        kw.setdefault("workspace", self.workspace(window, sinks))
        ctx.attention(self.geom, self.cache, 0, self.batch, q, out, scale=scale, window=window, sinks=sinks, **kw)
        return out

    def reference(self, window=0, sinks=0, scale=None, case=None):
        kv = {}
        def part(i):
            def f(b):
                if b not in kv:
                    kv[b] = self.kv(b)
                return kv[b][i]
            return f
        case = case or self.case
        n = sum(case.rows)
        return attention64(self.q[:n].double().numpy(), part(0), part(1), case, self.share,
                           self.D ** -0.5 if scale is None else scale, window, sinks, self.dtype, self.tag == 0)

    def check(self, ctx, window=0, sinks=0, scale=None, **kw):
        out = self.run(ctx, window, sinks, scale, **kw)
        assert ctx.query_status() == 0
        if hasattr(self, "behind"):
            assert (self.behind == 0xA5).all()           # nothing is written behind the workspace
        want, tol = self.reference(window, sinks, scale)
        n = want.shape[0]
        got = out[:n].double().cpu().numpy()
        err = np.abs(got - want)
        assert np.all(err <= tol), f"worst {np.nanmax(err / tol)} of the bound, NaN {np.isnan(got).sum()}"
        assert (out[n:] == 5.0).all()                    # rows behind the last sequence
        return out


TAGS = [0, 1, 2, 3]
BATCHES = {
    "one_token_cache": Case([1], [1]),
    "decode": Case([700], [1]),
    "decode_long": Case([5001], [1]),
    "decode_ragged": Case([40, 1, 333, 16, 17, 129], [1] * 6),
    "few_rows": Case([200, 65], [3, 5]),
    "prompt": Case([150], [150]),
    "chunk": Case([400, 90], [130, 33]),
    "empty": Case([30, 0, 0, 64], [2, 0, 3, 0]),
    "scattered": Case([500, 100], [20, 4], [[0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 255, 256, 300, 301, 302, 303, 498, 499],
                                          [99, 0, 50, 99]]),
    "more_rows_than_tokens": Case([5], [9]),
    "scattered_many": Case([700, 300], [150, 90], [[(i * 37) % 700 for i in range(150)], [(i * 11) % 300 for i in range(90)]]),
}
MASKS = {"causal": (0, 0), "window": (37, 0), "sinks": (100, 4), "one": (1, 0), "sinks_over": (16, 50),
         "wide": (2 ** 31 - 1, 2 ** 31 - 1)}


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("mask", list(MASKS))
def test_batches_and_masks(pk, ctx, tag, name, mask):
    Setup(pk, tag, 2, 8, 128, 16, 32, BATCHES[name]).check(ctx, *MASKS[mask])


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("H,Hq,D,P,G", [(8, 32, 128, 16, 32), (4, 8, 64, 16, 32), (4, 28, 128, 32, 32), (8, 64, 128, 64, 64),
                                        (1, 8, 64, 16, 64), (3, 3, 128, 16, 128), (32, 32, 64, 16, 32), (1, 71, 64, 16, 32),
                                        (2, 4, 80, 16, 16), (2, 2, 10, 5, 5), (3, 6, 256, 7, 64), (2, 4, 128, 24, 32),
                                        (2, 4, 128, 128, 16), (1, 1, 2, 1, 1), (11, 22, 128, 16, 32)])
@pytest.mark.parametrize("name", ["decode_ragged", "few_rows", "chunk"])
def test_geometries(pk, ctx, tag, H, Hq, D, P, G, name):
    Setup(pk, tag, H, Hq, D, P, G, BATCHES[name]).check(ctx, 50, 3)


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("name", ["decode_long", "decode_ragged", "few_rows", "prompt", "chunk", "scattered"])
def test_fp16(pk, ctx, tag, name):
    Setup(pk, tag, 2, 8, 128, 16, 32, BATCHES[name], dtype=F16).check(ctx)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 16, 17, 64, 65, 128, 129])
def test_row_counts(pk, ctx, tag, rows):
    """Every way the rows of a sequence can fill or overfill a kernel's tile of rows, over a cache long enough to split."""
    Setup(pk, tag, 1, 4, 64, 16, 32, Case([1500, 777], [rows, max(1, rows // 2)])).check(ctx, 600, 4)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("kv", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1023])
@pytest.mark.parametrize("rows", [1, 40])
def test_lengths_at_tile_borders(pk, ctx, tag, kv, rows):
    Setup(pk, tag, 2, 4, 64, 16, 32, Case([kv], [min(kv, rows)])).check(ctx)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 20, 200])
def test_large_and_small_logits(pk, ctx, tag, rows):
    """Logits spread over hundreds (one token takes all), logits all equal, a negative and a zero scale."""
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([300], [rows]))
    for scale in (5.0, 0.0, -0.2, 1e-6):
        s.check(ctx, scale=scale)


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("size", [2.0 ** -12, 2.0 ** 8])
def test_value_ranges(pk, ctx, tag, rows, size):
    """Queries from 2^-30 to 2^40 (bf16 numbers that fp16 does not hold) and values far from one."""
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([150], [rows]))
    q = s.q.float()
    q[:, 0] *= 2.0 ** 40
    q[:, 1] *= 2.0 ** -30
    s.q = q.to(BF16)
    rng = np.random.default_rng(3)
    for j in range(150):
        k, v = (random_rows(rng, 1, 2, 64, BF16).double().numpy()[0] for _ in range(2))
        s.lay.put(s.pages[s.table[0, j // 16]], j % 16, k, v * size)
    s.dev.copy_(torch.from_numpy(s.pages))
    q[:, 0] *= 2.0 ** -40                           # back, and once as large as they are under a small scale
    s.check(ctx, scale=2.0 ** -42)
    s.q = q.to(BF16)
    s.check(ctx)


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("rows", [1, 40, 100, 300])
@pytest.mark.parametrize("D", [64, 128])
def test_fp16_queries_see_whole_keys(pk, ctx, tag, rows, D):
    """Over quantised pages an fp16 query's logits are those of code * scale, not of its fp16 rounding: the bound has no term
    for K.  With a scale of 2^-14 or more the product is a multiple of 2^-24 of at most 19 bits, so two fp16 numbers hold it.
    One channel of K is far larger than the others, where rounding it would show."""
    s = Setup(pk, tag, 2, 4, D, 16, 32, Case([333], [rows]), dtype=F16)
    rng = np.random.default_rng(5)
    for j in range(333):
        k, v = (random_rows(rng, 1, 2, D, BF16, outliers=False).double().numpy()[0] for _ in range(2))
        k[:, 7] *= 300
        s.lay.put(s.pages[s.table[0, j // 16]], j % 16, k, v)
    s.dev.copy_(torch.from_numpy(s.pages))
    s.q[:, :, 7] *= 0.02
    got = s.check(ctx)[:rows].double().cpu().numpy()
    want, tol = attention64(s.q[:rows].double().numpy(), lambda b: s.kv(b)[0], lambda b: s.kv(b)[1], s.case, 2, D ** -0.5, 0, 0, F16,
                            False, k_rounding=0.0)
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_keys_beyond_fp16(pk, ctx, tag, rows, dtype):
    """A key of finite scales whose values pass fp16's range, far on the negative side: a weight of zero, as for one within it."""
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([310], [rows]), dtype=dtype)
    s.q = -s.q.abs() - 0.5
    outs = []
    for size in (4000.0, 120000.0):
        s.lay.put(s.pages[s.table[0, 0]], 5, np.full((2, 64), size), np.ones((2, 64)))
        s.dev.copy_(torch.from_numpy(s.pages))
        outs.append(s.run(ctx))
    assert ctx.query_status() == 0
    assert torch.isfinite(outs[0]).all() and torch.equal(*outs)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [2, 60, 300])
def test_nan_and_infinity_in_unseen_tokens(pk, ctx, tag, rows):
    """A token with NaN and infinities reaches the rows that see it and no other, its neighbours in a tile included."""
    case = Case([400], [rows])
    s = Setup(pk, tag, 2, 4, 64, 16, 32, case)
    at = 400 - max(1, rows // 2)                    # rows before this position do not see the token
    page, slot = s.table[0, at // 16], at % 16
    if tag == 0:
        s.k[page, slot], s.v[page, slot] = float("nan"), float("inf")
    else:
        kc, ks, vc, vs = s.lay.split(s.pages[page])
        for x, bad in ((ks, np.nan), (vs, np.inf)):        # an infinite K could be a logit of -infinity: a weight of zero
            n = 2 * 2 * 64 // 32
            x[slot * n:(slot + 1) * n] = np.array([bad] * (n // 2), np.float16).view(np.uint8)
        s.dev.copy_(torch.from_numpy(s.pages))
    out = s.run(ctx)
    assert ctx.query_status() == 0
    clean = at - (400 - rows)
    assert not torch.isfinite(out[clean:]).any()
    sub = Case([400], [clean], [list(range(400 - rows, at))])
    s.keep_q, s.q = s.q, s.q[:clean]
    if tag == 0:
        s.host[0][page, slot], s.host[1][page, slot] = 0, 0
    else:
        s.lay.put(s.pages[page], slot, np.zeros((2, 64)), np.zeros((2, 64)))
    want, tol = s.reference(case=sub)
    assert np.all(np.abs(out[:clean].double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("rows", [2, 60])
def test_value_infinities_keep_their_channel(pk, ctx, tag, rows):
    """Only the channels whose value is not finite are lost, in the rows that see it."""
    s = Setup(pk, tag, 1, 2, 64, 16, 32, Case([100], [rows]))
    at = 99
    page, slot = s.table[0, at // 16], at % 16
    if tag == 0:
        s.v[page, slot, 0, 5], s.v[page, slot, 0, 6] = float("inf"), float("-inf")
        lost = [5, 6]
    else:
        vs = s.lay.split(s.pages[page])[3]
        vs[slot * 4:slot * 4 + 2] = np.array([np.inf], np.float16).view(np.uint8)
        s.dev.copy_(torch.from_numpy(s.pages))
        lost = list(range(32))
    out = s.run(ctx).float().cpu()
    keep = [c for c in range(64) if c not in lost]
    assert torch.isfinite(out[:-1]).all() and torch.isfinite(out[-1][:, keep]).all()
    assert not torch.isfinite(out[-1][:, lost]).any()
    if tag == 0:
        assert (out[-1][:, 5] == float("inf")).all() and (out[-1][:, 6] == float("-inf")).all()


@pytest.mark.parametrize("tag", [0, 3])
@pytest.mark.parametrize("rows", [1, 50])
def test_strides(pk, ctx, tag, rows):
    """Queries and results [Hq][n][D], padded, and off the 16-byte grid."""
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([90, 70], [rows, rows]))
    n = 2 * rows
    s.check(ctx)
    q = s.q.to(DEV)
    heads_first = torch.empty((4, n, 64), dtype=BF16, device=DEV).transpose(0, 1)
    padded = torch.full((n, 5, 72), 5.0, dtype=BF16, device=DEV)
    shifted = torch.empty(n * 256 + 1, dtype=BF16, device=DEV)[1:].view(n, 4, 64)
    for view in (heads_first, padded[:, :4, :64], shifted):
        view.copy_(q)
        s.check(ctx, q=view)
        out = s.check(ctx, out=view)
        assert out.data_ptr() == view.data_ptr()
    assert (padded[:, 4] == 5).all() and (padded[:, :, 64:] == 5).all()


@pytest.mark.parametrize("tag", [0])
@pytest.mark.parametrize("rows", [1, 50])
def test_pool_layouts(pk, ctx, tag, rows):
    """The bf16 pool with heads outside tokens, padded pages, a second layer, and strides off the 16-byte grid."""
    s = Setup(pk, 0, 2, 4, 64, 16, 32, Case([90, 70], [rows, rows]))
    want = s.run(ctx)
    g = pk.make_geom(2, 2, 64, 64, pk.ROPE_HALF, 1e4, 16, 16, 32)
    for strides in ((0, 2 * 16 * 64 + 64, 64, 16 * 64 + 8), (s.n_pages * 2112, 2112, 132, 65), (s.n_pages * 2200, 2200, 128, 64)):
        size = 2 * max(strides[0], 1) + s.n_pages * strides[1] + 4096
        k, v = torch.full((size,), float("nan"), dtype=BF16, device=DEV), torch.full((size,), float("nan"), dtype=BF16, device=DEV)
        for x, src in ((k, s.k), (v, s.v)):
            torch.as_strided(x, (s.n_pages, 16, 2, 64), (strides[1], strides[2], strides[3], 1), strides[0]).copy_(src)
        pool = pk.make_pool(k, v, s.n_pages, strides)
        out = torch.zeros_like(want)
        ctx.attention(g, pool, 1, s.batch, s.q.to(DEV), out, workspace=s.workspace())
        assert ctx.query_status() == 0
        # another kernel may take another order of sums: a bf16 step of the largest value
        assert (out.float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()


@pytest.mark.parametrize("tag", [0, 1, 3])
@pytest.mark.parametrize("rows", [1, 40])
def test_out_of_range_is_left_out_and_latched(pk, ctx, tag, rows):
    case = Case([100, 200], [rows, rows])
    for what in ("bad_page", "kv_len", "short_table", "max_rows", "row_start"):
        s = Setup(pk, tag, 2, 4, 64, 16, 32, case)
        seen = case
        if what == "bad_page":
            s.keep["table"][1, 0] = s.n_pages
        elif what == "kv_len":
            s.batch.max_kv_len = 150
            seen = Case([100, 150], case.rows, case.positions())
        elif what == "short_table":
            s.keep["table2"] = s.keep["table"][:, :10].contiguous()
            s.batch.block_table, s.batch.table_stride = s.keep["table2"].data_ptr(), 10
            seen = Case([100, 160], case.rows, case.positions())
        elif what == "max_rows":
            if rows == 1:
                continue
            s.batch.max_rows = rows - 7
        else:
            s.keep["start"][2] = 0
        out = s.run(ctx)
        assert ctx.query_status() == pk.E_BOUNDS, what
        got = out.double().cpu().numpy()
        if what == "row_start":
            assert (out[rows:] == 5).all()
            seen = Case([100], [rows])
        elif what == "max_rows":
            for b in (0, 1):
                assert (out[(b + 1) * rows - 7:(b + 1) * rows] == 5).all()
                assert not (out[b * rows:(b + 1) * rows - 7] == 5).all()
            continue
        if what == "bad_page":                       # page 0 of sequence 1 is not seen
            full = s.kv
            s.kv = lambda b: [x[16 * b:] for x in full(b)]
            seen = Case([100, 184], case.rows, [case.positions()[0], [p - 16 for p in case.positions()[1]]])
        s.q = s.q[:sum(seen.rows)]
        kv = s.kv
        s.kv = lambda b: [x[:seen.kv[b]] for x in kv(b)]
        want, tol = s.reference(case=seen)
        assert np.all(np.abs(got[:want.shape[0]] - want) <= tol), what


@pytest.mark.parametrize("tag", [0, 3])
def test_negative_positions_give_zeros(pk, ctx, tag):
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([50, 7], [3, 2], [[-1, 4, -2000000000], [2000000000, 6]]))
    out = s.check(ctx, 40, 2)
    assert (out[0] == 0).all() and (out[2] == 0).all()
    assert (out[3] == out[3]).all()


@pytest.mark.parametrize("tag", [0, 2])
@pytest.mark.parametrize("rows", [1, 30])
def test_captured_and_replayed(pk, ctx, tag, rows):
    """A captured call follows the contents of its device arrays; the workspace's contents do not matter."""
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([900, 500], [rows, rows]))
    q = s.q.to(DEV)
    out = torch.zeros_like(q)
    ws = s.workspace()
    s.run(ctx, q=q, out=out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.attention(s.geom, s.cache, 0, s.batch, q, out, workspace=ws)
    for kv in ([900, 500], [600, 499], [rows, 1]):
        s.keep["kv"].copy_(torch.tensor(kv, dtype=torch.int32))
        ws.random_(0, 256)
        graph.replay()
        assert ctx.query_status() == 0
        case = Case(kv, [rows, rows])
        full = Setup.kv
        s.case = Case([900, 500], [rows, rows])
        s.kv = lambda b: [x[:kv[b]] for x in full(s, b)]
        want, tol = s.reference(case=case)
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("rows", [1, 30])
def test_two_streams_at_once(pk, ctx, rows):
    s = [Setup(pk, 3, 2, 8, 128, 16, 32, Case([4000], [rows]), seed=i) for i in range(2)]
    q = [x.q.to(DEV) for x in s]
    want = [x.run(ctx).clone() for x in s]
    ws = [x.workspace() for x in s]
    out = [torch.zeros_like(x) for x in q]
    streams = [torch.cuda.Stream() for _ in s]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in (0, 1):
            ctx.attention(s[i].geom, s[i].cache, 0, s[i].batch, q[i], out[i], workspace=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    assert ctx.query_status() == 0
    for i in (0, 1):
        assert torch.equal(out[i], want[i])             # the same bits, whatever runs beside


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 7, 64])
def test_same_bits_every_time(pk, ctx, tag, rows):
    s = Setup(pk, tag, 4, 16, 128, 16, 32, Case([3000, 100], [rows, rows]))
    a = s.run(ctx)
    for _ in range(5):
        assert torch.equal(s.run(ctx), a)


@pytest.mark.parametrize("rows", [1, 20])
def test_append_then_attend_as_a_decode_loop(pk, ctx, rows):
    """Chunks of a context appended one after the other, each attended as it arrives, on one stream without waiting."""
    H, Hq, D, P, G, tag = 2, 8, 128, 16, 32, 3
    lay = Layout(tag, H, D, P, G)
    rng = np.random.default_rng(9)
    steps = 12
    total = steps * rows + 61
    table = rng.permutation(-(-total // P))[None].astype(np.int32)
    pages = np.full((table.size, lay.page_bytes()), 0x7F, dtype=np.uint8)
    dev = torch.from_numpy(pages).to(DEV)
    cache, g = pk.make_qpool(dev, tag, table.size), pk.make_geom(1, H, D, D, pk.ROPE_HALF, 1e4, 16, P, G)
    k, v, q = (random_rows(rng, total, h, D, BF16) for h in (H, H, Hq))
    kd, vd, qd = k.to(DEV), v.to(DEV), q.to(DEV) * 0.2
    q = qd.cpu()
    outs, keeps, at = [], [], 0
    for n in [61] + [rows] * steps:
        case = Case([at + n], [n])
        batch, keep = device_batch(pk, case, table, DEV)
        out = torch.zeros_like(qd[at:at + n])
        ws = torch.empty(max(16, pk.attention_workspace_bytes(g, cache, batch, Hq, 64, 4)), dtype=torch.uint8, device=DEV)
        ctx.cache_append(g, cache, 0, batch, kd[at:at + n], vd[at:at + n])
        ctx.attention(g, cache, 0, batch, qd[at:at + n], out, window=64, sinks=4, workspace=ws)
        outs.append(out)
        keeps.append((batch, keep, ws))
        at += n
    assert ctx.query_status() == 0
    for j in range(total):
        lay.put(pages[table[0, j // P]], j % P, k[j].double().numpy(), v[j].double().numpy())
    vals = [lay.values(pages[p]) for p in table[0]]
    K, V = (np.concatenate([x[i] for x in vals])[:total] for i in (0, 1))
    want, tol = attention64(q.double().numpy(), lambda b: K, lambda b: V, Case([total], [total]), Hq // H, D ** -0.5, 64, 4, BF16, False)
    assert np.all(np.abs(torch.cat(outs).double().cpu().numpy() - want) <= tol)


def test_restore_then_attend(pk, ctx):
    """The resume path and what follows it: a checkpoint restored into the pool, then repair rows attending over it."""
    import patchkv_inputs as pin
    from patchkv_inputs.staging import StagedCheckpoint, device_pool
    ck = pin.config_tiny(dirty_tokens=0, top_k=0)
    st = StagedCheckpoint(ck, DEV)
    ctx.select_repair(st.select_args())
    k, v, pool = device_pool(ck, DEV)
    ctx.restore(st.geom(), pool, [st.session()])
    g, n = ck.geom, ck.n_suffix_tokens
    case = Case([n], [40], [sorted(np.random.default_rng(2).permutation(n)[:40].tolist())])
    table = ck.block_table.numpy()[None].astype(np.int32)
    batch, keep = device_batch(pk, case, table, DEV)
    q = random_rows(np.random.default_rng(1), 40, 8, g.head_dim, BF16, outliers=False) * 0.2
    out = torch.zeros_like(q, device=DEV)
    ws = torch.empty(max(16, pk.attention_workspace_bytes(st.geom(), pool, batch, 8)), dtype=torch.uint8, device=DEV)
    ctx.attention(st.geom(), pool, 1, batch, q.to(DEV), out, workspace=ws)
    assert ctx.query_status() == 0
    rows = lambda x: x.view(BF16).view(g.n_layers, -1, g.page_tokens, g.n_kv_heads, g.head_dim)[1][table[0].tolist()].flatten(0, 1)[:n].double().cpu().numpy()
    K, V = rows(k), rows(v)
    want, tol = attention64(q.double().numpy(), lambda b: K, lambda b: V, case, 8 // g.n_kv_heads, g.head_dim ** -0.5, 0, 0, BF16, True)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)


def test_pages_past_4_gib(pk, ctx):
    """Element and byte offsets of pages beyond 32 bits, quantised and bf16."""
    for tag in (3, 0):
        for rows in (1, 30):
            s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([40], [rows]), poison=False)
            n = s.n_pages
            if tag:
                stride = 1 << 30
                big = torch.empty((n - 1) * stride + s.lay.page_bytes(), dtype=torch.uint8, device=DEV)
                for i in range(n):
                    big[i * stride:i * stride + s.lay.page_bytes()] = s.dev[i]
                s.cache = pk.make_qpool(big.view(1, -1), tag, n, stride_page=stride)
            else:
                stride = 1 << 29
                kv = [torch.empty((n - 1) * stride + 2048, dtype=BF16, device=DEV) for _ in range(2)]
                for x, src in zip(kv, (s.k, s.v)):
                    for i in range(n):
                        x[i * stride:i * stride + 2048] = src[i].reshape(-1)
                s.cache = pk.make_pool(kv[0], kv[1], n, (0, stride, 128, 64))
            s.check(ctx)
            big = kv = s.cache = None


def test_refusals(pk, ctx):
    s = Setup(pk, 3, 4, 8, 64, 16, 32, Case([2000], [3]))
    p = Setup(pk, 0, 4, 8, 64, 16, 32, Case([2000], [3]))
    q = s.q.to(DEV)
    out = torch.full_like(q, 5.0)
    ws = s.workspace()

    def args(**kw):
        a = pk.AttentionArgs(C.sizeof(pk.AttentionArgs), 0, 8, 0, 0, 0.125, q.data_ptr(), out.data_ptr(), 512, 64, 512, 64, ws.data_ptr(), ws.numel())
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    def call(a, geom=s.geom, pool=None, cache=s.cache, layer=0, batch=s.batch):
        return pk.lib().patchkv_attention(ctx._h, C.byref(geom), None if pool is None else C.byref(pool),
                                          None if cache is None else C.byref(cache), layer, C.byref(batch), C.byref(a), None)

    assert call(args()) == 0
    torch.cuda.synchronize()
    out.fill_(5.0)
    for kw in (dict(struct_size=4), dict(type=2), dict(n_q_heads=0), dict(n_q_heads=6), dict(window=-1), dict(sinks=-1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(out=None), dict(q=q.data_ptr() + 1),
               dict(q_stride_row=-1), dict(out_stride_head=-8), dict(out_stride_head=32), dict(out_stride_row=64)):
        assert call(args(**kw)) == pk.E_INVALID, kw
    need = pk.attention_workspace_bytes(s.geom, s.cache, s.batch, 8)
    if need:
        for kw in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=ws.data_ptr() + 8)):
            assert call(args(**kw)) == pk.E_INVALID, kw
    assert call(args(), pool=p.cache) == pk.E_INVALID and call(args(), cache=None) == pk.E_INVALID
    assert call(args(type=1), pool=p.cache, cache=None) == pk.E_INVALID
    assert call(args(), layer=1) == pk.E_INVALID
    for field, value in (("k_base", None), ("n_pages", 0), ("stride_token", -1), ("struct_size", 0), ("v_base", p.v.data_ptr() + 2)):
        bad = pk.Pool.from_buffer_copy(p.cache)
        setattr(bad, field, value)
        assert call(args(), pool=bad, cache=None) == pk.E_INVALID, field
    wide = pk.make_geom(1, 4, 512, 64, 0, 1e4, 16, 16, 32)
    big = pk.make_qpool(torch.zeros((2, pk.record_bytes(3, 16, 4, 512, 32)), dtype=torch.uint8, device=DEV), 3, 2)
    assert call(args(), geom=wide, cache=big) == pk.E_UNSUPPORTED
    with pytest.raises(ValueError):
        ctx.attention(s.geom, s.cache, 0, s.batch, q.float(), out.float())
    with pytest.raises(ValueError):
        ctx.attention(s.geom, s.cache, 0, s.batch, q, out[:, :4])
    none = pk.Batch.from_buffer_copy(s.batch)
    none.n_seqs = 0
    assert call(args(), batch=none) == 0
    torch.cuda.synchronize()
    assert ctx.query_status() == 0 and (out == 5).all()


@pytest.mark.parametrize("tag", [0, 1, 3])
@pytest.mark.parametrize("n_seqs", [33, 100, 400])
def test_many_sequences(pk, ctx, tag, n_seqs):
    """More sequences than a warp has lanes, than SMs, and than pieces are worth."""
    rng = np.random.default_rng(n_seqs)
    kv = [int(x) for x in rng.integers(0, 90, n_seqs)]
    kv[n_seqs // 2] = 3000
    rows = [int(x) for x in rng.integers(0, 3, n_seqs)]
    Setup(pk, tag, 1, 2, 64, 16, 32, Case(kv, rows)).check(ctx, 200, 3)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 30, 200])
def test_pages_behind_the_window_may_be_gone(pk, ctx, tag, rows):
    """Table entries of tokens that no row sees may be anything; nothing is read there and nothing latched."""
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([900], [rows]))
    first = (900 - rows - 100 + 1) // 16                 # page of the first token in the earliest row's window
    s.keep["table"][0, 1:first] = torch.arange(first - 1, dtype=torch.int32, device=DEV) * -7 - 1
    s.check(ctx, 100, 5)


@pytest.mark.parametrize("tag", TAGS)
@pytest.mark.parametrize("rows", [1, 30, 200])
def test_a_broken_query_spoils_only_itself(pk, ctx, tag, rows):
    s = Setup(pk, tag, 2, 4, 64, 16, 32, Case([300, 0], [rows, rows]))
    good, tol = s.reference()
    s.q[0, 1, 3], s.q[rows - 1, 2, 60], s.q[rows, 0, 0] = float("nan"), float("inf"), float("nan")
    out = s.run(ctx)
    assert ctx.query_status() == 0
    got = out.double().cpu().numpy()
    assert np.isnan(got[0, 1]).all() and not np.isfinite(got[rows - 1, 2]).any()
    for r, h in ((0, 1), (rows - 1, 2)):
        got[r, h] = good[r, h]
    assert np.all(np.abs(got - good) <= tol)             # the second sequence has no tokens: zeros, whatever its queries


def test_two_graphs_with_workspaces_of_their_own(pk, ctx):
    s = [Setup(pk, 3, 2, 8, 128, 16, 32, Case([3000], [r]), seed=r) for r in (1, 90)]
    q = [x.q.to(DEV) for x in s]
    out, ws, graphs = [torch.zeros_like(x) for x in q], [x.workspace() for x in s], []
    for i in (0, 1):
        s[i].run(ctx, q=q[i], out=out[i], workspace=ws[i])
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            ctx.attention(s[i].geom, s[i].cache, 0, s[i].batch, q[i], out[i], workspace=ws[i])
        graphs.append(g)
    want = [x.clone() for x in out]
    streams = [torch.cuda.Stream() for _ in s]
    for _ in range(10):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert ctx.query_status() == 0
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_first_call_of_a_process_may_be_captured():
    """Nothing of the calls has to be warmed up outside a capture: a fresh process captures its first ones."""
    import subprocess
    import sys
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import torch
from paper_2609_26219_b200 import binding as pk
dev = "cuda:0"
ctx = pk.Context(device=0)
g = pk.make_geom(1, 2, 64, 64, pk.ROPE_HALF, 1e4, 16, 16, 32)
pages = torch.zeros((64, pk.record_bytes(3, 16, 2, 64, 32)), dtype=torch.uint8, device=dev)
cache = pk.make_qpool(pages, 3, 64)
for rows in (1, 40, 300):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    b = dict(row_start=i32([0, rows]), kv_len=i32([700]), block_table=torch.arange(64, dtype=torch.int32, device=dev)[None], n_rows=rows, max_rows=rows, max_kv_len=700)
    batch = pk.make_batch(**b)
    k = torch.ones((rows, 2, 64), dtype=torch.bfloat16, device=dev)
    q = torch.ones((rows, 4, 64), dtype=torch.bfloat16, device=dev)
    out = torch.zeros_like(q)
    ws = torch.empty(max(16, pk.attention_workspace_bytes(g, cache, batch, 4)), dtype=torch.uint8, device=dev)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.cache_append(g, cache, 0, batch, k, k)
        ctx.attention(g, cache, 0, batch, q, out, workspace=ws)
    graph.replay()
    assert ctx.query_status() == 0
    assert torch.isfinite(out).all() and float(out[0].float().mean()) > 0
print("ok")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stderr[-2000:]
