"""CPU checks of the live-cache entry points: struct sizes, the page reference itself, refusals that need no device."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from live_common import BITS, Layout, quantise64

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pk():
    from paper_2609_26219_b200 import build, binding
    build.build()
    binding.lib()
    return binding


def test_structs_match_the_header(pk):
    src = r'''
#include "patchkv.h"
#include <stdio.h>
int main(void) {
  printf("%zu %zu %zu %zu\n", sizeof(patchkv_qpool), sizeof(patchkv_batch), sizeof(patchkv_rows), sizeof(patchkv_attention_args));
  printf("%zu %zu %zu %zu\n", offsetof(patchkv_qpool, stride_page), offsetof(patchkv_batch, block_table),
         offsetof(patchkv_rows, stride_head), offsetof(patchkv_attention_args, workspace));
  return 0; }
'''
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "s.c"), os.path.join(d, "s")
        open(c, "w").write(src)
        subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), c, "-o", exe])
        got = [int(x) for x in subprocess.check_output([exe]).decode().split()]
    kinds = (pk.QPool, pk.Batch, pk.Rows, pk.AttentionArgs)
    assert got[:4] == [ctypes.sizeof(x) for x in kinds]
    assert got[4:] == [pk.QPool.stride_page.offset, pk.Batch.block_table.offset, pk.Rows.stride_head.offset,
                       pk.AttentionArgs.workspace.offset]


@pytest.mark.parametrize("tag", [1, 2, 3])
@pytest.mark.parametrize("H,D,P,G", [(8, 128, 16, 32), (1, 2, 1, 1), (3, 10, 5, 5)])
def test_a_page_is_one_record(pk, tag, H, D, P, G):
    lay = Layout(tag, H, D, P, G)
    assert sum(lay.sections()) == pk.record_bytes(tag, P, H, D, G)
    rng = np.random.default_rng(1)
    page = np.zeros(lay.page_bytes(), np.uint8)
    x = rng.standard_normal((2, H, D))
    lay.put(page, P - 1, x[0], x[1])
    for got, want, bits in zip(lay.values(page), x, BITS[tag]):
        q, s = quantise64(want, bits, G)
        assert np.array_equal(got[P - 1], (q.reshape(H, -1, G) * s.astype(np.float64)[..., None]).reshape(H, D))
        assert np.all(got[:P - 1] == 0)


def test_null_context_is_refused(pk):
    lib = pk.lib()
    g = pk.make_geom(1, 1, 64, 64, 0, 1e4, 16, 16, 32)
    for f in (lib.patchkv_cache_append, lib.patchkv_cache_read):
        assert f(None, ctypes.byref(g), None, 0, None, None, None) == pk.E_INVALID
    assert lib.patchkv_attention(None, ctypes.byref(g), None, None, 0, None, None, None) == pk.E_INVALID


def _batch(pk, n_seqs, n_rows, max_rows, max_kv):
    return pk.Batch(ctypes.sizeof(pk.Batch), n_seqs, n_rows, max_rows, max_kv, 4, 16, 16, None, 16)


def test_workspace_size_of_bad_arguments_is_zero(pk):
    lib = pk.lib()
    g = pk.make_geom(1, 8, 128, 128, 0, 1e4, 16, 16, 32)
    ok = _batch(pk, 1, 1, 1, 16384)
    size = lambda geom, tag, b, hq, w=0, s=0: lib.patchkv_attention_workspace_bytes(ctypes.byref(geom), tag, ctypes.byref(b), hq, w, s)
    assert size(g, 3, ok, 31) == 0 and size(g, 7, ok, 32) == 0 and size(g, 3, ok, 32, -1) == 0 and size(g, 3, ok, 32, 0, -1) == 0
    assert size(g, 3, _batch(pk, -1, 1, 1, 5), 32) == 0 and size(g, 3, _batch(pk, 1, 0, 0, 0), 32) == 0
    odd = pk.make_geom(1, 8, 129, 128, 0, 1e4, 16, 16, 32)
    assert size(odd, 3, ok, 32) == 0


def test_binding_refuses_what_it_can_see(pk):
    t = torch.zeros((2, 10), dtype=torch.int32)
    with pytest.raises(ValueError):
        pk.make_qpool(torch.zeros((4, 8), dtype=torch.int16), 3, 4)
    with pytest.raises(ValueError):
        pk.make_batch(row_start=t[0], kv_len=torch.zeros(2, dtype=torch.int64), block_table=t, n_rows=1, max_rows=1, max_kv_len=1)
    with pytest.raises(ValueError):
        pk.make_batch(row_start=t[0, :2], kv_len=t[:, 0].contiguous(), block_table=t, n_rows=1, max_rows=1, max_kv_len=1)
    with pytest.raises(ValueError):
        pk.make_batch(row_start=t[0], kv_len=t[:, 0].contiguous(), block_table=t[:, ::2], n_rows=1, max_rows=1, max_kv_len=1)
    with pytest.raises(ValueError):
        pk.make_batch(row_start=t[0], kv_len=t[:, 0].contiguous(), block_table=t, n_rows=3, max_rows=1, max_kv_len=1, pos=t[0, :2])
