"""CPU checks of the entry points around the attention: struct sizes, refusals that need no device, the reference itself."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from rotary_common import HALF, INTERLEAVED, frequencies, rotate64

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
  printf("%zu %zu %zu %zu\n", sizeof(patchkv_rotary_args), sizeof(patchkv_mass_args), sizeof(patchkv_evict_args), sizeof(patchkv_gather_args));
  printf("%zu %zu %zu %zu\n", offsetof(patchkv_rotary_args, rope_pos), offsetof(patchkv_mass_args, mass_stride),
         offsetof(patchkv_evict_args, mass_out), offsetof(patchkv_gather_args, dst_table));
  printf("%d %d\n", PATCHKV_MASS_F32, PATCHKV_MASS_U64);
  return 0; }
'''
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "s.c"), os.path.join(d, "s")
        open(c, "w").write(src)
        subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), c, "-o", exe])
        got = [int(x) for x in subprocess.check_output([exe]).decode().split()]
    assert got[:4] == [ctypes.sizeof(x) for x in (pk.RotaryArgs, pk.MassArgs, pk.EvictArgs, pk.GatherArgs)]
    assert got[4:8] == [pk.RotaryArgs.rope_pos.offset, pk.MassArgs.mass_stride.offset, pk.EvictArgs.mass_out.offset, pk.GatherArgs.dst_table.offset]
    assert got[8:] == [pk.MASS_F32, pk.MASS_U64]


def test_null_context_is_refused(pk):
    lib, g = pk.lib(), pk.make_geom(1, 1, 64, 64, 0, 1e4, 16, 16, 32)
    assert lib.patchkv_rotary_append(None, g, None, None, 0, None, None, None) == pk.E_INVALID
    assert lib.patchkv_attention_mass(None, g, None, None, 0, None, None, None) == pk.E_INVALID
    assert lib.patchkv_evict_select(None, None, None) == pk.E_INVALID
    assert lib.patchkv_cache_gather(None, g, None, None, 0, None, None) == pk.E_INVALID


def _batch(pk, n_seqs, n_rows, max_rows, max_kv):
    return pk.Batch(ctypes.sizeof(pk.Batch), n_seqs, n_rows, max_rows, max_kv, 4, 16, 16, None, 16)


def test_workspace_size_of_bad_arguments_is_zero(pk):
    lib = pk.lib()
    g = pk.make_geom(1, 8, 128, 128, 0, 1e4, 16, 16, 32)
    ok = _batch(pk, 1, 1, 1, 16384)
    size = lambda geom, tag, b, hq, w=0, s=0: lib.patchkv_attention_mass_workspace_bytes(geom, tag, b, hq, w, s)
    assert size(g, 3, ok, 32) > 0
    assert size(g, 3, ok, 31) == 0 and size(g, 7, ok, 32) == 0 and size(g, 3, ok, 32, -1) == 0 and size(g, 3, ok, 32, 0, -1) == 0
    assert size(g, 3, _batch(pk, -1, 1, 1, 5), 32) == 0 and size(pk.make_geom(1, 8, 129, 128, 0, 1e4, 16, 16, 32), 3, ok, 32) == 0


def test_the_reference_turns_by_sums_of_angles():
    """R(a) R(b) = R(a + b), norms of pairs stay, and channels behind the rotary ones are left."""
    rng = np.random.default_rng(0)
    x, theta = rng.standard_normal((5, 3, 20)), frequencies(12, 1e4)
    for style in (HALF, INTERLEAVED):
        a = rotate64(rotate64(x, [3] * 5, theta, style), [-10] * 5, theta, style)
        assert np.allclose(a, rotate64(x, [-7] * 5, theta, style)) and np.array_equal(a[..., 12:], x[..., 12:])
        assert np.allclose((a ** 2).sum(-1), (x ** 2).sum(-1))


def test_workspace_holds_the_sums_of_the_element_wise_kernel(pk):
    """Calls of one shape go to another kernel when their queries are not aligned: one workspace has to do for both, however loose the
    bound on the rows is."""
    lib = pk.lib()
    for D in (64, 128, 80):
        g = pk.make_geom(1, 2, D, D, 0, 1e4, 16, 16, 16 if D == 80 else 32)
        for n_rows, max_rows in ((1, 1), (1000000, 1), (5000, 3), (5000, 900)):
            assert lib.patchkv_attention_mass_workspace_bytes(g, 3, _batch(pk, 1, n_rows, max_rows, 64), 8, 0, 0) >= n_rows * 8 * 4


def test_workspace_goes_by_the_block_table_where_that_is_smaller(pk):
    g = pk.make_geom(1, 8, 128, 128, 0, 1e4, 16, 16, 32)
    size = lambda rows, kv: pk.lib().patchkv_attention_mass_workspace_bytes(g, 3, _batch(pk, 1, rows, rows, kv), 32, 0, 0)
    for rows in (1, 100):
        assert 0 < size(rows, 64) == size(rows, 2 ** 31 - 1)          # four pages of 16 tokens


def test_binding_refuses_host_tensors(pk):
    """A host address in a kernel would be a fault of the GPU."""
    f, i = torch.zeros((2, 8)), torch.zeros((2, 8), dtype=torch.int32)
    for call in (lambda: pk._mass_rows(f, "mass", (torch.float32,), 2), lambda: pk._table_rows(i, "keep", 2), lambda: pk._counts(i[0], "kept", 2),
                 lambda: pk._rows(torch.zeros((2, 2, 8), dtype=torch.bfloat16), "q")):
        with pytest.raises(ValueError):
            call()
