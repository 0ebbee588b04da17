"""The sizes of workspaces for bounds of all magnitudes, zeros among them: asked for in a process of their own, which has to live.  Needs no GPU."""
import subprocess
import sys

import pytest

PROGRAM = r"""
import ctypes, random, sys
from paper_2609_26219_b200 import binding as pk
lib, rng = pk.lib(), random.Random(int(sys.argv[1]))
counts = [0, 1, 2, 3, 5, 16, 17, 64, 100, 999, 4096, 65535, 10 ** 6, 2 ** 30 + 1, 2 ** 31 - 1]
some = lambda: rng.choice(counts)
sizes = []
for i in range(20000):
    D = rng.choice([2, 64, 80, 128, 256])
    H = rng.choice([1, 2, 3, 8, 40])
    g = pk.make_geom(1, H, D, D, 0, 1e4, 16, rng.choice([1, 16, 48, 1024]), rng.choice([G for G in (1, 2, 16, 32, 64, 128) if D % G == 0]))
    b = pk.Batch(ctypes.sizeof(pk.Batch), some() if i else 0, some() if i else 100, some() if i else 100, some(), some(), None, None, None, None)
    a = (g, rng.randrange(4), b, H * rng.choice([1, 2, 4, 8, 33]), rng.choice([0, 0, 1, 100, 2 ** 31 - 1]), rng.choice([0, 0, 4, 2 ** 31 - 1]))
    sizes.append((lib.patchkv_attention_workspace_bytes(*a), lib.patchkv_attention_mass_workspace_bytes(*a)))
print(max(s[0] for s in sizes), max(s[1] for s in sizes))
"""


@pytest.mark.parametrize("seed", [0, 1])
def test_any_bounds(seed):
    from paper_2609_26219_b200 import build
    build.build()
    out = subprocess.run([sys.executable, "-c", PROGRAM, str(seed)], cwd=build.ROOT, capture_output=True, text=True)
    assert out.returncode == 0, (out.returncode, out.stderr)
    assert all(0 < int(x) < 2 ** 63 for x in out.stdout.split())
