"""The library's code depends on its sources alone."""
import os

from paper_2609_26219_b200 import build


def test_every_source_is_compiled_once_and_whole():
    """Compiled in pieces that a scheduler cuts, the same sources gave other code at every build, and other times with it."""
    assert sorted(build.SOURCES) == sorted(f for f in os.listdir(build.CSRC) if f.endswith(".cu"))
    assert len(set(build.SOURCES)) == len(build.SOURCES)
    assert not any("split" in f or "threads" in f for f in build.FLAGS)
