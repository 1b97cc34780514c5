"""The kernel-source hash that guards the benchmark's committed records (HBM traffic, the
peak N) follows the units that the benchmark's kernels are built from, and no others."""
import bench
from paper_2609_24089_amd import build


def test_hash_ignores_other_units(monkeypatch):
    base = bench.kernel_source_hash()
    monkeypatch.setattr(build, "SOURCES", build.SOURCES + [("fb_something_else.hip", ["-O1"])])
    assert bench.kernel_source_hash() == base
    own = [unit for unit in build.SOURCES if unit[0] in bench.KERNEL_SOURCES]
    monkeypatch.setattr(build, "SOURCES", own)
    assert bench.kernel_source_hash() == base


def test_hash_follows_its_own_units(monkeypatch):
    base, units = bench.kernel_source_hash(), build.SOURCES
    for i, (name, flags) in enumerate(units):
        changed = list(units)
        changed[i] = (name, flags + ["-O1"])
        monkeypatch.setattr(build, "SOURCES", changed)
        assert (bench.kernel_source_hash() != base) == (name in bench.KERNEL_SOURCES), name


def test_every_kernel_source_is_hashed():
    """Each unit of the library is either hashed or one of the two-length kernels'."""
    for name, _ in build.SOURCES:
        assert name in bench.KERNEL_SOURCES or name.startswith("fb_ext"), name
