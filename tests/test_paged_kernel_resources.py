"""What the kernels of the rotation and of the paged cache take of a compute unit: the paged kernels are laid out for one or two workgroups
beside each other, and registers kept in scratch memory would be loaded between their tiles."""
import pytest

from test_kernel_resources import _named, kernels  # noqa: F401  (a fixture)

pytest.importorskip("msgpack")


def test_nothing_in_scratch_memory(kernels):  # noqa: F811
    for name, k in _named(kernels, "paged_few|paged_append|rope_fwd|rope_bwd|rope_weight").items():
        assert k[".private_segment_fixed_size"] == 0, name
    for name, k in _named(kernels, "paged_many").items():
        # (head_dim 64, two workgroups a unit, 128 registers: what a span keeps, one value of it read in the loop over tiles)
        most = 80 if "ELi64ELb0E" in name else 0
        assert k[".private_segment_fixed_size"] <= most, (name, k[".private_segment_fixed_size"])


def test_workgroups_that_share_a_unit_fit(kernels):  # noqa: F811
    unit = 160 * 1024
    for name, k in _named(kernels, "paged_few").items():
        assert 2 * k[".group_segment_fixed_size"] <= unit, name
        assert k[".vgpr_count"] <= 256, name             # two waves a SIMD
    for name, k in _named(kernels, "paged_many").items():
        two = "ELi64ELb0E" in name
        assert (2 if two else 1) * k[".group_segment_fixed_size"] <= unit, name
        assert k[".vgpr_count"] <= (128 if two else 256), name
