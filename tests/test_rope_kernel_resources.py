"""What the compiler makes of the norms' and rotations' kernels: no instance keeps registers in scratch memory, and wavefronts to a SIMD as their
launches count on."""
import pytest

from tests.test_paged_kernel_resources import resources


@pytest.mark.parametrize("source, instances, least", [
    ("rf2_rope.hip", 54, dict(apply_kernel=6, backward_kernel=4, runs_kernel=4, join_kernel=8)),
    ("rf2_permute_rope.hip", 28, dict(permute_rope_kernel=3, permute_v_kernel=8)),
    ("rf2_paged_store_rope.hip", 32, dict(store_rope_kernel=4)),
])
def test_no_instance_uses_scratch_memory(source, instances, least, tmp_path):
    found = resources(source, tmp_path)
    assert len(found) == instances
    assert not [f for f in found if f[1] != "0" or f[3] != "0"]
    for name, _, waves, _ in found:
        assert [n for n in least if n in name and int(waves) >= least[n]], (name, waves)
