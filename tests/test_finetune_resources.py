"""Register budget of the packed attention's, the fine-tuning losses' and the clipping's kernels (CPU
only: a compile, no launch): no scratch memory, no spilled VGPR, two waves of attention on a SIMD."""
import pytest

from test_functional_resources import _kernels

# unit -> kernels it must hold
KERNELS = {
    "packed.hip": ("k_packed_plan", "k_packed_fwd", "k_packed_dq", "k_packed_dkv", "k_packed_sum"),
    "finetune.hip": ("k_token_fwd", "k_token_bwd", "k_pairs", "k_few_pairs", "k_pairs_mean", "k_policy_count", "k_policyI", "k_policy_mean"),
    "clip.hip": ("k_norm_pieces", "k_normE", "k_clip_pieces"),
}


@pytest.mark.parametrize("unit", list(KERNELS))
def test_kernels_use_no_scratch(unit):
    kernels = _kernels(unit)
    for name in KERNELS[unit]:
        assert any(name in k for k in kernels), f"no {name} in {unit}"
    for name, use in kernels.items():
        assert use["ScratchSize"] == 0 and use["VGPRs Spill"] == 0, (name, use)


def test_two_waves_of_attention_on_a_simd():
    for name, use in _kernels("packed.hip").items():
        assert use["Occupancy"] >= 2, (name, use)
