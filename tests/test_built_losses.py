"""The built kernels of the losses and of gradient clipping: nothing spilled, and as many waves to a SIMD as their rows in
registers are laid out for."""
import re

from tests.test_built_kernels import _tool, code_objects, needs_llvm  # noqa: F401  (code_objects is a fixture)


def _resources(code_object):
    for entry in _tool("llvm-readelf", "--notes", code_object).split("- .agpr_count:")[1:]:
        name = re.search(r"\.name:\s+(\S+)", entry)[1]
        yield (name, int(re.search(r"\.vgpr_count:\s+(\d+)", entry)[1]),
               int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", entry)[1]),
               int(re.search(r"\.group_segment_fixed_size:\s+(\d+)", entry)[1]))


@needs_llvm
def test_no_spills_and_four_waves(code_objects):  # noqa: F811
    seen = {}
    for obj in code_objects:
        for name, registers, scratch, lds in _resources(obj):
            kernel = re.search(r"(k_(?:narrow|group|rows|stream|row_grad|finish_logp|finish_policy|seq_sums|seq_totals|weights|pairs|"
                               r"pref_middle|policy_stats|clip_\w+?))(?:I|E)", name)
            if kernel is None:
                continue
            seen[kernel[1]] = seen.get(kernel[1], 0) + 1
            assert scratch == 0 and lds <= 64 << 10, (name, scratch, lds)
            assert registers <= 128, (name, registers)   # 512 of a SIMD: four waves
    assert {"k_narrow", "k_group", "k_rows", "k_stream", "k_row_grad", "k_clip_sums", "k_clip_scale"} <= set(seen), seen
    # types x widths (x passes): every variant that a call can reach, and no more of them
    assert seen["k_rows"] == 3 * (3 + 3) and seen["k_stream"] == 3 * 2, seen


def _defined():
    """Kernels that the sources of the losses and of clipping define."""
    import os
    import paper_1906_08879_amd.build as build
    names = set()
    for source in ("kernels_losses.hip", "kernels_clip.hip"):
        with open(os.path.join(build.CSRC, source)) as f:
            names |= set(re.findall(r"__global__[^;{]*?\bvoid\s+(k_\w+)\(", f.read()))
    return names


@needs_llvm
def test_every_kernel_of_the_sources_is_built_without_spills(code_objects):  # noqa: F811
    defined, seen = _defined(), {}
    assert {"k_finish", "k_seq_sums", "k_pref_middle", "k_policy_stats", "k_clip_list", "k_clip_norm", "k_clip_small"} <= defined
    for obj in code_objects:
        for name, registers, scratch, lds in _resources(obj):
            kernel = re.search(r"\d(k_[a-z_]+?)(?:I|E)", name)
            if kernel is None or kernel[1] not in defined:
                continue
            seen[kernel[1]] = seen.get(kernel[1], 0) + 1
            assert scratch == 0 and lds <= 64 << 10 and registers <= 128, (name, registers, scratch, lds)
    assert set(seen) == defined, defined ^ set(seen)
    # a thread to a row, or a wave, for log probabilities, the policy loss and the preference's first pass of three types
    assert seen["k_finish"] == 3 * 3 * 2, seen
