"""The kernels of beams, pages and shared prefixes as they are built: all of them keep to registers."""
import re

from test_kernel_resources import code_objects, readelf  # noqa: F401

NAMES = ("attn_columns_kernel", "attn_prefix_kernel", "shared_plan_kernel", "beams_piece_kernel", "beams_group_kernel", "pages_survey_kernel",
         "pages_fork_kernel", "pages_copy_kernel", "compact_count_kernel", "compact_survey_kernel", "compact_list_kernel", "compact_move_kernel",
         "compact_tables_kernel")


def test_nothing_is_spilled(code_objects):  # noqa: F811
    found = {}
    for path in code_objects:
        for kernel in readelf("--notes", path).split("  - .agpr_count:")[1:]:
            field = dict(re.findall(r"^    \.(\w+): +(\S+)$", kernel, re.M))
            for name in NAMES:
                if name in field["name"]:
                    found.setdefault(name, []).append((int(field["vgpr_spill_count"]), int(field["private_segment_fixed_size"])))
    assert sorted(found) == sorted(NAMES)
    assert len(found["attn_columns_kernel"]) == 12 and len(found["attn_prefix_kernel"]) == 8
    assert all(use == (0, 0) for uses in found.values() for use in uses), found
