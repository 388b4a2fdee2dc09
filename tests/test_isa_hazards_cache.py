"""The checks of test_isa_hazards.py and test_isa_hazards_direct.py for the kernels outside the attention call that copy tiles to LDS in inline assembly, and a
count of all sources and kernels that do, so that a new one does not go unchecked."""
import os
import re

import pytest

import test_isa_hazards as hazards
import test_isa_hazards_direct as direct

# kernel templates: instantiations that copy (the tree's over 8-bit caches widen what they load instead), and of all
COPYING = {
    "fm_weights.hip": {"weights_kernel": (2, 2)},       # head dimensions
    "fm_tree.hip": {"tree_kernel": (4, 8)},             # x types of rows x 8-bit caches
}


@pytest.fixture(scope="module", params=sorted(COPYING))
def source_and_assembly(request, tmp_path_factory):
    return request.param, hazards._assembly(str(tmp_path_factory.mktemp("isa")), request.param)


def _functions(asm):
    return list(re.finditer(r"^(\w+):.*?^\.Lfunc_end\d+:", asm, re.S | re.M))


def test_every_source_that_copies_tiles_is_named():
    import importlib
    build = importlib.import_module("paper_2410_01359_amd.build")
    copying = [s for s in build.SOURCES if re.search(r"\b(tile_load_async\w*|async_copy\w+)\b", open(os.path.join(build.CSRC, s)).read())]
    assert sorted(copying) == sorted([*COPYING, *direct.DIRECT])


def test_every_kernel_that_copies_tiles_is_named(source_and_assembly):
    source, asm = source_and_assembly
    copying = [m.group(1) for m in _functions(asm) if "global_load_lds" in m.group(0)]
    assert len(copying) == sum(n for n, _ in COPYING[source].values()), copying
    for kernel, (some, every) in COPYING[source].items():
        kernels = hazards._kernels(asm, [kernel])
        assert len(kernels) == every and sum(m.group(1) in copying for m in kernels) == some


def test_lds_window_register_is_written_only_by_the_copy_helpers(source_and_assembly):
    source, asm = source_and_assembly
    copying = "\n".join(m.group(0) for m in _functions(asm) if "global_load_lds" in m.group(0))
    for kernel, (some, _) in COPYING[source].items():
        hazards.check_lds_window_register(copying, [kernel], some)


def test_no_copy_reads_its_base_too_early(source_and_assembly):
    for m in _functions(source_and_assembly[1]):
        if "global_load_lds" in m.group(0):
            bad = direct._copies_too_early(m.group(0).split("\n")[1:])
            assert not bad, f"{m.group(1)}: {sorted(bad)[:3]}"
