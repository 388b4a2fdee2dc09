"""No GPU: the traffic figures that bench.py reports go with the sources of the kernels that it times, whatever else the folder holds."""
import os
import shutil

import pytest

import bench


@pytest.fixture
def folder(tmp_path):
    return shutil.copytree(bench.CSRC, tmp_path / "csrc")


def test_other_sources_do_not_matter(folder):
    before = bench.kernels_digest(folder)
    (folder / "fm_another.hip").write_text('#include "fm_another.h"\n')
    (folder / "fm_another.h").write_text('#include "fm_common.h"\n')
    for name in os.listdir(folder):
        if name not in bench.timed_sources():
            (folder / name).write_text("// changed\n")
    assert bench.kernels_digest(folder) == before == bench.kernels_digest()


def test_every_source_of_a_timed_kernel_matters(folder):
    seen = {bench.kernels_digest(folder)}
    names = bench.timed_sources()
    assert {"fm_api.hip", "fm_fwd.hip", "fm_bwd.hip", "fm_preprocess.hip", "fm_common.h", "fm_interval.h"} <= set(names)
    for name in names:
        with open(folder / name, "a") as f:
            f.write("// changed\n")
        seen.add(bench.kernels_digest(folder))
    assert len(seen) == len(names) + 1


def test_a_header_that_comes_in_through_another(folder):
    before = bench.kernels_digest(folder)
    with open(folder / "fm_interval.h", "a") as f:
        f.write('#  include "fm_new.h"\n')
    (folder / "fm_new.h").write_text("// one\n")
    one = bench.kernels_digest(folder)
    (folder / "fm_new.h").write_text("// two\n")
    assert len({before, one, bench.kernels_digest(folder)}) == 3
