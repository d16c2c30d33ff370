"""The hash that ties a committed profile to its kernel's sources: what the kernel is compiled from changes it,
what other calls declare does not."""
import importlib.util
import os
import shutil

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def bench(tmp_path):
    spec = importlib.util.spec_from_file_location("bench_copy", os.path.join(ROOT, "bench.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    shutil.copytree(os.path.join(ROOT, "paper_2309_01885_amd", "csrc"), tmp_path / "paper_2309_01885_amd" / "csrc")
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    mod.ROOT = str(tmp_path)
    return mod


def change(path, old, new):
    text = path.read_text()
    assert old in text
    path.write_text(text.replace(old, new, 1))


@pytest.mark.parametrize("kernel", ["gram_x3w_kernel", "cd_step_kernel"])
def test_hash_follows_what_the_kernel_uses(bench, tmp_path, kernel):
    want = bench.kernel_source_hash(kernel)
    header = tmp_path / "include" / "qe.h"
    change(header, "#ifdef __cplusplus\n}", "#define QE_SOMETHING_NEW 7\nqe_status qe_new(int n);\n#ifdef __cplusplus\n}")
    change(header, "/* some grid scale <= 0 or not finite */", "/* some\n grid scale */")
    assert bench.kernel_source_hash(kernel) == want
    change(header, "QE_ERR_DIAG        2", "QE_ERR_DIAG        12")
    changed = bench.kernel_source_hash(kernel)
    # (a status that the kernel's sources name, or do not)
    text = "".join((tmp_path / "paper_2309_01885_amd" / "csrc" / f).read_text() for f in bench.KERNEL_SOURCES[kernel])
    assert (changed != want) == ("QE_ERR_DIAG" in text)
    for name in bench.KERNEL_SOURCES[kernel]:
        before = bench.kernel_source_hash(kernel)
        path = tmp_path / "paper_2309_01885_amd" / "csrc" / name
        path.write_text(path.read_text() + "\n// more\n")
        assert bench.kernel_source_hash(kernel) != before


def test_committed_profiles_match(bench):
    """The profiles that the benchmark reads belong to this tree's kernels."""
    bench.ROOT = ROOT
    assert set(bench.measured_traffic()) == set(bench.KERNEL_SOURCES)
    assert bench.profiled_panel_launch() is not None
