"""What the kernels' sources must not do, as no run shows it reliably: order memory between CTAs with less than the
cluster's scope, or read through the read-only path what a launch before them may still be writing."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_06309_gb300", "csrc")


def _code():
    """-> {file: its text without comments}"""
    out = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if path.endswith((".cu", ".cuh", ".h")):
            with open(path) as f:
                out[os.path.basename(path)] = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    assert len(out) > 10
    return out


def test_arrivals_on_other_ctas_release_to_the_cluster():
    """An arrival on an address that may be another CTA's (shared::cluster) is seen by threads of that CTA: it
    releases to the cluster, or is a relaxed one of that scope right behind a fence that does."""
    found = 0
    for name, text in _code().items():
        for m in re.finditer(r"(fence\.release[.\w:]*;[\s\\nt\"]*)?(mbarrier\.arrive[.\w:]*)", text):
            if "shared::cluster" in m.group(2):
                found += 1
                fenced = m.group(1) and re.match(r"fence\.release\.[\w:.]*\.cluster;", m.group(1))
                assert ".release.cluster." in m.group(2) or (fenced and ".relaxed.cluster." in m.group(2)), (name, m.group())
        # the other forms take addresses of the CTA's own
        assert not re.search(r"\bmbar_arrive(_expect_tx)?\(\s*map_to_rank", text), name
    assert found


def test_remote_arrivals_take_mapped_addresses():
    """mbar_arrive_remote is the only arrival whose address comes from map_to_rank."""
    for name, text in _code().items():
        mapped = set(re.findall(r"(\w+) = map_to_rank\(", text))
        for call in re.findall(r"\bmbar_arrive(?:_expect_tx)?\((\w+)", text):
            assert call not in mapped, (name, call)


def test_no_read_only_loads_of_what_a_launch_before_may_write():
    """Grids of rf_linear_i8 are resident before the launch that makes their digits and scales has ended: no loads
    that take memory for read-only while the kernel lives."""
    text = _code()["rf_linear_i8.cu"]
    assert "cudaGridDependencySynchronize" in text
    for name in ("rf_linear_i8.cu", "rf_quant.cu", "rf_norm.cu", "rf_epilogue.cuh", "rf_vec.cuh", "rf_stage.cuh"):
        assert not re.search(r"ld\.global[.\w:]*\.nc|__ldg\(", _code()[name]), name
