"""What the kernels' sources must not do, as no run shows it reliably: order memory between CTAs with less than the
cluster's scope."""
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
