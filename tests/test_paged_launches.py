"""That the sizes of test_gpu_paged_launches.py select the launches they are there for (csrc/paged.h), checked without a GPU."""
import os
import shutil
import subprocess

import pytest

from paper_2509_22622_amd import binding as B

from test_gpu_paged_launches import APPENDS, ATTENDS

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def launch(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host C++ compiler")
    exe = tmp_path_factory.mktemp("launch") / "paged_append_launch"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", str(exe), os.path.join(HERE, "paged_append_launch.cpp")], check=True)
    return lambda *a: tuple(map(int, subprocess.run([str(exe), *map(str, a)], check=True, capture_output=True, text=True).stdout.split()))


@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_selects(launch, case):
    """Whole tiles, units enough a workgroup, and workgroups that go from one kv head to the next and from the last one to the queries."""
    _, d, hq, hkv, _, _, _, _, news, least = APPENDS[case]
    units, most, rows = hkv + (hq + 1) // 2, 4096 // d, sum(news) + 3
    tile_rows, each = launch(rows, units, most)
    assert tile_rows == most and each >= least and hq % 2 == 1
    runs = [range(at, min(at + each, units)) for at in range(0, units, each)]
    assert any(hkv - 1 in r and hkv in r for r in runs) and any(0 in r and 1 in r for r in runs) and hkv >= 2
    if case == 5:
        assert -(-rows // tile_rows) > 512


def test_append_selects_an_odd_head_behind_another(launch):
    """One case at least ends a workgroup's run of several units with a query head by itself."""
    ends = []
    for _, d, hq, hkv, _, _, _, _, news, _ in APPENDS:
        units = hkv + (hq + 1) // 2
        _, each = launch(sum(news) + 3, units, 4096 // d)
        ends.append((units - 1) % each)
    assert any(ends), ends


@pytest.mark.parametrize("case", range(len(ATTENDS)))
def test_attn_selects(case):
    fmt, d, hq, hkv, page, lens, news, sink, window, max_new, max_len, tiles, splits = ATTENDS[case]
    c = B.PagedCache(1, hq, hkv, d, page, 10, kv_format=fmt, device=None)
    assert tiles == -(-hq // hkv * max_new // 16) and (news is None or len(news) == len(lens))
    assert c.attn_workspace_bytes(len(lens), max_new, max_len, sink, window) == len(lens) * hkv * tiles * splits * 16 * (d + 2) * 4


def test_attn_selects_every_branch():
    units = [(len(c[5]) * c[3] * c[11], c[12]) for c in ATTENDS]
    for low, high, splits in ((86, 256, 5), (257, 384, 5), (385, 512, 5), (513, 2048, 3)):
        assert sum(low <= n <= high and s == splits for n, s in units) >= 2, (low, high)
    assert any(s > 16 for _, s in units)                              # the join with a workgroup a row
