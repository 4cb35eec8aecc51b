"""That the sizes of test_gpu_paged_launches.py select the launches they are there for (csrc/paged.h), checked without a GPU."""
import os
import shutil
import subprocess

import pytest

from test_gpu_paged_launches import APPENDS

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
