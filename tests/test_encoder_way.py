"""Which launches the shapes of tests/test_gpu_encoder_sweeps.py lead to, without a GPU."""
import os
import shutil
import subprocess

import pytest

from test_gpu_encoder_sweeps import IN_TURN

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def way(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("way") / "check_encoder_way")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", exe, os.path.join(HERE, "check_encoder_way.cpp")], check=True)
    return lambda *sizes: subprocess.run([exe, *map(str, sizes)], capture_output=True, text=True, check=True).stdout.splitlines()


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_second_sweeps_are_reached(way):
    for n_seqs, hq, hkv, n_q, n_k, lens in IN_TURN:
        name, runs, delta_first = way(n_seqs, hq, hkv, n_seqs * n_q, n_seqs * n_k, n_q, n_k)
        assert (name, runs) == ("in turn", "1"), (n_seqs, hq, hkv, n_q, n_k)
        assert max(lens or [n_k]) > int(delta_first)
    assert any(0 < n <= int(delta_first) for _, _, _, _, _, lens in IN_TURN for n in lens or [])


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_ways(way):
    """A prompt's pass over a whole clip is one after the other; small batches and middling sizes are not."""
    assert way(1, 12, 12, 32760, 512, 32760, 512)[:2] == ["in turn", "1"]
    assert way(2, 4, 4, 154, 66, 77, 33)[0] == "small"
    assert way(1, 8, 8, 1000, 400, 1000, 400)[0] == "together"
    assert way(1, 8, 8, 0, 400, 1, 400)[0] == way(1, 8, 8, 1000, 0, 1000, 1)[0] == "in turn"
