"""Host-side checks of how problems beyond one launch are split (no GPU)."""
import os
import shutil
import subprocess

import pytest


def test_tensors_of_more_chunks_than_a_launch_takes_go_in_pieces(tmp_path):
    """Every element once, in whole chunks, no launch over its 5 chunks of 2048 elements."""
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("needs g++")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "adamw_launches")
    subprocess.run([gxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include",
                    "-I", os.path.join(root, "include"),
                    "-I", os.path.join(root, "paper_2608_10805_amd", "csrc_block"), "-x", "c++",
                    os.path.join(root, "tests", "planner", "adamw_launches.cpp"), "-o", exe], check=True)
    sizes = [1, 2048 * 5, 2048 * 12 + 7, 0, 100, 2048 * 5 + 1, 2047, 2048 * 10, 3]
    out = subprocess.run([exe], input=" ".join(map(str, sizes)), capture_output=True, text=True, check=True).stdout
    got, chunks = {}, {}
    for line in out.splitlines():
        launch, first, param, grad, at, n = map(int, line.split())
        assert first == chunks.get(launch, 0)
        chunks[launch] = first + -(-n // 2048)
        tensor, start = divmod(at, 64000000)
        assert param - (1 << 40) == grad - (1 << 41) == 2 * at
        assert start == got.get(tensor, 0) and start % 2048 == 0
        got[tensor] = start + n
    assert max(chunks.values()) <= 5
    assert got == {i: n for i, n in enumerate(sizes) if n}
