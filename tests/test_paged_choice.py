"""How nm_paged_attention shares its work among workgroups (csrc/nm_paged_choice.h), in a C++ driver of its own (CPU)."""
import shutil
import subprocess

import pytest

from test_gpu_decode_packs import PACK_CASES
from test_sanitizers import SAN, _run

BUILD = ["g++", "-std=c++17", *SAN, "-Wall", "-Werror", "-I", "paper_2305_14405_amd/csrc", "tests/sanitize/paged_driver.cpp", "-o"]


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_rows_cover_every_head_once(tmp_path):
    """Whatever heads, sizes, lengths and layouts: each query head of a request is in one row, with the key head of its group."""
    exe = str(tmp_path / "paged_driver")
    _run([*BUILD, exe], exe)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_cases_are_packed_as_they_say(tmp_path):
    """The cases that compare packed heads with binary64 are packed, by the numbers that stand there, and the others are not."""
    exe = str(tmp_path / "paged_driver")
    _run([*BUILD, exe], exe)
    assert all(B * hk * -(-min(window or columns * 32, columns * 32) // 128) >= 32 * 768 for B, _, hk, _, window, columns, _ in PACK_CASES)   # enough rows for it
    shapes = [(B, hq, hk, d, min(window or columns * 32, columns * 32)) for B, hq, hk, d, window, columns, _ in PACK_CASES]
    out = subprocess.run([exe, *(str(v) for s in shapes for v in s)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and [int(v) for v in out.stdout.split()] == [c[6] for c in PACK_CASES], out.stdout + out.stderr
