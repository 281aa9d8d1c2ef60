"""CPU checks of the index arithmetic that decides what the attention kernels read (the functions of
``csrc/ttf_places.h``, compiled for the host)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_07355_amd", "csrc")


def _values(tmp_path, body):
    """The integers that a program around `body` prints."""
    src, exe = tmp_path / "places.cpp", str(tmp_path / "places")
    src.write_text('#include <cstdio>\n#include "ttf_places.h"\nusing namespace ttf;\n'
                   "static void put(long long v) { std::printf(\"%lld\\n\", v); }\nint main() {\n" + body + "\n}\n")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", str(src), "-I", CSRC, "-o", exe], check=True)
    return [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]


@pytest.mark.parametrize("entry_bytes", [2, 4])
def test_key_pieces_stay_inside_the_head(tmp_path, entry_bytes):
    """Every 16 bytes that a lane reads of a head lie in it, and where it has a piece of its own, that is the one."""
    got = iter(_values(tmp_path, f"for (int D = 8; D <= 256; D += 8) for (int s = 0; s < {4 * entry_bytes}; ++s) for (int g = 0; g < 4; ++g)\n"
                                 f"  put(first_piece(g, D, {entry_bytes}) + next_piece(s, g, D, {entry_bytes}));"))
    for D in range(8, 257, 8):
        size = D * entry_bytes
        for s in range(4 * entry_bytes):
            for g in range(4):
                at = next(got)
                assert 0 <= at <= size - 16, (D, s, g)
                if s * 64 + g * 16 < size:
                    assert at == s * 64 + g * 16


def test_pages_are_looked_up_before_the_end_alone(tmp_path):
    """Also where a window over entries near 2^31 begins at a page whose number, with a lane's, is past 31 bits."""
    most = 2 ** 31 - 1
    cases = [(first // size, size, stop) for size in (1, 2, 7, 64, 1 << 20) for first in (0, 96, 5000, most - 31, most)
             for stop in (0, 1, 100, 0x7ff00000)]
    got = iter(_values(tmp_path, "for (int lane = 0; lane < 64; ++lane) {\n"
                       + "\n".join(f"put(page_begins({page}, lane, {size}, {stop}));" for page, size, stop in cases) + "\n}"))
    for lane in range(64):
        for page, size, stop in cases:
            assert next(got) == ((page + lane) * size < stop), (page, lane, size, stop)
