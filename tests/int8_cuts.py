"""How the library cuts products in 8-bit integers, from its own rule (csrc/int8_cut.hpp)
compiled for the host; no GPU work."""
from __future__ import annotations

import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_dir = _program = None


def _build():
    global _dir, _program
    if _program is None:
        _dir = tempfile.TemporaryDirectory()
        _program = os.path.join(_dir.name, "cuts")
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I",
                        os.path.join(ROOT, "paper_2504_03651_amd", "csrc"),
                        os.path.join(ROOT, "tests", "csrc", "int8_cuts.cpp"), "-o", _program], check=True)
    return _program


def cuts(sizes):
    """Of each (T, N, K, f32): (form, ranges, variant, bytes of parts, workspace for up to T)."""
    text = "".join("%d %d %d %d\n" % (t, n, k, bool(f)) for t, n, k, f in sizes)
    out = subprocess.run([_build()], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    return [(w[0], *map(int, w[1:])) for w in map(str.split, out)]
