"""The layers of tests/mxfp4_cases.py take every tile of the tiled products, with every number of units of K that its loop tells apart."""
import os
import subprocess

import numpy as np

from paper_2503_00245_amd import build as hip_build
from tests.mxfp4_cases import PATTERNS, TILED, picks

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_tiled_layers_reach_every_tile(tmp_path):
    exe = str(tmp_path / "check")
    subprocess.run([hip_build._hipcc(), "-x", "hip", "--offload-host-only", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I",
                    hip_build.CSRC, os.path.join(ROOT, "tests", "mxfp4_plan_check.cpp"), "-o", exe], check=True)
    seen = {(p, rows): set() for p in ("gate/up", "down") for rows in (64, 128, 256)}  # numbers of units of K, and "halves"
    for T, d, F, E, k, skew, hidden, down in TILED:
        loads = np.bincount(picks(E, k, skew)[0][np.arange(T) % PATTERNS].ravel(), minlength=E)
        assert loads.min() > 0
        r = subprocess.run([exe, str(T * k), str(E), str(d), str(F), *map(str, loads)], capture_output=True, text=True, check=True, timeout=60)
        got = list(map(int, r.stdout.split()))
        assert got[:2] == [hidden, down], (T, d, F, E, k, got)
        for p, rows, K, halves in (("gate/up", hidden, d, got[2]), ("down", down, F, got[3])):
            if rows > 32:
                seen[p, rows].add((K + 255) // 256)
                if halves:
                    seen[p, rows].add("halves")
    for (p, rows), units in seen.items():
        stages = 2 if rows == 256 else 3
        assert {stages, stages + 1} <= units, (p, rows, units)
        assert max(u for u in units if u != "halves") >= 2 * stages + 1, (p, rows, units)
        if (p, rows) != ("gate/up", 64):  # (gate/up in tiles of 64 rows: with one unit the rule has other tiles)
            assert 1 in units, (p, rows, units)
        if (p, rows) != ("down", 64):  # (down in tiles of 64 rows: never more than a round)
            assert "halves" in units, (p, rows, units)
