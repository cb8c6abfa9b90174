"""The calls of tests/span_cases.py reach every row-block shape: what the plans give them,
on the CPU (tests/host/span_rows.cpp)."""

import os
import shutil
import subprocess

import pytest

import span_cases as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_02544_amd", "csrc")
FORM = {"bf16": 0, "fp4": 1, "f32": 2}


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_every_shape_is_reached(tmp_path):
    exe = str(tmp_path / "span_rows")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC] +
                       [os.path.join(CSRC, f) for f in ("simsd_plan.cpp", "simsd_ops_plan.cpp", "simsd_span_plan.cpp")] +
                       [os.path.join(ROOT, "tests", "host", "span_rows.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    lines, keys = [], []
    most_q, most_kv = max(n for n, _ in S.LENS), max(kv for _, kv in S.LENS)
    for form in FORM:
        for d in (64, 128):
            for hq, hkv in S.HEADS:
                for window, sinks, m in S.windows(form):
                    for t in S.TOKENS:
                        lines.append(f"c {FORM[form]} {t} {len(S.LENS)} {hq} {hkv} {d} {most_q} {most_kv} {m} {window} {sinks}")
                        keys.append(("chunk", form, d, hq))
            for B, L, hq, hkv in S.STEPS if form != "f32" else ():
                for window, sinks, _ in S.windows(form):
                    for n in S.COPIES:
                        lines.append(f"v {FORM[form]} {n * len(S.PREFIXES)} {hq} {hkv} {d} {B} {L} {max(S.PREFIXES)} {window} {sinks}")
                        keys.append(("verify", form, d, hq))
    r = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True)
    found = {}
    for key, rows in zip(keys, r.stdout.split()):
        found.setdefault(key, set()).add(int(rows))
    for (kind, form, d, hq), rows in found.items():
        print(kind, form, d, hq, sorted(rows))
        assert rows <= S.SHAPES[form]
    for kind, form in {k[:2] for k in found}:
        for d in (64, 128):
            assert set.union(*[r for k, r in found.items() if k[:3] == (kind, form, d)]) == S.SHAPES[form], (kind, form, d)
