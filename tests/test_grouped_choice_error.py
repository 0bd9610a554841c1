"""How far the times that grouped_choice.h reckons are from the measured ones, and what its choice costs: the figures that stand in
its comments, held against the table of measured times."""
import os
import re
import subprocess

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2601_21198_b200", "csrc")


def test_the_stated_errors(tmp_path):
    table = open(os.path.join(ROOT, "tests", "csrc", "grouped_choice_check.cpp")).read()
    rows = re.findall(r"\{(\d+), (\d+), (\d+), (\d+), (true|false), (true|false), (true|false), ([\d.]+), ([\d.]+)\}", table)
    assert len(rows) == 264
    exe = str(tmp_path / "grouped_choice_error")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, os.path.join(ROOT, "tests", "csrc", "grouped_choice_error.cpp"), "-o", exe])
    asked = "\n".join(" ".join(r[:4]) + " " + " ".join(str(int(b == "true")) for b in r[4:7]) for r in rows)
    reckoned = np.array([line.split() for line in subprocess.run([exe], input=asked, capture_output=True, text=True, check=True).stdout.splitlines()], float)
    measured = np.array([r[7:] for r in rows], float)
    share = reckoned[:, :2] / measured
    taken = np.where(reckoned[:, 2] > 0, measured[:, 1], measured[:, 0])
    cost = (taken / measured.min(axis=1)).max()
    said = re.search(r"few, ([\d.]+) to ([\d.]+) of the measured time; many, ([\d.]+) to ([\d.]+); .*?costs at most ([\d.]+) of the other's time",
                     re.sub(r"\s*//\s*", " ", open(os.path.join(CSRC, "grouped_choice.h")).read()))
    found = [share[:, 0].min(), share[:, 0].max(), share[:, 1].min(), share[:, 1].max(), cost]
    assert said, "few %.2f to %.2f; many %.2f to %.2f; cost %.2f; beyond a fifth: %d and %d" % (*found, *(np.abs(share - 1) > 0.2).sum(axis=0))
    assert np.allclose(np.array(said.groups(), float), found, atol=0.0051)
