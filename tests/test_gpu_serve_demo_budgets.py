"""Budgets of the serving demo that are smaller than what it keeps of the last slots by default."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("budget", [1, 8, 15, 16])
def test_small_budgets(budget):
    from paper_2410_17765_b200 import serve_demo as S

    out, gained = S.generate(steps=12, batch=3, budget=budget, every=3, temperature=0.0)
    assert len(out) == 3 and all(len(s) >= 13 for s in out) and 1.0 <= gained <= S.Config().n


def test_a_small_budget_from_the_command_line():
    r = subprocess.run([sys.executable, "-m", "paper_2410_17765_b200.serve_demo", "--steps", "9", "--batch", "2", "--budget", "8"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "9 rounds of 2 sequences" in r.stdout, r.stderr[-500:]
