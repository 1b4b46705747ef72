"""What the package and its build need of a machine (no GPU needed)."""

import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


def test_all_names_without_torch():
    python("import sys; sys.modules['torch'] = None\n"
           "from paper_2607_01408_amd import *\n"
           "Plan, paths_host\n")


def test_the_operators_are_listed_and_found():
    python("import paper_2607_01408_amd as sg\n"
           "assert {'rms_norm', 'gated', 'Block8', 'Plan'} <= set(dir(sg))\n"
           "assert callable(sg.rms_norm)\n")
