"""The library and torch share one HIP runtime in whichever order a program loads them: with two, every
launch on torch's tensors and streams fails."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COUNT = "print(len({l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64.so' in l}))"


def runtimes(first, second):
    out = subprocess.run([sys.executable, "-c", f"{first}\n{second}\n{COUNT}"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    return int(out.stdout)


def test_one_runtime():
    load, torch = "import paper_2207_08867_amd as m; m.lib()", "import torch"
    assert runtimes(torch, load) == 1
    assert runtimes(load, torch) == 1
