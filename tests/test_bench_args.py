"""bench.py refuses arguments that the run it would make does not heed.  No GPU needed: they are looked at first."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("args", ["--codes e4m3", "--codes int8 --paged", "--codes int8 --trajectory", "--codes e4m3 --score-block 16 --chunk 4",
                                  "--codes e4m3 --predictor --draft 4", "--chunk 4 --draft 4"])
def test_refused(args):
    # (--gpus 2: should they be taken after all, the run ends there)
    r = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--gpus", "2"] + args.split(), capture_output=True, text=True, timeout=300)
    assert r.returncode == 2 and "error: --" in r.stderr and not r.stdout


def test_taken():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--gpus", "2", "--chunk", "4", "--codes", "e4m3"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 1 and "one MI355X" in r.stderr
