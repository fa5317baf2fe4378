"""The example decoder's command line: what it does not know is refused before anything runs."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_caches_are_held_in_4_or_16_bits():
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "decode_with_cache.py"), "--bits", "8"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 2 and "--bits" in out.stderr
