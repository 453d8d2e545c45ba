"""Host tests whose calls would run on a GPU, on addresses that are none, are not run where there is one."""

import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_calls_on_made_up_addresses_stay_off_a_gpu():
    """All of tests/test_rotary_cpu.py as on a machine with a GPU, with a library that takes every call that gets as far as
    the device for a fault."""
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU")
    code = """
import sys, pytest, torch
from paper_2609_33887_gb300 import rotary
from paper_2609_33887_gb300.bdcommit import BD_ERR_CUDA, BD_ERR_DEVICE
torch.cuda.is_available = lambda: True
real, faults = rotary.load_library, []

class Library:
    def __getattr__(self, name):
        def call(*args):
            rc = getattr(real(), name)(*args)
            if rc in (BD_ERR_CUDA, BD_ERR_DEVICE):
                faults.append(name)
            return rc
        return call

rotary.load_library = lambda: Library()
rc = pytest.main(["-q", "-p", "no:cacheprovider", "tests/test_rotary_cpu.py"])
sys.exit(rc or (3 if faults else 0))
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-500:])
    assert " skipped" in r.stdout
