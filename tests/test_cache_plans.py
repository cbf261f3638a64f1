"""How a call of the attention over the cache is divided, as far as the host decides it."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def test_a_plan_without_a_device_is_that_of_148_sms(eqat):
    """The question must not end the process."""
    code = ("from paper_2407_11062_b200 import binding as e\n"
            "d = e.make_cache_desc(128, 128, 8, 16, 4096, 1, 2048, 1000)\n"
            "for rows in (1, 1000):\n"
            "    a = e.make_attention_desc(64, rows, 0.1)\n"
            "    print(e.eqat_cache_attention_plan(d, a) == e.eqat_cache_attention_plan(d, a, 148))\n")
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""}, capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout.split() == ["True", "True"], (done.returncode, done.stdout, done.stderr[-500:])
