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


@pytest.mark.parametrize("sequences,new,most,length,heads,plan", [
    # one prompt beside decoding over long texts: the texts are the kernel's for few rows, in tiles of one token's rows
    (32, 2031, 2000, 32768, (64, 8), (8, 33)), (2, 2001, 2000, 32768, (64, 8), (8, 33)), (32, 2031, 2000, 4096, (64, 8), (8, 33)),
    (256, 767, 512, 2048, (64, 8), (8, 33)), (256, 767, 512, 1024, (32, 32), (1, 33)),
    # prompts only, of different lengths: one launch
    (4, 3952, 1336, 1344, (64, 8), (32, 1)), (4, 3952, 1336, 1344, (32, 32), (32, 1)), (8, 2350, 700, 704, (64, 8), (32, 1)),
    # none can be short, whatever the lengths
    (1, 1000, 1000, 1 << 20, (64, 8), (32, 1)), (2, 1020, 1000, 1 << 20, (64, 8), (32, 1)),
    # the same with max_new far above what the rows leave for one sequence
    (32, 2031, 1 << 20, 32768, (64, 8), (8, 33)), (4, 3952, 1 << 20, 1344, (64, 8), (32, 1)),
    # few rows only: tiles for an ordinary sequence
    (100, 103, 4, 4096, (64, 8), (16, 0)), (100, 100, 4, 4096, (64, 8), (8, 0)), (16, 64, 4, 6016, (64, 8), (32, 0)),
    (100, 100, 16, 4096, (8, 8), (1, 0))])
def test_unequal_batches(eqat, sequences, new, most, length, heads, plan):
    d = eqat.make_cache_desc(128, 128, heads[1], 16, 1 << 18, sequences, length // 16, new)
    assert eqat.eqat_cache_attention_plan(d, eqat.make_attention_desc(heads[0], most, 0.1), 148) == plan


@pytest.mark.parametrize("tokens,plan", [(1 << 20, (32, 1)), (1 << 25, (32, 1)), ((1 << 25) + 1024, (32, 0)), (1 << 30, (32, 0))])
def test_sequences_that_outlast_the_waits_are_not_for_the_kernel_for_prompts(eqat, tokens, plan):
    """There a wait may last for a whole item: 2^30 tokens would take 20 s, a wait gives up after 2.  In the kernel for few rows every wait
    is for a tile."""
    d = eqat.make_cache_desc(128, 128, 8, 1024, 1024, 1, tokens // 1024, 1000)
    assert eqat.eqat_cache_attention_plan(d, eqat.make_attention_desc(64, 1000, 0.1), 148) == plan


def test_heads_of_256_are_not_for_the_kernel_for_prompts(eqat):
    d = eqat.make_cache_desc(128, 256, 8, 16, 1024, 1, 1024, 1000)
    assert eqat.eqat_cache_attention_plan(d, eqat.make_attention_desc(64, 1000, 0.1), 148) == (8, 0)
