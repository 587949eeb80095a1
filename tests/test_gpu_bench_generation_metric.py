"""The generation bench names in its metric what its time includes."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("args,timed", [([], ""), (["--kv8"], ", timed with its 8-bit cache stores"),
                                        (["--kv8", "--states", "40"], ", timed with its 8-bit cache stores and attention to 40 encoder states")], ids=str)
def test_the_bench_names_what_it_times(args, timed):
    run = subprocess.run([sys.executable, "-m", "paper_2411_17178_amd.bench_generation", "--layers", "2", "--iters", "2", "--warmup", "1", "--batch", "2", *args],
                         capture_output=True, text=True, timeout=100, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert run.returncode == 0, run.stderr
    metric = json.loads(run.stdout.strip().splitlines()[-1])["metric"]
    assert metric == "windowed-attn effective TFLOP/s (retained pairs), all generation steps of a layer" + timed
