"""The serving loop of bench.py: prompts identified, their shared pages found, tokens appended and
answered; serve_path() checks the shared blocks and the last answers itself."""

import argparse
import json

import pytest
import torch

import bench
import paper_2607_23115_amd as g
from gpu_util import say

pytestmark = pytest.mark.gpu


def test_a_few_steps(capsys):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    say("bench serve_path")
    bench.serve_path(argparse.Namespace(steps=3, warmup=1), g, torch)
    line = json.loads(capsys.readouterr().out.splitlines()[-1])
    assert line["steps"] == 3 and line["value"] > 0 and line["config"]["worst_difference"] > 0
