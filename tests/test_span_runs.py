"""CPU checks of how attention over shared runs takes batches apart: when runs are read for
several requests at once, and that the workspace bound holds for every plan."""
import itertools
import os
import subprocess

import numpy as np
import pytest

import paper_2606_16264_amd as mx
from span_batches import CASES, JOINED, tables

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="session")
def planner(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "span_plan_print")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2606_16264_amd", "csrc"),
                    os.path.join(HERE, "span_plan_print.cpp"), "-o", exe], check=True)

    def ask(batches):
        """[runs, their tokens, items, page ids, listed, merged, sources, partials] of batches of
        (heads, requests of (n_new, ctx_len, table), runs, least bytes)."""
        text = []
        for heads, reqs, runs, least in batches:
            text.append(f"{heads[0]} {heads[1]} {heads[2]} {least} 0 0 {len(reqs)}")
            text += [f"{n} {ctx} {len(t)} " + " ".join(map(str, t)) for n, ctx, t in reqs]
            text.append(f"{len(runs)} " + " ".join(f"{a} {n} {k}" for a, n, k in runs))
        got = subprocess.run([exe], input="\n".join(text), capture_output=True, text=True, timeout=120, check=True)
        return [list(map(int, line.split())) for line in got.stdout.splitlines()]

    return ask


@pytest.mark.parametrize("name", CASES)
def test_gpu_batches_are_taken_apart(planner, name):
    """The batches that are to test runs on the GPU do have them read for several requests."""
    heads, reqs, runs = CASES[name]
    got, = planner([(heads, tables(reqs, runs, itertools.count()), runs, -1)])
    assert tuple(got[:2]) == JOINED[name]
