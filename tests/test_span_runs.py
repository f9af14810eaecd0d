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


def decodes(n, nkv, runs, d=128):
    """Decodes of a few own tokens below runs; the heads, requests and runs of a planner's batch."""
    return (nkv, nkv, d), tables([(1, 1, 3 + i) for i in range(n)], runs, itertools.count()), runs


@pytest.mark.parametrize("d,nkv,pages", [(128, 8, 64), (64, 8, 128), (128, 1, 512)])
def test_runs_are_joined_from_64_mib_on(planner, d, nkv, pages):
    """17 requests, for 16 of which a run of `pages` pages is not read again: 64 MiB."""
    assert 16 * pages * nkv * 16 * 2 * 2 * d == 64 << 20
    batches = [decodes(n, nkv, [(0, n, pages - k)], d) for n, k in ((17, 0), (17, 1), (16, 0), (18, 1))]
    got = planner([b + (-1,) for b in batches])
    assert [g[0] for g in got] == [1, 0, 0, 1]


def test_runs_are_joined_all_or_none(planner):
    """What counts is what all runs of a call save together: then the shortest of them is joined too."""
    half = [(0, 17, 32), (17, 16, 33)]
    alone, both, more = planner([decodes(33, 8, half[:1]) + (-1,), decodes(33, 8, half) + (-1,),
                                 decodes(36, 8, half + [(33, 3, 1)]) + (-1,)])
    assert 16 * 32 + 15 * 33 < 1024 <= 16 * 32 + 15 * 33 + 2 * 9
    assert alone[0] == both[0] == 0
    assert more[0] == 0
    assert planner([decodes(36, 8, half + [(33, 3, 9)]) + (-1,)])[0][0] == 3
    assert planner([decodes(36, 8, [(0, 17, 64), (17, 2, 1)]) + (-1,)])[0][0] == 2


def test_prompts_that_fill_their_tiles_read_runs_by_themselves(planner):
    """Long prompts take no part in a run; the rest of its requests does."""
    reqs, runs = [(1, 1, 5)] * 20 + [(0, 1024, 3), (0, 9, 0)], [(0, 22, 64)]
    got, = planner([((8, 8, 128), tables(reqs, runs, itertools.count()), runs, -1)])
    assert got[:2] == [1, 29]


def size_of(plan, d):
    """The workspace of a plan's arrays: the metadata, each array from a multiple of 16 bytes on,
    then the partial rows' outputs in fp32 and their maxima and sums, from multiples of 256."""
    items, pages, listed, merged, sources, partials = plan[2:]
    up = lambda n, k: -(-n // k) * k  # noqa: E731
    n = 0
    for count, size in ((items, 64), (pages, 4), (listed, 4), (merged, 16), (sources, 16)):
        n = up(n + count * size, 16)
    n = up(n, 256)
    for size in (4 * d, 8):
        n = up(n + partials * size, 256)
    return max(n, 256)


@pytest.mark.parametrize("seed", range(6))
def test_workspace_bound_covers_every_plan(planner, seed):
    """Random batches, below runs of any length, are taken apart whatever that saves: the bound for
    batches of their size covers what their plans need.  As the library takes them apart, this is
    the size that it names."""
    rng = np.random.default_rng(400 + seed)
    batches, bounds, sizes, joined = [], [], [], 0
    for _ in range(40):
        nkv = int(rng.choice([1, 2, 8, 19]))
        heads = nkv * int(rng.choice([1, 4, 16, 17, 40])), nkv, int(rng.choice([64, 128]))
        R = int(rng.integers(1, 14))
        dec = rng.random(R) < rng.choice([0.2, 0.7, 1.0])
        new = np.where(dec, 1, rng.integers(1, rng.choice([6, 40, 400]), R))
        own = rng.integers(1, rng.choice([20, 300, 20000]), R)
        runs, depth, start = [], np.zeros(R, int), np.zeros(R, int)
        for _ in range(int(rng.integers(0, 6))):
            a = int(rng.integers(0, R))
            n = int(rng.integers(1, R - a + 1))
            if (start[a:a + n] == start[a]).all():
                k = int(rng.choice([1, 2, 30, 400]))
                runs.append((a, n, k))
                start[a:a + n] += k
                depth[a:a + n] += 1
        reqs = tables([(d, int(n), int(c)) for d, n, c in zip(dec, new, own)], runs, itertools.count())
        s = mx.attn_shape(*heads, 1 << 30)
        b = mx.Batch(dec.astype(int), new, [c for _, c, _ in reqs], [t for _, _, t in reqs])
        bounds.append(mx.mx_workspace_bytes_shared(s, b.T, b.R, sum(len(t) for _, _, t in reqs), int(depth.max())))
        sizes.append(mx.mx_workspace_bytes_shared_for(b, s, mx.SharedRuns(runs)))
        batches.append((heads, reqs, runs))
    for plan, b, n, bound in zip(planner([x + (-1,) for x in batches]), batches, sizes, bounds):
        assert size_of(plan, b[0][2]) == n <= bound
    for plan, b, bound in zip(planner([x + (0,) for x in batches]), batches, bounds):
        assert size_of(plan, b[0][2]) <= bound, b[0]
        joined += plan[0] > 0
    assert joined > 10
