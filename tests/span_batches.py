"""Batches of attention over shared runs that the planner does take apart into runs and own
keys: test_span_runs.py checks that it does, test_gpu_span_runs.py runs them.

A case is ((q heads, KV heads, head dim), requests of (decode, n_new, own cached tokens),
runs of (first request, requests, pages)); `JOINED` says how many runs are read for several
requests at once and how many tokens take part in them, each run's counted."""
D, P = 1, 0

CASES = {
    # out may be q: decodes and short prompts below a run, a prompt beside them that reads it by itself
    "in place": ((8, 2, 64), [(D, 1, 20), (P, 9, 0), (P, 400, 7), (P, 3, 5)] + [(D, 1, 3)] * 40, [(0, 44, 208)]),
    # a tree: rows with three parts
    "tree": ((8, 2, 128), [(D, 1, 7 * i) for i in range(24)] + [(P, 5, 33)],
             [(0, 25, 180), (0, 9, 40), (9, 8, 3), (18, 7, 12)]),
    "paged": ((8, 2, 128), [(D, 1, 200), (P, 9, 64), (D, 1, 4), (P, 200, 0)] + [(D, 1, i) for i in range(40)],
              [(0, 44, 100)]),
    # 64 MiB exactly
    "far pages": ((8, 8, 128), [(D, 1, 30 * i) for i in range(16)] + [(P, 5, 12)], [(0, 17, 64)]),
    # a document of many splits
    "splits": ((16, 2, 64), [(D, 1, 5 * i) for i in range(12)], [(0, 12, 800)]),
}
JOINED = {"in place": (1, 53), "tree": (4, 29 + 9 + 8 + 11), "paged": (1, 51), "far pages": (1, 21), "splits": (1, 12)}


def tables(reqs, runs, ids):
    """(n_new, ctx_len, page table) of the requests, with page ids taken from `ids`."""
    t = [[] for _ in reqs]
    for first, n, k in runs:
        run = [next(ids) for _ in range(k)]
        for r in range(first, first + n):
            t[r] += run
    return [(n, 16 * len(x) + own, x + [next(ids) for _ in range(-(-(own + n) // 16))])
            for (_, n, own), x in zip(reqs, t)]
