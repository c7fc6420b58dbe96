"""Where the attention's workgroups store, followed on the host (attention_jobs.hip): for thousands of calls every row of the parts lies in the workspace
that the call asked for and is stored once, and what is stored in parts is joined; and which of its request's keys a row sees."""

import os
import random
import subprocess

import pytest

from paper_1711_07240_amd import build as B

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def jobs(tmp_path_factory):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no compiler")
    program = tmp_path_factory.mktemp("jobs") / "attention_jobs"
    flags = [f for f in B.FLAGS if f not in ("-fno-gpu-rdc", "-O3")]
    subprocess.run([B.HIPCC, "-O1"] + flags + ["--cuda-host-only", "-x", "hip", os.path.join(HERE, "attention_jobs.hip"), "-o", str(program)], check=True,
                   capture_output=True)

    def ask(calls):
        lines = [" ".join(n if isinstance(n, str) else str(int(n)) for n in c) for c in calls]
        done = subprocess.run([str(program)], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True, timeout=300)
        return list(zip(lines, done.stdout.splitlines(), strict=True))

    return ask


def _call(elem, fresh, Hq, Hk, D, prefix, max_pages, page, pad=0, single=False):
    return [elem, sum(fresh) + pad, len(fresh), single, Hq, Hk, D, prefix, max_pages, page] + ([] if single else list(fresh))


# one request of 600 tokens; 544 requests of one; heads without sharing
ALONE = [([600], 32, 8, 128, 4096), ([1] * 544, 32, 8, 128, 4096), ([1] * 700, 32, 32, 128, 1000), ([1] * 640, 8, 8, 64, 1000), ([300], 64, 64, 32, 600),
         ([1] * 3, 8, 2, 64, 70000), ([40, 2], 8, 8, 80, 513)]


def test_a_prefix_alone(jobs):
    """max_pages = 0, with the prefix in one part, which is the result, and in several."""
    for line, answer in jobs([_call(elem, fresh, Hq, Hk, D, prefix, 0, 16, single=single) for elem in (2, 4) for fresh, Hq, Hk, D, prefix in ALONE
                              for single in ((False, True) if max(fresh) == 1 else (False,))]):
        assert answer == "ok", line


def test_calls_of_all_sizes(jobs):
    rng = random.Random(1)
    calls = []
    for _ in range(4000):
        Hk = rng.choice([1, 2, 3, 8, 20, 64])
        Hq = Hk * rng.choice([1, 1, 2, 4, 17])
        B_ = int(2 ** rng.uniform(0, 10.5))
        fresh = [1] * B_ if rng.random() < 0.5 else [rng.choice([0, 1, 3, rng.randrange(1, 200)]) for _ in range(B_)]
        while sum(fresh) * Hq > 60000:
            fresh = fresh[:-(-len(fresh) // 2)] if len(fresh) > 1 else [1]
        single = set(fresh) == {1} and rng.random() < 0.5
        page = 2 ** rng.randrange(0, 11)
        calls.append(_call(rng.choice([2, 4]), fresh, Hq, Hk, 8 * rng.randrange(1, 33), rng.choice([0, 1, 513, int(2 ** rng.uniform(0, 17))]),
                           rng.choice([0, 0, int(2 ** rng.uniform(0, 16)) // page + 1]), page, 0 if single else rng.choice([0, 0, 5]), single))
    # (more than 1024 heads are refused)
    wrong = [(line, answer) for call, (line, answer) in zip(calls, jobs(calls)) if answer != ("status 2" if call[4] > 1024 else "ok")]
    assert not wrong, (len(wrong), wrong[:3])


@pytest.mark.parametrize("g", [1, 3, 17])
def test_keys_that_rows_see(jobs, g):
    """The j-th of n new tokens its request's first tokens - n + j + 1, whether the table has room for all of them or not; of those the ones that it has room for."""
    sizes = [(1, 64, 4, 16), (2, 65, 4, 16), (4, 18, 1, 16), (100, 100, 4, 16), (36, 100, 4, 16), (5, 2, 4, 16), (3, 0, 4, 16), (3, -7, 4, 16), (9, 700, 0, 16),
             (2, (1 << 31) - 1, 65536, 1024), (40, 1000, 7, 1), (6, 6, 1, 1)]
    for (n, tokens, most, page), (line, answer) in zip(sizes, jobs([("sees", *size, g) for size in sizes])):
        tokens = max(tokens, 0) if most else 0
        want = [min(max(tokens - n + j + 1, 0), most * page) for j in range(n) for _ in range(g)]
        assert [int(x) for x in answer.split()] == want, line
