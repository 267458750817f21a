"""How attention of few rows over a cache held in 4 bits divides its work, walked on the host with the kernel's own functions
(CPU): every item that a workgroup works on has rows, every query it reads is a packed row of the call, every unit of work
is done exactly once, the join looks for the parts where they are, and the workspace that is asked for holds them."""
import os
import random
import subprocess

import pytest

from test_attention_division import MIXED, call

HERE = os.path.dirname(os.path.abspath(__file__))
NAMES = ("many", "tile_rows", "wgs", "aligned", "worked", "empty", "read", "wrong", "lost", "past")


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("division4") / "attention4_plan_ref")
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", exe, os.path.join(HERE, "attention4_plan_ref.cpp")], check=True)

    def run(calls):
        text = "\n".join(" ".join(str(x) for x in c) for c in calls) + "\n"
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        rows = [dict(zip(NAMES, (int(x) for x in line.split()))) for line in out.strip().splitlines()]
        assert len(rows) == len(calls)
        for c, r in zip(calls, rows):
            assert r["past"] == 0, (c[:11], r)
            if not r["many"]:
                assert r["empty"] == 0 and r["read"] < c[5] and r["wrong"] == 0 and r["lost"] == 0, (c[:11], r)
        return rows

    return run


def test_prompts_among_single_tokens(walk):
    walk(MIXED)


def test_stretches_that_end_with_sequences(walk):
    calls = [call([(1, kv - 40 * b) for b in range(B)], 32, 8, 128, bf16=bf16)
             for B in (1, 2, 4, 8, 16, 31, 33, 63, 64, 65, 256, 257, 300) for kv in (16000, 30000, 13000, 12200) for bf16 in (False, True)
             if kv > 40 * B]
    rows = walk(calls)
    assert any(r["aligned"] for r in rows) and any(not r["aligned"] and not r["many"] for r in rows)
    short = walk([call([(1, kv)] * B, 32, 8, 128, bf16=True) for B in (4, 16, 64) for kv in (100, 500, 1000)])
    assert all(r["aligned"] for r in short if not r["many"])


def test_starts_out_of_bounds(walk):
    for start, kv in (([0, 4, 1 << 30, (1 << 31) - 1], [100, 150, 120]), ([0, 1 << 30, 1 << 30, 6], [90, 80, 70]),
                      ([5, 5, 6, 2], [40, 900, 30]), ([-7, 3, 3, 6], [10, 2000, 600])):
        for bf16 in (0, 1):
            walk([[bf16, 32, 8, 128, 16, 6, 4, 1 << 22, 0, 0, 3] + start + kv])
    walk([[bf16, 32, 8, 128, 16, 6, 4, 1 << 22, 0, 0, 3, 0, 1 << 30, 4, 6, kv, 700, 3000]
          for bf16 in (0, 1) for kv in range(100, 9000, 100)])


@pytest.mark.parametrize("seed", range(8))
def test_random_calls(walk, seed):
    rng = random.Random(seed)
    calls = []
    for _ in range(80):
        H, G = rng.choice([(32, 8), (16, 16), (8, 1), (28, 4), (12, 4), (64, 8), (1024, 1024)])
        lens = []
        for _ in range(rng.choice([1, 2, 5, 17, 40, 70, 300, 600])):
            n = rng.choice([0, 1, 1, 1, 2, 5, rng.randint(1, 40), rng.randint(1, 900) if rng.random() < 0.1 else 1])
            lens.append((n, rng.choice([0, 1, n, n + rng.randint(0, 300), n + rng.randint(0, 5000), n + rng.randint(0, 60000)])))
        window = rng.choice([0, 0, rng.randint(1, 2000)])
        calls.append(call(lens, H, G, rng.choice([8, 64, 80, 128, 192, 256]), bf16=rng.random() < 0.6, window=window,
                          masked=window == 0 and rng.random() < 0.3, max_new=rng.choice([None, None, 1024, 7]),
                          max_kv=rng.choice([None, 1 << 22, 1 << 17])))
    rows = walk(calls)
    assert sum(not r["many"] for r in rows) >= 20
