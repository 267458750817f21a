"""How attention of few rows divides its work, walked on the host with the kernel's own functions (CPU):
every item that a workgroup works on has rows, every query it reads is a packed row of the call, and every
unit of work is done exactly once."""
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("division") / "attention_plan_ref")
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", exe, os.path.join(HERE, "attention_plan_ref.cpp")], check=True)

    def run(calls):
        text = "\n".join(" ".join(str(x) for x in call) for call in calls) + "\n"
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        names = ("many", "tile_rows", "tiles", "parts", "wgs", "worked", "empty", "read", "wrong")
        rows = [dict(zip(names, (int(x) for x in line.split()))) for line in out.strip().splitlines()]
        assert len(rows) == len(calls)
        return rows

    return run


def call(lens, H, G, D, bf16=False, page=16, window=0, masked=False, max_new=None, max_kv=None, rows=None):
    start = [0]
    for n, _ in lens:
        start.append(start[-1] + n)
    kv = [k for _, k in lens]
    return [int(bf16), H, G, D, page, rows or max(1, start[-1]), max_new or max(1, max(n for n, _ in lens)),
            max_kv or max(1, max(kv)), window, int(masked), len(lens)] + start + kv


def check(walk, calls):
    rows = walk(calls)
    for c, r in zip(calls, rows):
        if not r["many"]:
            assert r["empty"] == 0 and r["read"] < c[5] and r["wrong"] == 0, (c[:11], r)
    return rows


MIXED = [
    # a prompt among single tokens, float32
    call([(2048, 2048), (1, 512), (1, 400)], 32, 8, 128),
    call([(600, 600)] + [(1, 300 + b) for b in range(8)], 32, 8, 128),
    call([(512, 2048)] + [(1, 2048)] * 63, 32, 8, 128),
    call([(1, 2048)] * 20 + [(512, 2048)] + [(1, 700)] * 43, 32, 8, 128),
    call([(300, 900), (0, 40), (2, 800), (1, 30)], 12, 4, 80, window=250),
    # two tiles of the largest heads in bfloat16
    call([(16, 90000), (1, 70000), (3, 8), (12, 60000)], 16, 4, 256, bf16=True, max_kv=1 << 20),
    call([(60, 4000), (3, 4000), (1, 1)], 4, 4, 192, bf16=True, max_kv=1 << 20),
    # bounds far above the lengths
    call([(5, 300), (1, 40), (1, 900)], 32, 8, 128, max_new=400, rows=400),
    call([(5, 300), (0, 40), (1, 900)], 32, 8, 64, max_new=9, max_kv=1 << 22, bf16=True),
]


def test_prompts_among_single_tokens(walk):
    for r in check(walk, MIXED):
        assert not r["many"] and r["worked"] > 0


def test_starts_out_of_bounds(walk):
    """Row starts that no call can have: sequences without rows, wherever they begin, are passed over."""
    for start, kv in (([0, 4, 1 << 30, (1 << 31) - 1], [100, 150, 120]), ([0, 1 << 30, 1 << 30, 6], [90, 80, 70]),
                      ([5, 5, 6, 2], [40, 900, 30]), ([-7, 3, 3, 6], [10, 2000, 600])):
        for bf16 in (0, 1):
            check(walk, [[bf16, 32, 8, 128, 16, 6, 4, 1 << 22, 0, 0, 3] + start + kv])
    # rows behind such a sequence, in the same stretch
    check(walk, [[bf16, 32, 8, 128, 16, 6, 4, 1 << 22, 0, 0, 3, 0, 1 << 30, 4, 6, kv, 700, 3000]
                 for bf16 in (0, 1) for kv in range(100, 9000, 100)])


@pytest.mark.parametrize("seed", range(8))
def test_random_calls(walk, seed):
    rng = random.Random(seed)
    calls = []
    for _ in range(60):
        H, G = rng.choice([(32, 8), (16, 16), (8, 1), (28, 4), (12, 4), (64, 8)])
        lens = []
        for _ in range(rng.choice([1, 2, 5, 17, 70, 600])):
            n = rng.choice([0, 1, 1, 1, 2, 5, rng.randint(1, 40), rng.randint(1, 900) if rng.random() < 0.1 else 1])
            lens.append((n, rng.choice([0, 1, n, n + rng.randint(0, 300), n + rng.randint(0, 5000)])))
        window = rng.choice([0, 0, rng.randint(1, 2000)])
        calls.append(call(lens, H, G, rng.choice([64, 80, 128, 192, 256]), bf16=rng.random() < 0.4, window=window,
                          masked=window == 0 and rng.random() < 0.3, max_new=rng.choice([None, None, 1024, 7]),
                          max_kv=rng.choice([None, 1 << 22, 1 << 17])))
    rows = check(walk, calls)
    assert sum(not r["many"] for r in rows) >= 20
