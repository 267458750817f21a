"""The forms that attention over a cache held in 4 bits takes, on the host with the launch's own functions (CPU): the GPU tests have a
call of each that any call was found to take."""
import os
import random
import subprocess

import pytest

torch = pytest.importorskip("torch")

from test_attention_division import call  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("forms") / "attention4_forms_ref")
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", exe, os.path.join(HERE, "attention4_forms_ref.cpp")], check=True)

    def run(calls):
        text = "\n".join(" ".join(str(x) for x in c) for c in calls) + "\n"
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [(c[0], *(int(x) for x in line.split())) for c, line in zip(calls, out)]

    return run


def taken(forms):
    from test_gpu_serving4_forms import BF16, FORMS, lengths

    return forms([call(lengths(B, n, kv), H, G, D, bf16=dtype == BF16) for dtype, H, G, D, B, n, kv in FORMS])


def test_each_form_once(forms):
    have = taken(forms)
    assert len(set(have)) == len(have) == 50
    # (bfloat16, many, padded head, tile): every kernel that is compiled
    kernels = {(bf16, 0, D, rows) for bf16, D, rows in [(1, 64, 16), (1, 64, 32), (1, 128, 16), (1, 128, 32), (1, 256, 16), (1, 256, 32),
                                                        (0, 64, 16), (0, 64, 32), (0, 128, 16), (0, 256, 16)]}
    kernels |= {(1, 1, 64, 128), (1, 1, 64, 256), (1, 1, 128, 128), (1, 1, 128, 256), (1, 1, 256, 128)}
    assert {f[:4] for f in have} == kernels
    for k in kernels:
        joined = [f[4:] for f in have if f[:4] == k]
        assert sorted(joined) == ([(0, 0), (0, 1)] if k[1] else [(0, 0), (0, 1), (1, 0), (1, 1)])


@pytest.mark.parametrize("seed", range(4))
def test_other_calls_take_no_other_form(forms, seed):
    have = set(taken(forms))
    rng = random.Random(seed)
    calls = []
    for _ in range(1500):
        H, G = rng.choice([(32, 8), (16, 16), (8, 1), (28, 4), (12, 4), (64, 8), (4, 1), (1024, 1024)])
        B, n = rng.choice([1, 2, 3, 8, 16, 33, 64, 130, 300]), rng.choice([1, 1, 2, 4, 5, 9, 17, 33, 130])
        kv = int(2 ** rng.uniform(3, 17)) + n
        lens = [(rng.randint(0, n), rng.randint(0, kv)) for _ in range(B)]
        window = rng.choice([0, 0, 0, rng.randint(1, 4000)])
        calls.append(call(lens, H, G, rng.choice([8, 64, 80, 128, 192, 256]), bf16=rng.random() < 0.6, window=window,
                          masked=not window and rng.random() < 0.2, max_new=n, max_kv=kv))
    assert set(forms(calls)) <= have
