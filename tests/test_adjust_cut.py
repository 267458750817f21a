"""How adjusted logits are cut into workgroups, on the host with the launch's own function (CPU): every row and token has one, and the
GPU tests' shapes take every form there is."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cut") / "adjust_cut_ref")
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", exe, os.path.join(HERE, "adjust_cut_ref.cpp")], check=True)

    def run(calls):
        text = "\n".join(" ".join(str(x) for x in c) for c in calls) + "\n"
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.strip().splitlines()]

    return run


def test_workgroups_cover_all_rows_and_tokens(cut):
    calls = [(bf16, B, R, V) for bf16 in (0, 1) for B in (1, 3, 64, 500, 5000) for R in (1, 5, 20, 33, 1056) for V in (1, 1000, 8192, 8193, 524288)]
    for (_, B, R, V), (seg, per, wgs) in zip(calls, cut(calls)):
        assert 1 <= per <= R and wgs == -(-V // seg) * B * -(-R // per)


@pytest.mark.parametrize("bf16", [0, 1])
def test_gpu_tests_take_every_form(cut, bf16):
    """Few rows in short stretches (test_gpu_adjust.py), one row and several in long ones; as many as the sequence has, a number that
    does not divide them, workgroups that begin inside a path; and the headline's form."""
    from test_gpu_adjust_rows import SHAPES

    rows = [(B, K * (gamma + 1), V, gamma + 1) for B, K, gamma, V in SHAPES]
    forms = cut([(bf16, B, R, V) for B, R, V, _ in rows])
    short, per_few, _ = cut([(bf16, 3, 8, 20001)])[0]
    long, per_headline, _ = cut([(bf16, 64, 20, 128256)])[0]
    assert per_few == 1 and short < long and per_headline == 20
    assert all(seg == long and per > 1 for seg, per, _ in forms)
    assert any(per == R for (_, R, _, _), (_, per, _) in zip(rows, forms))
    assert any(R % per and per % S and S % per for (_, R, _, S), (_, per, _) in zip(rows, forms))
    assert any(per == 20 and V > 10 * long for (_, _, V, _), (_, per, _) in zip(rows, forms))
    assert all(V % 8 or V == 1000 for _, _, V, _ in rows)
