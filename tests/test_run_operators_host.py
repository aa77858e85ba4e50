"""The driver that the operators' profile is taken with (perf/run_operators.py):
its cases, commands and units, without a GPU."""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
from perf import operators, run_operators  # noqa: E402


def test_cases_have_names_of_their_own_and_all_keys():
    names = [c["name"] for c in operators.listed() + run_operators.FORMS]
    assert len(set(names)) == len(names) == len(run_operators.cases())
    keys = {c["op"]: set(c) for c in operators.listed()}
    for c in run_operators.FORMS:
        assert set(c) == keys[c["op"]], c["name"]
        w = operators.work(c)
        assert w["bytes"] > 0 and w["flops"] > 0


def test_commands(capsys):
    run_operators.commands("out")
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == len(run_operators.cases()) * (1 + len(run_operators.COUNTERS))
    for line in lines:  # counters in runs of their own, with the kernel trace alone
        assert line.startswith("rocprofv3 --pmc " if "--pmc" in line else "rocprofv3 --kernel-trace ")
        assert " -- python3 perf/run_operators.py run " in line


def test_units():
    case = run_operators.cases()["plain_long_128_bf16"]
    assert run_operators.units(case, "attention_kernel<x>") == 32 * 8192 * 8193 // 2
    case = run_operators.cases()["loss_prompts_f32"]
    assert run_operators.units(case, "loss_rows_kernel<x>") == (case["t"] - case["skip"]) * case["v"]
    name = "void mezo::attention_kernel<false, 64u, 4u, false, (mezo::Mode)1>(mezo::AttentionArgs)"
    assert run_operators._short(name) == "attention_kernel<false, 64u, 4u, false, 1>"
