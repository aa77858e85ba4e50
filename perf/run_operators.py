"""Runs cases of the forward pass's operators, or of those of generation, for a
profiler, and summarises what it wrote.

    python3 perf/run_operators.py run CASE [PASSES]          # under rocprofv3, one case a run
    python3 perf/run_operators.py commands OUT [generation]  # the commands of all cases, runs into OUT/<case>/<what>
    python3 perf/run_operators.py summary OUT [generation]   # the tables, from those runs

CASE is a listed case of perf/operators.py or perf/more_operators.py (those of
generation), or one of FORMS or MORE_FORMS below: forms of the operators with code of
their own that no listed case reaches.
"""
from __future__ import annotations

import collections
import csv
import glob
import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from perf import more_operators, operators  # noqa: E402

_ATTEND = {"op": "attend", "dtype": "bf16", "docs": 1, "lo": 8192, "hi": 8192, "new": 0, "capacity": 0, "heads": 32,
           "kv_heads": 32, "dim": 128, "prefix": False, "softcap": 0.0, "bias": False, "lens": 5}

FORMS = [
    # one long causal document, nothing else: heads of 128 and of 64
    {**_ATTEND, "name": "plain_long_128_bf16"},
    {**_ATTEND, "name": "plain_long_64_bf16", "dim": 64},
    # packed documents without a bias
    {**_ATTEND, "name": "plain_packed_64_bf16", "docs": 16, "lo": 50, "hi": 2048, "dim": 64, "prefix": True, "lens": 4},
    # a bias by distance with heads of 128; with a cap as well
    {**_ATTEND, "name": "biased_long_128_bf16", "bias": True},
    {**_ATTEND, "name": "capped_biased_long_128_bf16", "bias": True, "softcap": 30.0},
    # a cap past those that have the short form
    {**_ATTEND, "name": "cap300_long_128_bf16", "softcap": 300.0},
    # full precision with heads of 128: prompts and long caches
    {**_ATTEND, "name": "packed_128_f32", "dtype": "f32", "docs": 16, "lo": 50, "hi": 2048, "heads": 16, "kv_heads": 16,
     "prefix": True, "lens": 4},
    {**_ATTEND, "name": "tokens_cache_128_f32", "dtype": "f32", "docs": 12, "lo": 500, "hi": 16384, "new": 1,
     "capacity": 16384, "kv_heads": 8, "lens": 2},
    # a few new tokens over a long cache: split keys and the join
    {**_ATTEND, "name": "new_tokens_cache_128_bf16", "lo": 16000, "hi": 16000, "new": 64, "capacity": 16000},
    # full precision out of a large product on whole tiles; few tiles and a long k
    {"op": "linear", "dtype": "f32", "out": "f32", "m": 2048, "k": 4096, "n": 4096, "pad": 0, "fresh": False,
     "name": "linear_2048_f32"},
    {"op": "linear", "dtype": "bf16", "out": "bf16", "m": 128, "k": 16384, "n": 4096, "pad": 0, "fresh": False,
     "name": "linear_128_bf16"},
]

_PAGED = {"op": "attend", "dtype": "bf16", "docs": 4, "lo": 600, "hi": 8192, "new": 1000, "tree": False, "page": 32,
          "heads": 32, "kv_heads": 32, "dim": 128, "prefix": False, "softcap": 0.0, "bias": False, "lens": 6}
_APPEND = {"op": "append", "dtype": "f32", "docs": 16, "lo": 50, "hi": 2048, "new": 0, "tree": False, "page": 32,
           "heads": 32, "kv_heads": 32, "dim": 128, "rot": 128, "interleaved": False, "lens": 3}
_PRODUCT = {"op": "product", "dtype": "bf16", "out": "bf16", "m": 1, "k": 4096, "n": 16384, "pad": 0}

MORE_FORMS = [
    # prompts in full precision, and turned by vectors of two elements
    {**_APPEND, "name": "append_prompts_f32"},
    {**_APPEND, "name": "append_prompts_rot20_bf16", "dtype": "bf16", "rot": 20},
    # full precision: a tree, and single tokens over long caches
    {**_PAGED, "name": "trees_128_f32", "dtype": "f32", "docs": 8, "lo": 500, "new": 61, "tree": True, "kv_heads": 8,
     "lens": 5},
    {**_PAGED, "name": "tokens_128_f32", "dtype": "f32", "docs": 12, "lo": 500, "hi": 16384, "new": 1, "page": 16,
     "kv_heads": 8, "lens": 2},
    # chunks in full precision
    {**_PAGED, "name": "chunks_128_f32", "dtype": "f32"},
    # a chunk with capped scores; small pages
    {**_PAGED, "name": "chunks_capped_128_bf16", "softcap": 30.0},
    {**_PAGED, "name": "chunks_page8_128_bf16", "page": 8},
    # few activations: full precision, a vocabulary's rows, batches of 24 and 64; a few hundred
    {**_PRODUCT, "name": "product_1_f32", "dtype": "f32", "out": "f32"},
    {**_PRODUCT, "name": "product_24_f32", "dtype": "f32", "out": "f32", "m": 24},
    {**_PRODUCT, "name": "product_vocabulary_bf16", "n": 50272},
    {**_PRODUCT, "name": "product_64_bf16", "m": 64},
    {**_PRODUCT, "name": "product_192_bf16", "m": 192},
    {**_PRODUCT, "name": "product_256_bf16", "m": 256},
    # rows of weights that end within a block
    {**_PRODUCT, "name": "product_ragged_bf16", "k": 4100},
    {**_PRODUCT, "name": "product_ragged_16_f32", "dtype": "f32", "out": "f32", "m": 16, "k": 4100},
    # full precision on whole blocks; tiles of 128
    {**_PRODUCT, "name": "product_2048_f32", "dtype": "f32", "out": "f32", "m": 2048, "n": 4096},
    {**_PRODUCT, "name": "product_2048_bf16", "m": 2048, "n": 4096},
]

COUNTERS = {
    "fetch": "FETCH_SIZE",
    "write": "WRITE_SIZE",
    "valu": "SQ_ACTIVE_INST_VALU SQ_INSTS_VALU SQ_VALU_MFMA_BUSY_CYCLES SQ_BUSY_CU_CYCLES SQ_LDS_BANK_CONFLICT SQ_WAVES "
            "GRBM_GUI_ACTIVE",
}


def cases(generation=False):
    return {c["name"]: c for c in (more_operators.listed() + MORE_FORMS if generation else operators.listed() + FORMS)}


def run(name, passes, generation=False):
    """`passes` passes over three states in turn, after one over each."""
    import torch
    module = more_operators if generation else operators
    module.own = True
    states = [module.prepare(cases(generation)[name], seed) for seed in range(3)]
    for s in states:
        module.run(s)
    torch.cuda.synchronize()
    for i in range(passes):
        module.run(states[i % 3])
    torch.cuda.synchronize()


def commands(out, generation=False):
    kind = " generation" if generation else ""
    for name in cases(generation):
        print(f"rocprofv3 --kernel-trace --stats -f csv -d {out}/{name}/trace -o p -- "
              f"python3 perf/run_operators.py run {name} 30{kind}")
        for what, counters in COUNTERS.items():
            print(f"rocprofv3 --pmc {counters} --kernel-trace -f csv -d {out}/{name}/{what} -o p -- "
                  f"python3 perf/run_operators.py run {name} 2{kind}")


def _rows(out, name, what, file):
    for path in glob.glob(os.path.join(out, name, what, "**", file), recursive=True):
        with open(path) as f:
            yield from (r for r in csv.DictReader(f) if "mezo::" in r.get("Name", r.get("Kernel_Name", "")))


def _short(kernel):
    for long, short in (("(mezo::Mode)", ""), (", mezo::AttentionArgs", ""), (", mezo::PagedArgs", ", pages")):
        kernel = kernel.replace(long, short)
    return kernel.split("(mezo::")[0].split("mezo::")[1]


def _counters(out, name):
    sums = collections.defaultdict(lambda: collections.defaultdict(list))
    for what in COUNTERS:
        for r in _rows(out, name, what, "p_counter_collection.csv"):
            sums[_short(r["Kernel_Name"])][r["Counter_Name"]].append(float(r["Counter_Value"]))
    return {k: {c: sum(v) / len(v) for c, v in d.items()} for k, d in sums.items()}


def summary(out, generation=False):
    """One line a case and kernel, averages over its dispatches (of all states)."""
    from paper_2306_10015_amd import profile_summary
    print("| case | kernel | µs (min) | read MB | written MB | VALU % | matrix % | CU busy % | LDS conflicts "
          "| VALU instr a unit |")
    print("|---|---|---|---|---|---|---|---|---|---|")
    for name, case in cases(generation).items():
        counted = _counters(out, name)
        trace = sorted(_rows(out, name, "trace", "p_kernel_stats.csv"), key=lambda r: -float(r["AverageNs"]))
        for r in trace:
            kernel = _short(r["Name"])
            c = counted.get(kernel, {})
            line = [f"`{name}`", f"`{kernel}`", f"{float(r['AverageNs']) / 1e3:.1f} ({float(r['MinNs']) / 1e3:.1f})"]
            if c:
                simds = 4 * c["SQ_BUSY_CU_CYCLES"]
                unit = units(case, kernel)
                line += [f"{c['FETCH_SIZE'] * 2 / 1e3:.1f}", f"{c['WRITE_SIZE'] / 1e3:.1f}",
                         f"{100 * 4 * c['SQ_ACTIVE_INST_VALU'] / simds:.0f}",
                         f"{100 * c['SQ_VALU_MFMA_BUSY_CYCLES'] / simds:.0f}",
                         f"{100 * c['SQ_BUSY_CU_CYCLES'] / (256 * c['GRBM_GUI_ACTIVE'] / 8):.0f}",
                         f"{c['SQ_LDS_BANK_CONFLICT']:.0f}",
                         f"{64 * c['SQ_INSTS_VALU'] / unit:.1f}" if unit else ""]
            print("| " + " | ".join(line + [""] * (10 - len(line))) + " |")
    print()
    for unit in (("paged_attention.hip", "cache_append.hip", "nf4_linear.hip") if generation
                 else ("attention.hip", "f8.hip", "token_loss.hip")):
        print(f"Sources of `{unit}` ({', '.join(f'`{os.path.basename(s)}`' for s in profile_summary.unit_sources(unit))}) "
              f"sha256: `{profile_summary.source_hash(unit)}`  ")


def units(case, kernel):
    """What a case's kernel works through: scores that count, values quantized, logits,
    weights decoded."""
    if kernel.startswith("attention_kernel"):
        module = more_operators if "page" in case else operators
        return module.work(case)["flops"] // (4 * case["dim"])
    if kernel.startswith(("nf4_thin", "nf4_ragged", "nf4_expand")):
        return case["n"] * case["k"]
    if kernel.startswith("loss_rows"):
        return (case["t"] - case["skip"]) * case["v"]
    if kernel.startswith("f8_quantize") and not case["fresh"]:
        return case["m"] * case["k"]
    return 0


if __name__ == "__main__":
    if sys.argv[1] == "run":
        run(sys.argv[2], int(sys.argv[3]) if len(sys.argv) > 3 else 30, "generation" in sys.argv[4:])
    else:
        {"commands": commands, "summary": summary}[sys.argv[1]](sys.argv[2], "generation" in sys.argv[3:])
