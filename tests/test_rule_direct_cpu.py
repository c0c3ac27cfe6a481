"""Calls under a rule that go without a plan, their pieces worked out on the CPU by the library's own source, and plans of short prompts,
which split nothing: pieces inside the call's rows and pages, each row once, each key that a row sees once."""
import os
import random
import subprocess

import pytest

from tests.test_rule_plan_cpu import BF16, CLANG, F32, FAR, HEADS, ROOT, TYPES, documents, plan, rules, starts, text  # noqa: F401


@pytest.fixture(scope="module")
def direct(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("direct") / "rule_direct")
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-I", os.path.join(ROOT, "tests", "host_hip"), "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2605_30852_amd", "csrc"), "-x", "c++",
                    os.path.join(ROOT, "tests", "host_hip", "rule_direct.cpp"), "-o", exe], check=True)

    def run(cases):
        r = subprocess.run([exe], input="\n".join(t for _, t in cases), capture_output=True, text=True, timeout=600)
        lines = r.stdout.splitlines()
        assert r.returncode == 0 and len(lines) == len(cases), (r.returncode, len(lines), len(cases), r.stderr[-500:])
        bad = [(name, line) for (name, _), line in zip(cases, lines) if line != "plan" and not line.startswith("ok")]
        assert not bad, bad[:5]
        return lines

    return run


def test_short_prompts(direct):
    """Lengths that are known to be short, or keys that a window bounds."""
    rng, cases = random.Random(11), []
    for heads in HEADS:
        for types in TYPES[:1] + TYPES[2:]:
            for n, most, far in ((1, 30, 0), (4, 9, 400), (6, 3, 480)):
                rows = [rng.randint(0, most) for _ in range(n)]
                rows[-1] = max(rows[-1], 1)
                cached = [rng.randint(0, far) for _ in rows]
                lens = [r + c for r, c in zip(rows, cached)]
                for rule in rules(rng, rows, cached):
                    for max_len in {max(lens), 512}:
                        cases.append(((heads, types, rows, cached, rule, max_len), text(
                            False, heads, types, 64, lens, list(range(n)), starts(rows), rows=sum(rows), max_len=max_len, **rule)))
    lines = direct(cases)
    assert sum(line != "plan" for line in lines) > len(lines) // 2


def test_windows_over_long_caches(direct):
    """A window of at most 512 keys, whatever the lengths; rows behind the last sequence."""
    rng, cases = random.Random(12), []
    for heads in HEADS:
        for n in (1, 3):
            rows = [rng.randint(1, 20) for _ in range(n)]
            cached = [rng.choice([0, 40, rng.randint(0, 9000)]) for _ in rows]
            lens = [r + c for r, c in zip(rows, cached)]
            total = sum(rows) + 5
            for window in (1, 16, 17, 500, 512):
                for max_len in (0, max(lens)):
                    for rule in (dict(), dict(first=documents(rng, rows, cached, 9) + [0] * 5), dict(first=[FAR] * total)):
                        cases.append(((heads, rows, cached, rule, window), text(
                            False, heads, (BF16, BF16), 640, lens, list(range(n)), starts(rows), rows=total, max_len=max_len, window=window,
                            **rule)))
    assert all(line != "plan" for line in direct(cases))


def test_lengths_that_no_rows_fit(direct):
    """Sequences shorter than their rows, sequences that are none, starts that do not ascend."""
    rng, cases = random.Random(13), []
    for heads in HEADS[:2]:
        for _ in range(60):
            rows = [rng.randint(0, 20) for _ in range(4)]
            lens = [rng.choice([0, -3, 5, 90, 200]) for _ in rows]
            seqs = [rng.choice([0, 1, 2, 3, 9, -1]) for _ in rows]
            cu = starts(rows)
            total = cu[-1] + 3
            if rng.random() < 0.3:
                rng.shuffle(cu)
            rule = dict(window=rng.choice([0, 30]), first=[rng.randint(-2, 210) for _ in range(total)],
                        opened=[rng.randint(-2, 210) for _ in rows])
            cases.append(((heads, rows, lens, seqs, cu, rule), text(False, heads, (BF16, BF16), 16, lens, seqs, cu, rows=total, max_len=200,
                                                                  **rule)))
    assert all(line != "plan" for line in direct(cases))


def test_decode_rows(direct):
    """Short sequences, with groups or without, and as many rows under a window as fill the GPU, open keys beside it."""
    rng, cases = random.Random(14), []
    for heads in HEADS:
        for n, far, max_len in ((1, 512, 512), (30, 300, 300), (512 // heads[1], 3000, 0), (512 // heads[1] + 3, 5000, 5000)):
            lens = [rng.choice([0, 1, rng.randint(0, far)]) for _ in range(n)]
            for rule in rules(rng, [1] * n, [max(0, x - 1) for x in lens]):
                groups = dict(plens=[40]) if max_len == 300 and rng.random() < 0.5 else {}
                cases.append(((heads, lens, rule), text(True, heads, (BF16, BF16), 320, lens, list(range(n)), [0, n] if groups else [0],
                                                        max_len=max_len, **groups, **rule)))
    lines = direct(cases)
    assert sum(line != "plan" for line in lines) > len(lines) // 3


def test_plans_that_split_nothing(plan):  # noqa: F811
    """Prompts of at most 128 keys whose tiles are more than go without a plan: no piece is split, nothing is joined."""
    rng, cases = random.Random(15), []
    for heads in HEADS:
        for types in TYPES:
            for max_len in (1, 40, 127, 128):
                n = max(4, 8000 // heads[1] // max_len)  # two tiles of 16 queries a CU, and more
                rows = [rng.randint(max_len // 2, max_len) or 1 for _ in range(n)]
                cached = [rng.randint(0, max_len - r) for r in rows]
                lens = [r + c for r, c in zip(rows, cached)]
                for rule in list(rules(rng, rows, cached))[::3]:
                    cases.append(((heads, types, max_len, rule), text(False, heads, types, 8, lens, list(range(n)), starts(rows),
                                                                      rows=sum(rows), max_len=max_len, **rule)))
    got = plan(cases)
    assert all(records == 0 for _, records, _ in got)
