"""The plan of the attention under a rule, its own source compiled for the CPU and run there thread by thread: whatever a call's
arrays hold, each piece it hands out lies inside the call's rows, pages and records, keys that no row sees are left out where a run
of them is long, and each key that a row sees is covered once."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib", "llvm", "bin", "clang++")
F32, BF16 = 0, 1
FAR = (1 << 31) - 1
HEADS = [(32, 8, 128), (6, 2, 64), (16, 1, 128), (5, 1, 64)]
TYPES = [(BF16, BF16), (F32, BF16), (F32, F32)]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "rule_plan")
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-I", os.path.join(ROOT, "tests", "host_hip"), "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2605_30852_amd", "csrc"), "-x", "c++",
                    os.path.join(ROOT, "tests", "host_hip", "rule_plan.cpp"), "-o", exe], check=True)

    def run(cases):
        r = subprocess.run([exe], input="\n".join(t for _, t in cases), capture_output=True, text=True, timeout=600)
        lines = r.stdout.splitlines()
        assert r.returncode == 0 and len(lines) == len(cases), (r.returncode, len(lines), len(cases), r.stderr[-500:])
        bad = [(name, line) for (name, _), line in zip(cases, lines) if not line.startswith("ok")]
        assert not bad, bad[:5]
        return [tuple(map(int, line.split()[1:])) for line in lines]

    return run


def text(prefix, heads, types, max_pages, lens, seqs, cu, plens=(), rows=None, max_len=0, window=0, first=None, opened=None):
    hq, hkv, dh = heads
    rows = len(seqs) if prefix else rows
    head = [int(prefix), hq, hkv, dh, types[0], types[1], len(lens), max_pages, len(seqs), rows, len(plens), max_len, window,
            int(first is not None), int(opened is not None)]
    return " ".join(map(str, [*head, *seqs, *cu, *plens, *lens, *(first or []), *(opened or [])]))


def starts(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


def documents(rng, rows, cached, mean):
    """First keys of rows in documents, some rows in none of them, some seeing everything."""
    out = []
    for r, c in zip(rows, cached):
        at = 0
        for i in range(r):
            if rng.random() < 1.0 / mean:
                at = c + i
            out.append(rng.choice([at] * 12 + [FAR, c + i + 1, 0, -5]))
    return out


def rules(rng, rows, cached):
    far = max(c + r for r, c in zip(rows, cached)) + 1
    for window in (0, 1, 17, 700):
        yield dict(window=window)
        yield dict(window=window, opened=[rng.choice([0, 1, 63, 64, 65, rng.randint(0, far), far + 7, -1]) for _ in rows])
    yield dict(window=rng.randint(1, 500), first=documents(rng, rows, cached, 90), opened=[rng.randint(0, 200) for _ in rows])
    yield dict(first=documents(rng, rows, cached, 20))
    yield dict(first=[FAR] * sum(rows))
    yield dict(first=[rng.randint(0, far) for _ in range(sum(rows))], window=FAR)


def test_prompts(plan):
    rng, cases = random.Random(1), []
    for heads in HEADS:
        for types in TYPES:
            for n, most, far in ((1, 600, 0), (5, 90, 3000), (30, 9, 200), (3, 2, 9000)):
                rows = [rng.randint(0, most) for _ in range(n)]
                rows[0] = max(rows[0], 1)
                cached = [rng.choice([0, rng.randint(0, far)]) for _ in rows]
                lens = [r + c for r, c in zip(rows, cached)]
                for rule in rules(rng, rows, cached):
                    cases.append(((heads, types, rows, cached, rule),
                                  text(False, heads, types, 640, lens, list(range(n)), starts(rows), rows=sum(rows), **rule)))
    plan(cases)


def test_lengths_that_no_rows_fit(plan):
    """Sequences shorter than their rows, sequences that are none, rows behind the last sequence, starts that do not ascend."""
    rng, cases = random.Random(2), []
    for heads in HEADS[:2]:
        for _ in range(40):
            rows = [rng.randint(0, 80) for _ in range(4)]
            lens = [rng.choice([0, -3, 5, 90, 200]) for _ in rows]
            seqs = [rng.choice([0, 1, 2, 3, 9, -1]) for _ in rows]
            cu = starts(rows)
            total = cu[-1] + 3
            if rng.random() < 0.3:
                rng.shuffle(cu)
            rule = dict(window=rng.choice([0, 30]), first=[rng.randint(-2, 210) for _ in range(total)],
                        opened=[rng.randint(-2, 210) for _ in rows])
            cases.append(((heads, rows, lens, seqs, cu, rule), text(False, heads, (BF16, BF16), 16, lens, seqs, cu, rows=total, **rule)))
    plan(cases)


def test_groups(plan):
    rng, cases = random.Random(3), []
    for heads in HEADS:
        for types in TYPES:
            for groups, most in (([1], 4000), ([1] * 40, 900), ([9, 24, 1, 3], 3000), ([70, 5], 700), ([2, 0, 2], 100)):
                n = sum(groups)
                plens = [rng.randint(0, most) for _ in groups]
                lens = [max(0, p + rng.randint(-5, 300)) for g, p in zip(groups, plens) for _ in range(g)]
                for rule in rules(rng, [1] * n, [max(0, x - 1) for x in lens]):
                    with_groups = dict(plens=plens) if rng.random() < 0.8 else {}
                    cu = starts(groups) if with_groups else [0]
                    cases.append(((heads, types, groups, plens, lens, rule),
                                  text(True, heads, types, 400, lens, list(range(n)), cu, **with_groups, **rule)))
    plan(cases)


def test_unseen_keys_are_left_out(plan):
    """Under a window of 64 a row of 8000 keys takes the pages of its window and of the open keys, not more than a tile beyond."""
    cases = []
    for opened in (0, 4, 100):
        cases.append((opened, text(True, (32, 8, 128), (BF16, BF16), 500, [8000] * 3, [0, 1, 2], [0], window=64, opened=[opened] * 3)))
        cases.append((opened, text(False, (32, 8, 128), (BF16, BF16), 500, [8000], [0], [0, 32], rows=32, window=64, opened=[opened])))
    got = plan(cases)
    for (opened, _), (_, _, keys), n in zip(cases, got, [3, 1] * 3):
        assert keys <= n * (64 + 32 + (opened + 63) // 64 * 64 + 16), (opened, keys)
