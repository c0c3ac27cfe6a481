"""The plan of the attention over a cache of several sequences, its own source compiled for the CPU and run there thread by
thread: whatever a call's arrays hold, each piece it hands out lies inside the call's rows, pages and records (a place that is
counted and not written, or records past their room, would be reads and writes anywhere on a GPU), and each row's keys are
covered once."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib", "llvm", "bin", "clang++")
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "seq_plan")
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-I", os.path.join(ROOT, "tests", "host_hip"), "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2605_30852_amd", "csrc"), "-x", "c++",
                    os.path.join(ROOT, "tests", "host_hip", "seq_plan.cpp"), "-o", exe], check=True)

    def run(cases):
        """cases: (name, text); all have to be ok. Returns each one's pieces and records."""
        r = subprocess.run([exe], input="\n".join(t for _, t in cases), capture_output=True, text=True, timeout=300)
        lines = r.stdout.splitlines()
        assert r.returncode == 0 and len(lines) == len(cases), (r.returncode, len(lines), len(cases), r.stderr[-500:])
        bad = [(name, line) for (name, _), line in zip(cases, lines) if not line.startswith("ok")]
        assert not bad, bad[:5]
        return [tuple(map(int, line.split()[1:])) for line in lines]

    return run


def text(prefix, heads, types, max_pages, lens, seqs, cu, plens=(), rows=None, max_len=0):
    hq, hkv, dh = heads
    rows = len(seqs) if prefix else rows
    head = [int(prefix), hq, hkv, dh, types[0], types[1], len(lens), max_pages, len(seqs), rows, len(plens), max_len]
    return " ".join(map(str, [*head, *seqs, *cu, *plens, *lens]))


def starts(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


HEADS = [(32, 8, 128), (6, 2, 64), (16, 1, 128), (5, 1, 64), (4, 4, 64)]
TYPES = [(BF16, BF16), (F32, BF16), (F32, F32)]


def test_prompts(plan):
    rng, cases = random.Random(1), []
    for heads in HEADS:
        for types in TYPES:
            for n, most, far in ((1, 700, 0), (7, 90, 3000), (40, 9, 200), (3, 1, 20000), (300, 5, 40)):
                rows = [rng.randint(0, most) for _ in range(n)]
                lens = [r + rng.choice([0, rng.randint(0, far)]) for r in rows]
                lens[rng.randrange(n)] = rng.choice([0, -3, 1 << 30, 5])
                seqs = rng.sample(range(n), n)
                by_seq = [0] * n
                for s, ln in zip(seqs, lens):
                    by_seq[s] = ln
                if n > 3:
                    seqs[rng.randrange(n)] = rng.choice([-1, n, 1 << 30])
                total = sum(rows) + rng.choice([0, 3])
                for max_len in (0, 5000):
                    cases.append(((heads, types, n, max_len), text(False, heads, types, 1300, by_seq, seqs, starts(rows), rows=max(1, total), max_len=max_len)))
    plan(cases)


def test_prompts_of_more_sequences_than_the_plan_keeps(plan):
    rng = random.Random(2)
    n = 4500
    rows = [rng.choice([0, 1, 1, 2]) for _ in range(n)]
    lens = [r + rng.randint(0, 9) for r in rows]
    plan([("many", text(False, (2, 1, 64), (BF16, BF16), 4, lens, list(range(n)), starts(rows), rows=sum(rows)))])


def test_prompts_whose_rows_do_not_ascend(plan):
    rng, cases = random.Random(3), []
    for heads in HEADS:
        n = 64
        for what in range(4):
            lens = [rng.randint(0, 4000) for _ in range(n)]
            cu = {0: [rng.randint(0, 400) for _ in range(n + 1)], 1: [0, 400] * (n // 2) + [0],
                  2: [rng.choice([-7, 0, 1 << 30, 200]) for _ in range(n + 1)], 3: list(range(n, -1, -1))}[what]
            cases.append(((heads, what), text(False, heads, TYPES[what % 3], 300, lens, list(range(n)), cu, rows=400)))
    plan(cases)


def groups_case(rng, heads, types, n, cu, far=3000, max_len=0):
    lens = [rng.randint(0, far) for _ in range(n)]
    plens = [rng.choice([0, rng.randint(0, far), far]) for _ in range(len(cu) - 1)]
    return text(True, heads, types, (far + 15) // 16, lens, list(range(n)), cu, plens, max_len=max_len)


def test_groups(plan):
    rng, cases = random.Random(4), []
    for heads in HEADS:
        for types in TYPES:
            for n in (1, 9, 70, 400):
                cut = sorted(rng.randint(0, n) for _ in range(rng.randint(0, n - 1)))
                for max_len in (0, 3000, 600):
                    cases.append(((heads, types, n), groups_case(rng, heads, types, n, [0, *cut, n], max_len=max_len)))
    cases.append(("all", groups_case(rng, (32, 8, 128), (BF16, BF16), 4096, list(range(0, 4097, 2)), 60)))
    plan(cases)


def test_groups_that_do_not_ascend(plan):
    """Overlapping groups would take more records than there is room for: no row shares anything then."""
    rng, cases = random.Random(5), []
    for heads in ((32, 8, 128), (1, 1, 64), (16, 1, 128), (6, 2, 64)):
        for n in (8, 256, 1000):
            odd = {"every other": [0 if i % 2 else n for i in range(n + 1)], "back and forth": [n if i % 2 else 0 for i in range(n + 1)],
                   "anywhere": [rng.randint(0, n) for _ in range(n + 1)], "outside": [rng.choice([-5, 0, n, n + 9, 1 << 30]) for _ in range(n + 1)],
                   "downwards": list(range(n, -1, -1)), "one step back": [0, n, n - 1, n], "from behind": [-4, 2, n + 7, n + 8]}
            for what, cu in odd.items():
                for types in (TYPES[n % 3], TYPES[2]):
                    cases.append(((heads, n, what, types), groups_case(rng, heads, types, n, cu[:n + 1])))
    plan(cases)
