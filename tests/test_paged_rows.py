"""How many keys a row of the fp32 paged attention looks at, whatever the device data say: the kernel's own arithmetic, compiled for the host
(paged_rows_main.cpp)."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    src, where = os.path.join(ROOT, "tests", "paged_rows_main.cpp"), tmp_path_factory.mktemp("rows")
    out = [str(where / n) for n in ("rows.o", "runtime.o", "rows")]
    for cmd in (["hipcc", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-w", "-I" + os.path.join(ROOT, "include"),
                 "-I" + os.path.join(ROOT, "paper_2505_19634_amd", "csrc"), "-x", "hip", "-c", src, "-o", out[0]],
                ["g++", "-DPAGED_ROWS_RUNTIME", "-c", src, "-o", out[1]],
                ["g++", "-no-pie", out[0], out[1], "-Wl,--unresolved-symbols=ignore-all", "-o", out[2]]):
        subprocess.run(cmd, check=True, capture_output=True, text=True)
    return out[2]


def rows(program, columns, shift, T, starts, lengths):
    line = " ".join(map(str, [columns, shift, T, len(lengths)] + starts + lengths))
    res = subprocess.run([program], input=line + "\n", check=True, capture_output=True, text=True)
    return [tuple(map(int, l.split())) for l in res.stdout.splitlines()]


def test_what_the_contract_allows(program):
    starts, lengths = [1, 4, 4, 9], [10, 7, 3]   # the last branch has more new tokens than tokens
    got = {(t, b): keys for t, b, keys, _ in rows(program, 4, 4, 11, starts, lengths)}
    for t in range(11):
        for b in range(3):
            n = starts[b + 1] - starts[b]
            want = max(0, lengths[b] - n + t - starts[b] + 1) if starts[b] <= t < starts[b + 1] else -1
            assert got[t, b] == want, (t, b)


def test_a_row_never_sees_more_than_the_table_holds(program):
    """Three branches of 64 tokens, four columns of 16, 40 rows, starts 0, 40, 2, 4: row 39 is looked for in the last branch, which holds rows 2 and 3."""
    cases = [(4, 4, 40, [0, 40, 2, 4], [64, 64, 64])]
    rng = random.Random(1)
    for _ in range(40):
        B, T = rng.randint(1, 5), rng.randint(1, 50)
        cases.append((rng.randint(1, 6), 4, T, [rng.randint(-5, T + 9) for _ in range(B + 1)], [rng.choice([-3, 0, 17, 90, 2 ** 31 - 1]) for _ in range(B)]))
    for columns, shift, T, starts, lengths in cases:
        for t, b, keys, length in rows(program, columns, shift, T, starts, lengths):
            assert -1 <= keys <= length <= columns << shift, (starts, lengths, t, b, keys)
