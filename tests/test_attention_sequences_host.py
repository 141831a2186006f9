"""Which rows belong to which sequence, as attention's kernels find it (span_of in csrc/attention.h), run on the CPU and held to a search through all
offsets: a row behind the last one has no sequence, whatever the offsets are, since what a kernel gives a sequence it writes."""
import os
import random
import subprocess

import pytest

from paper_2509_03110_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    to = tmp_path_factory.mktemp("sequences")
    with open(os.path.join(build.CSRC, "attention.h")) as f:
        text = f.read()
    text = text[text.index("struct Sequences {"):]
    with open(os.path.join(to, "sequences.inc"), "w") as f:
        f.write(text[:text.index("#endif")])
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", str(to), os.path.join(HERE, "sequences_driver.cpp"), "-o",
                    os.path.join(to, "driver")], check=True)
    return os.path.join(to, "driver")


def run(driver, kind, cases):
    r = subprocess.run([driver, kind], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout == "%d cases\n" % len(cases), r.stdout + r.stderr[-2000:]


def case(rows, offsets):
    return [rows, len(offsets) - 1] + offsets


def spread(rows, n):
    return [rows * i // n for i in range(n + 1)]


def test_sequences_around_a_wavefronts_lanes(driver):
    run(driver, "list", [case(rows, spread(rows, n)) for rows in (1, 33, 64, 100, 128, 200, 300, 1000) for n in list(range(1, 5)) + list(range(58, 69)) + [126, 127, 128, 200]])


def test_offsets_padded_with_empty_sequences(driver):
    run(driver, "list", [case(rows, head * [0] + spread(rows, n) + tail * [rows]) for rows in (100, 128, 300) for n in (1, 5, 30) for head in (0, 3, 64)
                         for tail in (1, 32, 33, 34, 57, 58, 59, 60, 61, 62, 63, 64, 130)])


def test_any_offsets(driver):
    rng = random.Random(1)
    cases = []
    for _ in range(400):
        rows = rng.randint(1, 400)
        n = rng.choice([rng.randint(1, 8), rng.randint(55, 75), rng.randint(1, 300)])
        lo, hi = rng.choice([(0, rows), (-20, rows + 20), (rng.randint(0, rows), rows), (0, rng.randint(0, rows))])
        values = [rng.randint(min(lo, hi), max(lo, hi)) for _ in range(rng.choice([n + 1, 3, 12]))]
        cases.append(case(rows, sorted(rng.choice(values) for _ in range(n + 1))))
    run(driver, "list", cases)


def test_more_sequences_than_half_of_32_bits_count(driver):
    """Numbers of sequences near the limits of int: nearly all are empty, of offsets that are not in memory."""
    run(driver, "many", [[100, n, tail] for n in (2 ** 30 - 1, 2 ** 30 + 70, 2 ** 31 - 1) for tail in (1, 5, 100)])
