"""Whether rows by three strides lie on each other (csrc/strided.h), against the elements themselves (no GPU)."""
import random
import subprocess

from paper_2503_08524_amd import build as d3_build

PROGRAM = """
#include <cstdio>
#include "strided.h"
int main() {
    long long w, n[3], s[3], apart;
    while (scanf("%lld %lld %lld %lld %lld %lld %lld %lld", &w, n, n + 1, n + 2, s, s + 1, s + 2, &apart) == 8)
        putchar(d3::rows_overlap(w, {{n[0], s[0]}, {n[1], s[1]}, {n[2], s[2]}}, apart) ? '1' : '0');
}
"""


def _overlap(w, n, s, apart):
    """(truth, nested): an element that two rows have in common; every stride passes over what the smaller ones span."""
    at = [a + i * s[0] + j * s[1] + k * s[2] + e for a in ({0, apart} if apart else {0}) for i in range(n[0]) for j in range(n[1]) for k in range(n[2]) for e in range(w)]
    span, nested = w, True
    for size, many in sorted((abs(x), y) for x, y in zip(s, n) if y > 1):
        nested &= size >= span
        span += (many - 1) * size
    return len(set(at)) < len(at), nested


def test_rows_that_lie_on_each_other(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", d3_build.CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    rng, cases = random.Random(1), []
    for _ in range(6000):
        w = rng.choice([1, 2, 4])
        n = [rng.randint(1, 4) for _ in range(3)]
        s, span = [0, 0, 0], w
        for j in rng.sample(range(3), 3):                      # most are nested, with gaps or without; some have a stride that is any
            s[j] = (span + rng.choice([0, 0, 1, w, 3 * w])) * rng.choice([1, 1, -1])
            span += (n[j] - 1) * abs(s[j])
            if rng.random() < 0.1:
                s[j] = rng.randint(-2, 12)
        apart = rng.choice([0, span, -span, 1]) if rng.random() < 0.2 else rng.randint(-2 * span, 2 * span)
        cases.append((w, n, s, apart))
    text = "\n".join(" ".join(map(str, [w, *n, *s, apart])) for w, n, s, apart in cases)
    got = subprocess.run([str(tmp_path / "t")], input=text, capture_output=True, text=True, check=True).stdout
    assert len(got) == len(cases)
    count = [0, 0]
    for case, g in zip(cases, got):
        truth, nested = _overlap(*case)
        if nested:
            assert (g == "1") == truth, case
            count[truth] += 1
        else:
            assert g == "1", case
    assert min(count) > 500
    # sizes at the ends of 64 bits
    far = subprocess.run([str(tmp_path / "t")], input=f"128 268435456 4 2 {2 ** 62} 128 {-2 ** 63 + 1} 512\n128 268435456 4 2 512 128 {2 ** 40} {-2 ** 62}\n", capture_output=True, text=True, check=True).stdout
    assert far == "10"
