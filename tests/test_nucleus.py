"""Arithmetic of the search for a nucleus' end (csrc/nucleus.h), checked on the CPU."""
import math
import os
import random
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_08537_b200", "csrc")

# needed() of the rows of standard input, four numbers each
NEEDED = """
#include "nucleus.h"
#include <stdio.h>
int main() {
    double enough, sure, w;
    unsigned in;
    while (scanf("%lf %lf %lf %u", &enough, &sure, &w, &in) == 4) printf("%.17g\\n", ardiff::needed(enough, sure, w, in));
}
"""


def program(d, name, source):
    (d / f"{name}.cpp").write_text(source)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", CSRC, str(d / f"{name}.cpp"), "-o", str(d / name)])
    return str(d / name)


@pytest.fixture(scope="module")
def needed(tmp_path_factory):
    exe = program(tmp_path_factory.mktemp("nucleus"), "needed", NEEDED)

    def call(rows):
        text = "\n".join(f"{e!r} {s!r} {w!r} {n}" for e, s, w, n in rows)
        # (a second for what takes milliseconds: a search that does not end is stopped here)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=20, check=True).stdout.split()
        assert len(out) == len(rows)
        return [float(v) for v in out]
    return call


def test_needed_is_the_least_number_that_reaches(needed):
    rng = random.Random(1)
    rows = []
    for _ in range(2000):
        n = rng.randint(1, 1 << 18)
        w = math.exp(-rng.uniform(0, 40))
        sure = rng.choice([0.0, rng.random(), 1000 * rng.random()])
        rows.append((sure + w * n * rng.uniform(0.0, 1.3), sure, w, n))
    for (enough, sure, w, n), got in zip(rows, needed(rows)):
        assert got == int(got) and 1 <= got <= n + 1
        assert got == n + 1 or sure + got * w >= enough
        assert got == 1 or sure + (got - 1) * w < enough


def test_needed_ends_where_the_mass_in_front_is_far_above(needed):
    """Thousands of logits at the largest value and thousands of equal ones 40 to 300 nats below: the elements in front hold twice the
    mass that is asked for, and more."""
    rng = random.Random(2)
    rows = [(rng.uniform(0.001, 0.5) * 3000, 3000.0 + rng.random(), math.exp(-rng.uniform(40, 300)), 3000) for _ in range(2000)]
    assert needed(rows) == [1.0] * len(rows)


def test_needed_of_weights_that_are_nothing(needed):
    assert needed([(0.5, 1.0, 0.0, 7), (0.5, 0.5, 0.0, 7)]) == [1.0, 1.0]
    assert needed([(0.5, 0.25, 0.0, 7), (0.5, 0.25, 5e-324, 7)]) == [8.0, 8.0]


# of the numbers of standard input, each as the bits of a float: its key, and the bits of the value of that key and of its two neighbours
KEYS = """
#include "nucleus.h"
#include <stdio.h>
int main() {
    unsigned b;
    while (scanf("%u", &b) == 1) {
        float x, v[3];
        memcpy(&x, &b, 4);
        const unsigned k = ardiff::key_of(x);
        unsigned o[3];
        for (int i = 0; i < 3; ++i) v[i] = ardiff::value_of(k - 1u + i);
        memcpy(o, v, 12);
        printf("%u %u %u %u\\n", k, o[0], o[1], o[2]);
    }
}
"""


def test_keys_are_the_logits_order_without_gaps(tmp_path):
    exe = program(tmp_path, "keys", KEYS)
    rng = np.random.default_rng(1)
    most = np.float32(np.finfo(np.float32).max)
    bits = [0, 1, 2, 0x7fffff, 0x800000, 0x3f800000, int(most.view(np.uint32))] + rng.integers(0, 0x7f7fffff, 4000).tolist()
    bits = np.array([b | sign for b in bits for sign in (0, 0x80000000)], np.uint32)
    x = bits.view(np.float32)
    out = subprocess.run([exe], input=" ".join(map(str, bits)), capture_output=True, text=True, timeout=20, check=True).stdout
    out = np.array(out.split(), np.uint64).reshape(-1, 4)
    key, near = out[:, 0], out[:, 1:].astype(np.uint32).view(np.float32)
    order = np.argsort(x, kind="stable")
    assert np.array_equal(np.diff(x[order]) > 0, np.diff(key[order].astype(np.int64)) > 0)
    assert np.array_equal(near[:, 1], x)                         # (-0 comes back as +0, which is equal)
    inf = np.float32(np.inf)
    with np.errstate(over="ignore"):
        assert np.array_equal(near[:, 0], np.nextafter(x, -inf)) and np.array_equal(near[:, 2], np.nextafter(x, inf))
