"""Rules of the norms and products that the kernels share with the host, compiled from the library's own headers."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    """A program that reads one question per line and answers it."""
    from paper_2211_00839_b200 import build
    out = str(tmp_path_factory.mktemp("rules") / "rules")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(os.path.dirname(os.path.dirname(build._nvcc())), "include"),
                    "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, os.path.join(ROOT, "tests", "operator_rules.cpp"), "-o", out], check=True)

    def ask(questions):
        text = "\n".join(" ".join(map(str, q)) for q in questions) + "\n"
        answers = subprocess.run([out], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(answers) == len(questions)
        return [tuple(map(int, a.split())) for a in answers]
    return ask


def test_a_ring_orders_no_copy_twice_in_a_phase(rules):
    """Copies that arrive in time, later than the wait for them, or never: no barrier takes a second order before its phase is over."""
    rng = random.Random(3)
    questions = []
    for _ in range(4000):
        stages, rows = rng.randint(1, 4), rng.randint(1, 40)
        late = [rng.choice([0, 0, 0, 0, 1, 2, 5, 10 ** 6]) if rng.random() < 0.3 else 0 for _ in range(rows)]
        questions.append(("ring", stages, rows, *late))
    for (_, stages, rows, *late), (twice, in_time) in zip(questions, rules(questions)):
        assert not twice, (stages, late)
        first = next((k for k, l in enumerate(late) if l > (stages - 1 if k >= stages else k)), rows)
        if first == rows:
            assert in_time == rows


def test_arguments_that_share_a_byte(rules):
    """Against the sets of bytes: what shares one is always found; column slices of one buffer that do not are told apart."""
    rng = random.Random(4)
    questions = []
    for _ in range(20000):
        pitch = rng.choice([1, 2, 4]) * rng.randint(1, 12)
        both = []
        for _ in range(2):
            size = rng.choice([s for s in (1, 2, 4) if pitch % s == 0])
            ld = pitch // size if rng.random() < 0.8 else rng.randint(1, 12)
            both += [size * rng.randint(20, 60), rng.randint(0, 5), ld, rng.randint(0, ld), size]
        questions.append(("meet", *both))
    bytes_of = lambda at, rows, ld, n, size: {at + r * ld * size + k for r in range(rows) for k in range(n * size)}  # noqa: E731
    apart = 0
    for (_, *q), (meet,) in zip(questions, rules(questions)):
        a, b = bytes_of(*q[:5]), bytes_of(*q[5:])
        if a & b:
            assert meet, q
        elif q[2] * q[4] == q[7] * q[9] and a and b:
            inside = max(min(a), min(b)) <= min(max(a), max(b))
            # (within the first or behind the last row of the other, columns may be shared by rows that are not there)
            columns = {x % (q[2] * q[4]) for x in a} & {x % (q[2] * q[4]) for x in b}
            assert bool(meet) <= bool(columns), q
            apart += inside and not meet
        elif not a or not b:
            assert not meet, q
    assert apart > 200
