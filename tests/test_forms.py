"""CPU checks that the GPU tests' sizes still take the kernel forms that they are
there for: the rules that choose them run on the host."""
import math
import random

from attend_forms import MANY_BLOCKS, THREE_TILES, plan
from linear_forms import CASES, form
from paper_2506_01979_amd import synth


def test_linear_cases_take_every_form():
    """Every form that the models' projections take at 1 .. 256 rows, and that 30000
    other sizes take, is one of a case's."""
    sizes = set()
    for s in synth.SHAPES.values():
        qd, kv = s.n_heads * s.head_dim, s.n_kv_heads * s.head_dim
        for m, k in ((qd + 2 * kv, s.hidden), (s.hidden, qd), (2 * s.ffn, s.hidden), (s.hidden, s.ffn), (s.vocab, s.hidden)):
            sizes.update((m, k, n) for n in range(1, 257))
    rng = random.Random(0)
    for _ in range(30000):
        m, k = (int(round(math.exp(rng.uniform(0, math.log(most))))) for most in (300000, 32768))
        sizes.add((m, k, rng.randint(1, 256)))
    taken = {}
    for c in sizes:
        taken.setdefault(form(*c), c)
    tested = {form(m, k, n) for m, k, ns in CASES for n in ns}
    assert len(tested) > 80
    assert not set(taken) - tested, {f: taken[f] for f in set(taken) - tested}


def test_attend_cases_take_their_forms():
    assert all(plan(*c)[0] == 3 for c in THREE_TILES)
    rows = [c[5] * (c[0] // c[1]) for c in THREE_TILES]
    assert {-(-r // 16) % 3 for r in rows} == {0, 2}             # whole and ragged row blocks
    assert {c[2] for c in THREE_TILES} == {64, 128}
    assert {plan(*c)[0] for c in MANY_BLOCKS} == {1, 2, 3}
    assert all(c[3] / (4 * plan(*c)[2]) > 64 for c in MANY_BLOCKS)
