"""What the sampling kernel rests on and no call shows.  The last step of sampling looks for one token of the chosen value and goes to the place where it found it: the value has to have one.
The choice inside a block is restated here, with what the source does where no value of the block has weight.  Needs no GPU."""
import os
import re
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest

from paper_2410_11305_amd import build

SOURCE = re.sub(r"//.*", "", open(os.path.join(build.HERE, "csrc", "sample.hpp")).read())
DRAW = SOURCE[SOURCE.index("const double target = u * kept_mass;"):]


def choose(values, target, top):
    """values: (key, tokens, weight, mass up to it) of a block, the largest first; the key that is looked for."""
    hit = [i for i, (_, n, _, upto) in enumerate(values) if n and upto > target]
    have = [i for i, (_, n, weight, _) in enumerate(values) if n and weight > 0]
    at = hit[0] if hit else have[-1] if have else 0
    guarded = re.search(r"const uint32_t key = some \? [^;]* : top;", DRAW) and "const bool some = (hit | have) != 0;" in DRAW
    return top if guarded and not (hit or have) else values[at][0]


@pytest.mark.parametrize("tokens,weight", [(0, 0.0), (5, 0.0), (5, 5e-324)])
def test_the_chosen_value_has_a_token(tokens, weight):
    """A block that the target falls into by the rounding of the sums in front of it, its own mass too small to change them."""
    top = 0xC000
    block = [(0x9000 - i, tokens if i == 40 else 0, weight if i == 40 else 0.0, 1.5) for i in range(64)]
    present = {top} | {key for key, n, _, _ in block if n}
    assert choose(block, 1.5, top) in present


def test_the_choice_is_the_sources():
    assert "const int at = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(have | 1ull);" in DRAW
    assert "ballot_w64(x.n && x.upto > target), have = __builtin_amdgcn_ballot_w64(x.n && x.weight > 0.0);" in DRAW


def test_the_two_parts_of_ln_2():
    """The first has few enough bits for an exact product with any exponent; both together are ln 2 to 2^-93."""
    getcontext().prec = 50
    whole, rest = (Fraction(float.fromhex(x)) for x in re.search(r"ln2 = ([^,]*), ln2_rest = ([^;]*);", SOURCE).groups())
    assert (whole * 2 ** 40).denominator == 1 and 800 / 0.693 < 2 ** 11
    assert abs(whole + rest - Fraction(Decimal(2).ln())) < Fraction(1, 2 ** 93)
