"""The ramp of PURO_ROPE_INDEX where its slow end lies past the last pair (no GPU).  The published rule takes the ends as indexes among all
rot_dim channels, at most rot_dim - 1, so such a ramp leaves the last pairs partly kept."""
import math

import pytest

import paper_2608_27370_gb300 as P
from paper_2608_27370_gb300 import _build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    _build.build()


def ends(rot, base, trained, fast, slow):
    """By counting: turns fall with the index, so the fast end, rounded down, is the last index with at least `fast` turns, and the slow
    end, rounded up, the first with at most `slow`."""
    turns = [trained * base ** (-2 * i / rot) / (2 * math.pi) for i in range(rot)]
    return max([0] + [i for i in range(rot) if turns[i] >= fast]), min([i for i in range(rot) if turns[i] <= slow] + [rot - 1])


def frequencies(rot, base, factor, lo, hi):
    keep = [min(1.0, max(0.0, (hi - i) / max(hi - lo, 0.001))) for i in range(rot // 2)]
    return [(k + (1 - k) / factor) * base ** (-2 * i / rot) for i, k in enumerate(keep)]


# The ends worked out by hand: rot ln(trained / (2 pi turns)) / (2 ln base); of rot 128, base 10^4 and 131072: 64 x 6.4799 / 9.2103 = 45.03 and
# 64 x 9.9456 / 9.2103 = 69.11, so pair 63 is kept by (70 - 63) / (70 - 45).  Of rot 16 and 2^30
# the slow end is 16.5, past every channel: 15.
CASES = [(128, 1e4, 8.0, 65536, 40, 65), (128, 1e4, 8.0, 131072, 45, 70), (64, 1e4, 8.0, 131072, 22, 35), (16, 1e4, 4.0, 1 << 30, 13, 15),
         (128, 1e6, 4.0, 32768, 23, 40), (256, 5e5, 2.0, 8192, 36, 70)]


@pytest.mark.parametrize("rot,base,factor,trained,lo,hi", CASES)
def test_the_ends_are_channels_not_pairs(rot, base, factor, trained, lo, hi):
    assert ends(rot, base, trained, 32.0, 1.0) == (lo, hi)
    got = P.rope_frequencies(rot, base, P.ROPE_INDEX, factor, trained, 32.0, 1.0, device="cpu")
    for g, w in zip(got.tolist(), frequencies(rot, base, factor, lo, hi)):
        # as in the definitions' test: pow's argument and result, the ramp, and one unit
        assert abs(g / 2 ** 64 - w / (2 * math.pi)) <= 2 ** -47 * w / (2 * math.pi) + 2 ** -64


def test_the_last_pair_is_partly_kept():
    plain = P.rope_frequencies(128, 1e4, device="cpu")
    for trained, keep in ((65536, 2 / 25), (131072, 7 / 25)):
        last = int(P.rope_frequencies(128, 1e4, P.ROPE_INDEX, 8.0, trained, device="cpu")[-1])
        assert abs(last / int(plain[-1]) - (keep + (1 - keep) / 8)) <= 1e-9
