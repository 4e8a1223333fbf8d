"""Numbers that do not fit the library's 32-bit arguments are refused, not cut (no GPU needed: arguments are read before the call)."""
import pytest

from paper_2512_10310_b200 import binding as B

GATHER = B.gather_params("bf16", 4, 128, 16, 8, 1e6)


@pytest.mark.parametrize("number", [2 ** 31, 2 ** 32 + 4, -2 ** 31 - 1])
def test_numbers_beyond_32_bits(number):
    for at in range(4):
        counts = [number if i == at else 4 for i in range(4)]
        with pytest.raises(OverflowError):
            B.evlnSelectKeys(None, GATHER, None, *counts, None, stream=0)
    with pytest.raises(OverflowError):
        B.evlnGatherKeys(None, GATHER, number, None, None, None, None, None, None, None, stream=0)
    paged = B.paged_params(28, 4, 128, 1, 64, 4, 2, 1e6)
    with pytest.raises(OverflowError):
        B.evlnPaged8RopeAppend(None, paged, None, *[None] * 3, [number], [0, 1], *[None] * 6, stream=0, strides=(1, 1, 1))


def test_numbers_that_fit_go_through():
    for call in (lambda: B.evlnSelectKeys(None, GATHER, None, 2 ** 31 - 1, -2 ** 31, 0, 0, None, stream=0),
                 lambda: B.evlnGatherKeys(None, GATHER, 4, None, None, None, None, None, None, None, stream=0)):
        with pytest.raises(B.EvlnError) as e:
            call()
        assert e.value.status == B.EVLN_INVALID_VALUE
