"""The hardware's cosine and sine, on which the codes of rotated rows rest, over all phases there are."""
import pytest

pytestmark = pytest.mark.gpu


def test_cosine_and_sine_of_every_phase():
    """tri_append4 and tri_pack4 work out in double precision what lies within 2^-20 of a pair's larger rotated element of a border.  For |re| + |im|, at most twice that element, a rotated one may then be off by
    (|re| + |im|) 2^-21.  Two roundings take 2^-23 of it at most, the angle 5e-9: the rest is cosine's and sine's."""
    from workload import device
    cosine, sine = device.turn_error()
    print("off by %.3g and %.3g" % (cosine, sine))
    assert 0 < cosine < 2.0 ** -21 - 2.0 ** -23 - 5e-9 and 0 < sine < 2.0 ** -21 - 2.0 ** -23 - 5e-9
