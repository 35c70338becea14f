"""A token shift of rwkvq_lowrank has a description and an image, or neither."""
from tests.test_lowrank_host import EINVAL, MU, P, status


def test_a_description_without_an_image_is_refused():
    assert status(mu=MU) == EINVAL
    assert status(image=P) == EINVAL
    assert status(mu=MU, tokens=0, x=0, y=0) == EINVAL
