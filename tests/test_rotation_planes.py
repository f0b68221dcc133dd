"""Position planes that are one plane, broadcast: host checks."""
import torch

import paper_2502_11494_amd as D
from paper_2502_11494_amd import binding

from test_attend_host import FAKE, append, cache, rotate, rotation


def test_strides_of_planes():
    three = rotation(planes=3, sections=[16, 24, 24])
    # a stride of 0 is accepted (what is refused here is the address behind it)
    assert rotate(three, plane=0, q=FAKE + 4) == D.DART_ERR_ALIGN and append(three, cache(), plane=0, q=FAKE + 4) == D.DART_ERR_ALIGN
    for plane in (1, 4, -1, -5):
        assert rotate(three, plane=plane) == D.DART_ERR_SHAPE and append(three, cache(), plane=plane) == D.DART_ERR_SHAPE


def test_the_binding_takes_expanded_planes():
    pos = torch.arange(7)
    assert binding._planes(pos.expand(3, -1), 3, 7) == (pos.data_ptr(), 0)
    assert binding._planes(pos.expand(3, -1).contiguous(), 3, 7)[1] == 7
    assert binding._planes(pos[2:3].expand(3, -1), 3, 1) == (pos[2:].data_ptr(), 0)
    assert binding._planes(pos, 1, 7) == (pos.data_ptr(), 0)
