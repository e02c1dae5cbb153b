"""What a network takes of a router: logits, bias and the rows that take part.  No GPU involved: what reaches the choice is looked at."""
import numpy as np
import pytest
import torch

from paper_2302_06361_amd import network


class Recorder:
    """stands in for the context: keeps what a choice is made from"""
    device = torch.device("cpu")

    def choose(self, router, logits, valid=None, out=None):
        self.router, self.logits, self.valid = router, logits, valid
        return out


def routed(**router):
    ctx = Recorder()
    network._Routed(dict(dict(logits=np.zeros((6, 4)), top_k=2), **router), 2, ctx, 3, "experts").part(2, 3)
    return ctx


@pytest.mark.parametrize("values", [[0, 1, 2, 0, 255, 0], [0, 256, 512, 0, -256, 0], [0, 2 ** 40, 1, 0, -1, 0], [0.0, 0.25, 1e-30, 0.0, -0.5, 0.0], [False, True, True, False, True, False]])
def test_rows_that_take_part(values):
    """whatever is not zero takes part, of any type"""
    for given in (values, np.array(values)):
        got = routed(valid=given).valid
        assert got.itemsize == 1 and (got != 0).tolist() == [bool(v) for v in values[2:5]]
