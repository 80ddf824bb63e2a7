"""Activations in 8 bits at the largest sizes that are accepted."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import held8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 127, 2 ** 31 - 128])
def test_rows_up_to_the_last_value(n):
    """One row of nearly 2^31 values, whose length rounded up to whole blocks passes 31 bits; its ends are looked at."""
    print("case", n, flush=True)
    x = torch.zeros((1, n), dtype=torch.float16, device="cuda")
    ends = torch.arange(300, device="cuda").half() - 150
    x[0, :300], x[0, -300:] = ends, ends
    got = pp.act8_pack(x).unpack()
    for part in (slice(0, 640), slice(n - 640 - n % 128, n)):
        assert np.array_equal(got[0, part].cpu().numpy(), held8(x[:, part].cpu().numpy()).astype(np.float16)[0])
    assert int((got != 0).sum()) == int((x != 0).sum())


def test_more_rows_than_a_launch_has_units():
    rows = (1 << 24) + 5
    x = torch.zeros((rows, 1), dtype=torch.float32, device="cuda")
    x[:100, 0], x[-100:, 0] = torch.arange(100, device="cuda") - 50.0, torch.arange(100, device="cuda") - 50.0
    got = pp.act8_pack(x).unpack()
    assert torch.equal(got, x)                       # a block of one value that is a whole number of seven bits is held as it is
