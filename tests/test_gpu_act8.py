"""Activations in 8 bits on the GPU against the definition in 64 bits: every value has to be the same."""
import numpy as np
import pytest
import torch

import paper_2206_10620_amd as pp
from adapter_util import held8

pytestmark = pytest.mark.gpu
DT = {"f16": np.float16, "f32": np.float32}


def round_trip(x):
    print("case", x.shape, x.dtype, flush=True)
    held = pp.act8_pack(torch.from_numpy(x).cuda())
    return held, held.unpack().cpu().numpy()


@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (17, 127), (16, 128), (5, 129), (33, 300), (2, 4099), (300, 1)], ids=str)
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_values(dtype, shape):
    rs = np.random.RandomState(shape[0] + shape[1])
    x = (rs.standard_normal(shape) * np.exp2(rs.randint(-12, 12, (shape[0], 1)))).astype(DT[dtype])
    x[rs.random_sample(shape) < 0.3] = 0
    held, got = round_trip(x)
    want = held8(x).astype(DT[dtype])
    assert np.array_equal(got, want)
    assert np.array_equal(got > 0, x > 0) and np.array_equal(got < 0, x < 0)          # no sign is lost
    # the other storage type reads the same values
    other = held.unpack(pp.PP_F32 if dtype == "f16" else pp.PP_F16).cpu().numpy()
    assert np.array_equal(other, held8(x).astype(other.dtype))


def test_borders():
    """Ties, the step from 127 to the next power of two, the smallest and largest numbers."""
    for dtype in (np.float16, np.float32):
        rows = [[127, 63.5, 64.5, 0.5, 1.5, -2.5], [127.0625 if dtype == np.float16 else 127.00001, 1, 3, 5, -1, -3], [254, 1, 3, 125, -253, 0], [0, 0, 0, -0.0, 0, 0],
                [np.finfo(dtype).tiny, 1e-7, -6e-8, 0, 0, 0], [np.finfo(dtype).smallest_subnormal, 0, 0, 0, 0, 0], [65024, -65024, 512, 1, 0, 0]]
        x = np.array(rows, dtype)
        assert np.array_equal(round_trip(x)[1], held8(x).astype(dtype))
    x = np.array([[3.3e38, -1e38, 1.0], [1e-44, -1.2e-38, 0]], np.float32)
    assert np.array_equal(round_trip(x)[1], held8(x).astype(np.float32))
    # values that only 8 bits round above binary16's largest come back as that
    x = np.array([[65504, -65504, 100]], np.float16)
    held, got = round_trip(x)
    largest = np.finfo(np.float32).max
    assert round_trip(np.array([[largest, -largest, 0]], np.float32))[1].tolist() == [[largest, -largest, 0]]
    assert got.tolist() == [[65504, -65504, 1024]] and held.unpack(pp.PP_F32).cpu().tolist() == [[65536, -65536, 1024]]


def test_infinities_and_nan_stay_in_their_block():
    for dtype in (np.float16, np.float32):
        x = np.ones((3, 400), dtype)
        x[0, 5], x[1, 200], x[2, 399] = np.inf, np.nan, -np.inf
        x[0, 300] = -2
        got = round_trip(x)[1]
        assert np.array_equal(got, held8(x).astype(dtype), equal_nan=True)


def test_nothing_is_written_behind_the_ends():
    rows, n = 5, 131
    x = torch.randn((rows, n), dtype=torch.float16, device="cuda")
    size = pp.pp_act8_bytes(rows, n)
    buf = torch.full((size + 256,), 77, dtype=torch.uint8, device="cuda")
    out = torch.full((rows * n + 64,), 7.0, dtype=torch.float16, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    assert pp.pp_act8_pack(x.data_ptr(), rows, n, pp.PP_F16, buf.data_ptr(), s) == pp.PP_OK
    assert pp.pp_act8_unpack(buf.data_ptr(), rows, n, pp.PP_F16, out.data_ptr(), s) == pp.PP_OK
    assert bool((buf[size:] == 77).all()) and bool((out[rows * n:] == 7.0).all())
    assert bool((buf[: rows * 256].view(rows, 256)[:, n:] == 0).all())                 # zeros behind a row


def test_on_a_stream_of_its_own():
    x = torch.randn((64, 1000), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = pp.act8_pack(x, stream=stream.cuda_stream).unpack(stream=stream.cuda_stream)
    stream.synchronize()
    assert np.array_equal(got.cpu().numpy(), held8(x.cpu().numpy()).astype(np.float32))


def test_offsets_beyond_32_bits():
    """2^31 - 256 values in rows of 4 MB and in one row; the ends are looked at."""
    for rows, n in ((1 << 10, (1 << 21) - 1), (1, (1 << 31) - 256)):
        print("case", rows, n, flush=True)
        x = torch.zeros((rows, n), dtype=torch.float16, device="cuda")
        x[-1, -300:] = torch.arange(300, device="cuda").half() - 150
        x[0, :300] = torch.arange(300, device="cuda").half() - 150
        got = pp.act8_pack(x).unpack()
        for r, part in ((0, slice(0, 640)), (rows - 1, slice(n - 640 - n % 128, n))):
            assert np.array_equal(got[r, part].cpu().numpy(), held8(x[r: r + 1, part].cpu().numpy()).astype(np.float16)[0])
        assert int((got != 0).sum()) == int((x != 0).sum())
        del x, got
