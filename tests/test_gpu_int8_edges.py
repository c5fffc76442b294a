"""The 8-bit layer at the ends of its range, and where its kernels' loops run for many turns.

Sums are compared whole: with scales of one an output is its sum, rounded once to float."""
import ctypes

import pytest
import torch

from paper_1501_07338_amd import vcnn
from test_gpu_int8 import call, make


# Many turns of: the ring of 256 x 256 tiles (rows of whole 16 bytes, an odd and an even number of slabs, a ragged last one) and
# the registers of unaligned rows; of 128 x 128 tiles, whole and divided; the unrolled steps of few samples, one to four tiles of
# them, aligned and not; dot products of one and two samples.
MANY_TURNS = [(1000, 1040, 12300), (1000, 1104, 12300), (1000, 1077, 12300), (300, 2064, 1000), (130, 6000, 520), (90, 3001, 700),
              (8, 4096, 130), (16, 6500, 40), (20, 4096, 50), (30, 7001, 33), (40, 3001, 70), (48, 4096, 130), (60, 3000, 500),
              (64, 9000, 35), (100, 7000, 40), (1, 13000, 70), (2, 9000, 70)]


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("batch,k,out", MANY_TURNS)
def test_loops_of_many_turns(batch, k, out, offset):
    x, w, _, _, _ = make(batch + k, batch, k, out)
    one = torch.ones(max(batch, out))
    need = vcnn.fc_i8_workspace_bytes(batch, k, out)
    work = torch.empty(need, dtype=torch.uint8, device="cuda:0") if need else None
    want = (x.double() @ w.double().t()).float()
    assert torch.equal(call(vcnn.F32, vcnn.ACT_NONE, x, w, one[:batch], one[:out], None, work, offset), want)


def test_more_outputs_than_a_grid_is_wide_are_refused():
    """512 threads for sixteen outputs: with 2^27 outputs a launch would have 2^32 threads.  Needs no GPU."""
    lib, need = vcnn.lib(), ctypes.c_size_t()
    f = 0x1000  # never dereferenced: validation fails first
    for batch, out in ((1, 1 << 27), (3, (1 << 26) + 1), (64, 2 ** 31 - 1), (1 << 20, 1 << 20), (2 ** 31 - 1, 256)):
        assert lib.vcnn_fc_i8_workspace_bytes(batch, 8, out, ctypes.byref(need)) == vcnn.ERR_UNSUPPORTED
        assert lib.vcnn_fc_fwd_i8(vcnn.F32, batch, 8, out, 0, f, f, f, f, None, f, None, 0, None) == vcnn.ERR_UNSUPPORTED
        assert "too large" in vcnn.last_error()
    assert vcnn.fc_i8_workspace_bytes(3, 8, 1 << 26) == 0 == vcnn.fc_i8_workspace_bytes(2 ** 30, 8, 256)
