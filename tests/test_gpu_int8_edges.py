"""The 8-bit layer at the ends of its range."""
import ctypes

from paper_1501_07338_amd import vcnn


def test_more_outputs_than_a_grid_is_wide_are_refused():
    """512 threads for sixteen outputs: with 2^27 outputs a launch would have 2^32 threads.  Needs no GPU."""
    lib, need = vcnn.lib(), ctypes.c_size_t()
    f = 0x1000  # never dereferenced: validation fails first
    for batch, out in ((1, 1 << 27), (3, (1 << 26) + 1), (64, 2 ** 31 - 1), (1 << 20, 1 << 20), (2 ** 31 - 1, 256)):
        assert lib.vcnn_fc_i8_workspace_bytes(batch, 8, out, ctypes.byref(need)) == vcnn.ERR_UNSUPPORTED
        assert lib.vcnn_fc_fwd_i8(vcnn.F32, batch, 8, out, 0, f, f, f, f, None, f, None, 0, None) == vcnn.ERR_UNSUPPORTED
        assert "too large" in vcnn.last_error()
    assert vcnn.fc_i8_workspace_bytes(3, 8, 1 << 26) == 0 == vcnn.fc_i8_workspace_bytes(2 ** 30, 8, 256)
