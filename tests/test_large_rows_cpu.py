"""Sizes past what 32-bit indices hold: refused, or sized in 64 bits, before anything is launched (no GPU needed)."""
import pytest


@pytest.fixture(scope="module")
def E():
    from paper_2510_27258_gb300 import build, hla
    build.build()
    return hla


def test_conv_channels(E):
    L, top = E.lib(), (1 << 31) - 1
    # B = 0: nothing is launched where the arguments are taken
    forward = lambda C: L.hla_conv_forward(256, 256, 256, 256, 1, 0, 1, C, 4, C, C, 1, None, None, None, None)  # noqa: E731
    for C in (430_000_000, top - 256):
        assert forward(C) == E.HLA_OK
        assert L.hla_conv_backward_workspace_bytes(1, 1, C, 4, 1) >= 4 * 5 * C
    for C in (top - 200, top):
        assert forward(C) == E.HLA_ERR_UNSUPPORTED
        assert L.hla_conv_backward_workspace_bytes(1, 1, C, 4, 1) == 0
