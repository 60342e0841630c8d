"""What the dense attention entry points refuse where an option is in its range by
itself and not beside another (no GPU needed)."""
import pytest

from test_dense_abi import BAD, WS, call, dims, opts


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("scale,cap,want", [
    (1e-10, 1e30, BAD), (1e-30, 1e30, BAD), (1e-30, 1e9, BAD),
    (0.125, 1e30, WS), (1e-7, 1e30, WS), (1e-30, 1e7, WS), (1e-30, 0.0, WS), (2.0 ** 20, 1e-30, WS)])
def test_a_cap_beyond_what_scale_over_cap_holds(scale, cap, want, backward):
    # scale / softcap below the smallest normal float would lose its digits, or be 0
    # and every score with it (WS: everything but the workspace was right)
    m = dims(Nq=3, Nk=5000)
    assert call(m=m, o=opts(scale=scale, softcap=cap), backward=backward, ws_bytes=8) == want
