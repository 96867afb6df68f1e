"""More of what the extension's entry points and their binding refuse (no GPU needed)."""
import pytest

from paper_2609_38198_amd import _lib as fd


def test_adamw_refuses_an_unknown_rounding():
    lib = fd.load()
    t = fd.AdamwTensor(p=256, g=256, m=256, v=256, m_scale=256, v_scale=256, n=4, gt=0, decay=1.0)
    for bits in (32, 8):
        o = fd.AdamwOpts(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1,
                         state_bits=bits, rounding=2)
        assert lib.fd_adamw_step(t, 1, o, None) == 1
        assert b"rounding" in lib.fd_last_error()
    lib.fd_adamw_default_opts(o)
    assert o.rounding == fd.FD_ROUNDING["nearest"] == 0
    with pytest.raises(ValueError):
        fd.fd_adamw_step(None, 1, rounding="up")
