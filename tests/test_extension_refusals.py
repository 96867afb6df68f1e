"""More of what the extension's entry points and their binding refuse (no GPU needed)."""
import numpy as np
import pytest
import torch

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


class Elsewhere:
    """Looks like a torch tensor on GPU `dev` (-1: in host memory) to the binding, which
    refuses it before it would use its address."""

    def __init__(self, *shape, dtype=torch.float32, dev=0, strides=None):
        self.shape, self.dtype, self.dev = tuple(shape), dtype, dev
        self.strides = strides or tuple(int(np.prod(shape[i + 1:])) for i in range(len(shape)))

    is_cuda = property(lambda self: self.dev >= 0)
    device = property(lambda self: torch.device("cuda", self.dev) if self.dev >= 0 else torch.device("cpu"))

    def get_device(self):
        return self.dev

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self.strides == Elsewhere(*self.shape).strides

    def data_ptr(self):
        raise AssertionError("the address of a tensor that had to be refused")

    def new_empty(self, shape, dtype=None):
        return type(self)(*(shape if isinstance(shape, (tuple, list)) else (shape,)),
                          dtype=dtype or self.dtype, dev=self.dev)


class Here(Elsewhere):
    def data_ptr(self):
        return 256


@pytest.mark.parametrize("dev", [-1, 1])
def test_binding_refuses_tensors_of_another_device(dev):
    x, w, wd, v = Here(4, 8), Here(16, 8), Here(8, 16), Here(8)
    ms = Here(4, 2)

    def away(*shape, dtype=torch.float32):
        return Elsewhere(*shape, dtype=dtype, dev=dev)

    room = away(1 << 24, dtype=torch.uint8)
    apart = Elsewhere(1 << 12, 64, dtype=torch.uint8, strides=(128, 1))
    calls = [lambda: fd.fd_layer_norm(x, away(8)), lambda: fd.fd_layer_norm(x, v, away(8)),
             lambda: fd.fd_layer_norm(x, Y=away(4, 8)), lambda: fd.fd_layer_norm(x, stats=away(4, 2)),
             lambda: fd.fd_layer_norm_backward(x, x, v, away(4, 2)),
             lambda: fd.fd_layer_norm_backward(away(4, 8), x, v, ms),
             lambda: fd.fd_layer_norm_backward(x, x, v, ms, ws=room),
             lambda: fd.fd_layer_norm_backward(x, x, v, ms, dgamma=away(8)),
             lambda: fd.fd_gated_forward(x, w, away(16, 8), wd),
             lambda: fd.fd_gated_forward(x, w, w, wd, R=away(4, 8)),
             lambda: fd.fd_gated_forward(x, w, w, wd, ws=room),
             lambda: fd.fd_gated_forward(x, w, w, wd, ws=apart),
             lambda: fd.fd_gated_backward(x, x, w, w, wd, saved=room),
             lambda: fd.fd_gated_backward(x, x, w, w, wd, saved=apart),
             lambda: fd.fd_gated_backward(x, x, w, w, wd, ws=room),
             lambda: fd.fd_kernel_matmul(x, None, 1.0, Here(4, 2), ws=room),
             lambda: fd.fd_kernel_matmul(x, None, 1.0, away(4, 2)),
             lambda: fd.fd_degree(x, 1.0, ws=room)]
    state = fd.AdamwState([Here(8)], [Here(8)])
    calls += [lambda: fd.fd_adamw_plan([v], [away(8)], state),
              lambda: fd.fd_adamw_plan([v], [v], fd.AdamwState([away(8)], [v])),
              lambda: fd.fd_adamw_plan([v, away(8)], [v, v], fd.AdamwState([v, v], [v, v]))]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="GPU|contiguous"):
            call()
            raise AssertionError(f"call {i} was taken")


def test_more_than_a_launch_holds_is_refused():
    # 2^32 threads: beyond, a launch would run the rest alone and report nothing
    lib = fd.load()
    b = fd.GatedBlock(N=1 << 30, D=72, F=1024, O=72, type=1, act=0, X=256, Wg=256, Wu=256, Wd=256,
                      ldx=72, ldwi=72, ldwd=1024)
    assert lib.fd_gated_forward(b, None, 0, 256, 72, None, 0, 256, 1 << 62, None) == 2
    assert b"launch" in lib.fd_last_error()
    t = fd.AdamwTensor(p=256, g=256, m=256, v=256, n=(1 << 35) + 1, gt=0, decay=1.0)
    assert lib.fd_adamw_step(t, 1, None, None) == 1


def test_assembly_names_the_registers_that_it_writes():
    # a statement that writes M0 without saying so is right until the compiler keeps something there
    import glob
    import os
    import re

    csrc = os.path.join(os.path.dirname(fd.__file__), "csrc")
    found = 0
    for path in glob.glob(os.path.join(csrc, "*.h*")):
        for text in re.findall(r"asm volatile\((.*?)\);", open(path).read(), re.S):
            if re.search(r"\bm0,", text.split(":")[0]):
                found += 1
                assert '"m0"' in text.split(":")[-1], path
    assert found


def test_layer_norm_gradients_types():
    x, v, ms = Here(4, 8, dtype=torch.bfloat16), Here(8, dtype=torch.float32), Here(4, 2)
    half = Here(8, dtype=torch.float16)
    for kw in (dict(gamma=v, dbeta=Here(8, dtype=torch.bfloat16)), dict(gamma=v, wdtype=torch.bfloat16),
               dict(gamma=None, dgamma=v, dbeta=Here(8, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            fd.fd_layer_norm_backward(x, x, stats=ms, **kw)
    for kw in (dict(gamma=half), dict(gamma=None, dbeta=half), dict(gamma=None, wdtype=torch.float64)):
        with pytest.raises(TypeError):
            fd.fd_layer_norm_backward(x, x, stats=ms, **kw)


def test_fine_flag_and_unknown_activations():
    lib = fd.load()
    kw = dict(N=5003, D=509, F=1365, O=509, type=1, X=256, Wg=256, Wu=256, Wd=256, ldx=509, ldwi=509,
              ldwd=1365)
    coarse, fine = fd.GatedBlock(act=1, **kw), fd.GatedBlock(act=1 | fd.FD_GATED_FINE, **kw)
    for backward in (0, 1, 2):
        assert lib.fd_gated_workspace_size(fine, backward) > lib.fd_gated_workspace_size(coarse, backward) > 0
    for act in (2, fd.FD_GATED_FINE | 2, 0x200, -1):
        b = fd.GatedBlock(act=act, **kw)
        assert lib.fd_gated_forward(b, None, 0, 256, 509, None, 0, 256, 1 << 40, None) == 1, act
