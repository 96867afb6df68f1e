"""The example as a user runs it: coordinates from the eigensolver, a network trained on them,
and its distance from the Nystrom extension at new points."""
import os
import sys

import pytest

from gpu_util import case

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


# A network that has learnt nothing is a distance of one away.  Coordinates of this torus are
# cosines and sines of its angles, linear in the points: float32 leaves 5% far behind; bfloat16
# rounds points, activations of four layers and the coordinates (2^-8 each).
@pytest.mark.parametrize("dtype, bits, far", [("f32", 32, 0.05), ("bf16", 8, 0.1)])
def test_network_replaces_the_nystrom_extension(monkeypatch, dtype, bits, far):
    import extension_net

    case(f"example {dtype} {bits}-bit states")
    monkeypatch.setattr(sys, "argv", ["extension_net.py", "--dtype", dtype, "--bits", str(bits),
                                      "--points", "6000", "--steps", "300"])
    assert extension_net.main() <= far
