"""What the reference keeps of gates far out, held to what it is defined by (CPU)."""
import numpy as np

from oracle import gated as G


def test_kept_gates_far_out():
    r = np.random.default_rng(3)
    x, ga, gi = (r.normal(size=(70, 3)) for _ in range(3))
    plain = G.kept(x, ga, gi, 70)
    ga[3, 0], ga[40, 1], gi[5, 0], gi[6, 0], gi[41, 2] = np.inf, -np.inf, np.inf, -np.inf, -np.inf
    ga[4, 0], gi[40, 0], gi[42, 2], gi[43, 0], gi[44, 0] = 100.0, -3e38, -89.0, -100.0, 80.0
    gi[45, 0] = -80.0
    kx, ka, ki = G.kept(x, ga, gi, 70)
    assert ka[3, 0] == ka[4, 0] == ki[5, 0] == 31.75  # the largest codes of their blocks
    # -80 does shut a gate, but not to 0: its block has whole numbers
    assert ki[45, 0] == -80 and ki[44, 0] == 80 and ki[43, 0] == -100 and ki[40, 0] == -np.inf
    assert ka[40, 1] == -np.inf and kx[40, 1] == 0 and ki[40, 1] == 0
    assert ki[6, 0] == ki[41, 2] == ki[42, 2] == -np.inf
    # the neighbours of an input gate's -inf are kept as they are without it
    rest = (np.arange(70) != 41) & (np.arange(70) != 42)
    assert np.array_equal(ki[rest, 2], plain[2][rest, 2])
    assert np.abs(ki[7:32, 0] - gi[7:32, 0]).max() <= 0.125  # half a step of the block that reaches 31.75
    with np.errstate(over="ignore"):
        assert np.float32(1) / (np.float32(1) + np.exp(-np.float32(G.OPEN))) == 1
        assert np.float32(1) / (np.float32(1) + np.exp(-np.float32(G.SHUT))) == 0
