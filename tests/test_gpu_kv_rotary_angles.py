"""The angle by which the append rotates, seen where a sine or cosine is next to zero: the pair (1, 0) becomes (cos, sin).

Bound: the angle's 2^-33 turns, half a step of bf16 (2^-8 of the value) and 2^-21 of it for what fp32 adds."""
import fractions
import math

import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup

pytestmark = pytest.mark.gpu

# 2 pi to 10^-60: 60 digits reduce positions under 2^31 times frequencies under 2^3 turns to 10^-49 turns
PI2 = fractions.Fraction(6283185307179586476925286766559005768394338798750211641949889, 10 ** 60)


def expected(turns):
    """Cosine and sine of an exact number of turns: the nearest quarter turn comes off first."""
    k = round(4 * turns)
    x = 2 * math.pi * float(turns - fractions.Fraction(k, 4))
    c, s = math.cos(x), math.sin(x)
    return ((c, s), (-s, c), (-c, -s), (s, -c))[k % 4]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("position", [1, -1, 3, -4099, 1 << 20, (1 << 31) - 1, -(1 << 31)])
def test_angles_next_to_quarter_turns(position, interleaved):
    import torch
    import paper_2608_23805_amd as msi
    log(f"case rotary angles position={position} interleaved={interleaved}")
    rest = [0.99, -0.99, 1.5, 2.96, -7.01, 64.9, 1e4 + 0.9, -3e6 - 0.97]                # 2^-32 turns past a quarter turn
    freq = [float((fractions.Fraction(k, 4) + fractions.Fraction(r) / 2 ** 32) * PI2 / position) for k in range(4) for r in rest]
    rot = 2 * len(freq)
    s = Setup(980, [1], [1], 1, rot, "e4m3")
    q = torch.zeros((1, 1, rot), dtype=torch.bfloat16, device="cuda")
    one = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
    two = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
    q[..., one] = 1.0
    out = torch.empty_like(q)
    kv = torch.zeros((1, 1, rot), dtype=torch.bfloat16, device="cuda")
    msi.kv_append_rotary(s.cache, s.seqs, msi.KvRotary(freq, interleaved=interleaved),
                         torch.tensor([position], dtype=torch.int32, device="cuda"), q, out, kv, kv)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()[0, 0]
    want = np.array([expected(position * fractions.Fraction(f) / PI2) for f in freq])
    for g, w in ((got[one], want[:, 0]), (got[two], want[:, 1])):
        assert np.all(np.abs(g - w) <= 2 * math.pi * 2.0 ** -33 + (2.0 ** -8 + 2.0 ** -21) * np.abs(w)), (g, w)
