"""The 8-bit forms of the AdamW states in the tests' oracle, at ties and ends."""
import torch

from tests import train_ref as ref


def test_ties_go_to_even_codes():
    m = torch.zeros(128, dtype=torch.float64)
    u = torch.zeros(128, dtype=torch.float64)
    m[0], u[0] = 448.0, 1.9375                             # scales of one
    # half-way between neighbours 1, 1.125 and 1.125, 1.25 of E4M3, and 1, 1.0625 and 1.0625, 1.125 of the other
    m[1], m[2], m[3] = 1.0625, -1.1875, 2.0 ** -10
    u[1], u[2], u[3] = 1.03125, 1.09375, 1e-30
    mc, sm, uc, su = ref.hold(m, u)
    assert sm.tolist() == [1.0] and su.tolist() == [1.0]
    assert mc[:4].tolist() == [0x7E, 0x38, 0x80 | 0x3A, 0x00]
    assert uc[:5].tolist() == [255, 0x7F0 - 0x700, 0x7F2 - 0x700, 1, 0]
    vm, vv, vu = ref.values(mc, sm, uc, su)
    assert vm[:4].tolist() == [448.0, 1.0, -1.25, 0.0] and vu[:3].tolist() == [1.9375, 1.0, 1.125]


def test_values_of_all_codes():
    assert len(ref.E4M3) == 127 and float(ref.E4M3[-1]) == 448.0 and float(ref.E4M3[1]) == 2.0 ** -9
    assert len(ref.Q) == 256 and float(ref.Q[255]) == 1.9375 and float(ref.Q[1]) == 1.0625 * 2.0 ** -15
    c = torch.arange(1, 256, dtype=torch.int32)
    assert torch.equal(((c + 1792) << 19).view(torch.float32).double(), ref.Q[1:])
