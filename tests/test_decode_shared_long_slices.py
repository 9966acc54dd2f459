"""Prefixes with more than 32 queries whose slices hold several times the rows that the workgroups' ring of LDS tiles holds (128), so that
stages are used again and again, against fp64.  Inputs, tolerances and comparison are those of test_decode_shared.py."""
import ctypes

import pytest

from test_decode_shared import check

RING_ROWS = 128  # 2 stages of 64 rows, or 4 of 32

# 33 to 64 queries per prefix and head (two waves of columns), and more (four); last column chunks that are not full; lengths that end
# inside a tile, a slice, at a tile's border, and at once
LONG = [
    dict(B=40, Hq=128, Hk=16, T=5, d=64, L=2, P=2000, Np=8, plens=[2000, 1999, 1537, 1, 0, 1000, 704, 1983]),
    dict(B=24, Hq=192, Hk=16, T=3, d=128, L=0, P=1500, Np=8, plens=[1500, 1499, 33, 0, 768, 1121, 385, 1472]),
    dict(B=80, Hq=128, Hk=16, T=5, d=64, L=0, P=1501, Np=4, plens=[1501, 1440, 777, 65]),
    dict(B=36, Hq=256, Hk=16, T=0, d=128, L=1, P=1300, Np=4, plens=[1300, 1299, 673, 31]),
]


@pytest.mark.parametrize("c", LONG)
def test_slices_hold_several_rings(c):
    """The workspace holds (d + 2) floats for every slice's state of every head: so many slices there are at most."""
    from paper_2603_15619_amd.binding import MODAPrefix, MODAShape, lib

    B, Hq, d, P = c["B"], c["Hq"], c["d"], c["P"]
    need = lib().moda_attn_decode_shared_workspace_bytes(ctypes.byref(MODAPrefix(c["Np"], P, P)), 0,
                                                         ctypes.byref(MODAShape(B, Hq, c["Hk"], 0, d, 0, 0, 1, 0.0, 1)))
    slices = need // (4 * (d + 2) * B * Hq) - 1  # (one state is that of the own rows)
    assert B // c["Np"] * (Hq // c["Hk"]) > 32 and slices >= 1 and P / slices >= 2.5 * RING_ROWS


@pytest.mark.gpu
@pytest.mark.parametrize("rising", [False, True])
@pytest.mark.parametrize("c", LONG)
def test_prefixes_of_many_tiles(c, rising):
    """rising: keys grow along the prefix, so that the running maximum rises from tile to tile."""
    import torch

    def change(x):
        if rising:
            grow = torch.linspace(0.1, 4.0, x["Kprefix"].shape[2], device="cuda")[None, None, :, None]
            x["Kprefix"] = (x["Kprefix"].float() * grow).bfloat16().contiguous()

    check(**c, prefix_alloc=c["P"] + 3, seed=c["P"], change=change)
