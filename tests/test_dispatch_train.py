"""What the operators around the products launch, at the edges of their rules (host code: nothing is launched)."""
import pytest

from dispatch_train import dispatch

F32, BF16 = 0, 1


@pytest.mark.parametrize("B,P,C,G,dtype,off", [(65535, 1, 33800, 65, BF16, 0), (65535, 1, 60000, 100, BF16, 0), (65535, 10, 65536, 128, BF16, 1),
                                               (65535, 323, 2964, 78, BF16, 1), (16926, 9, 65536, 256, F32, 1), (65468, 1, 65500, 100, BF16, 0)])
def test_normalisations_of_many_groups_are_launched(B, P, C, G, dtype, off):
    """As many images and groups as are taken: more threads than 32 bits count would be an image's channels in
    registers each."""
    for call in dispatch([(kind, B, P, C, G, dtype, off, act) for kind in ("norm_fwd", "norm_bwd") for act in range(3)]):
        assert call.rc == 0, call
