"""Linear attention over segments of many chunks, whose gradients' ends are walked in halves: even and odd counts of chunks, short last
segments and last segments of one half, both storage types, shared heads, several tiles of columns."""
import pytest

import test_gpu_la as la
from paper_2503_01868_amd import binding

from gpu_util import say

pytestmark = la.pytestmark


# B, L, H, group, dk, dv, dtype, halves of segments that the gradients' ends are walked in
CASES = [(1, 2048, 64, 1, 16, 16, "bf16", 8),     # 32 chunks: four segments of 8
         (2, 2100, 32, 1, 16, 24, "bf16", 7),     # 33: three of 10 and one of 3, a half
         (1, 1100, 128, 1, 8, 16, "bf16", 4),     # 18: 10 and 8
         (1, 2110, 128, 1, 16, 16, "bf16", 4),    # 33: 18 and 15; forward in segments of 9
         (1, 1090, 64, 1, 16, 16, "f32", 7),      # 35 of 32 steps: three of 10 and one of 5
         (4, 515, 32, 1, 24, 16, "f32", 4),       # 17: 10 and 7
         (1, 2100, 64, 4, 16, 16, "bf16", 7),     # q and k shared by four heads
         (1, 1090, 32, 2, 16, 130, "f32", 7)]     # two tiles of columns


@pytest.mark.parametrize("B,L,H,group,dk,dv,dtype,halves", CASES)
def test_segments_of_many_chunks(B, L, H, group, dk, dv, dtype, halves):
    say("la segments B=%d L=%d H=%d group=%d dk=%d dv=%d %s" % (B, L, H, group, dk, dv, dtype))
    tiles, state = (2, 64 * 128) if dv > 64 else (1, 64 * 64)
    count = group * tiles
    shares = 2 * count * B * L * (H // group) * dk * 4 + (tiles * B * L * H * 4 if tiles > 1 else 0) if count > 1 else 0
    bytes_ = binding.lib().hyena_la_bwd_workspace_bytes(B, L, H, group, dk, dv, 1 if dtype == "bf16" else 0, 1)
    assert round((bytes_ - shares) / (B * H * tiles * (state * 4 + 8))) == halves  # (the case is what it is meant to be)
    la.check(*la.make(L + H, B, L, H, group, dk, dv, dtype, resets=0.002), dk ** -0.5, dtype)
