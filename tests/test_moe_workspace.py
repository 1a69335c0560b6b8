"""What a layer of experts asks for as its workspace is what it holds there, and no more."""
import pytest

import paper_2507_01676_amd as embx
from test_serving_arguments import FAKE, moe, size


@pytest.mark.parametrize("scale", [None, FAKE])
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("m,f,d,experts,top_k", [(1, 1, 1, 1, 1), (5, 2816, 1024, 8, 2), (19, 333, 1001, 7, 3), (300, 40, 48, 64, 32),
                                                 (1000, 704, 1024, 64, 6), (4096, 2816, 1024, 8, 2), (65536, 5632, 1024, 32, 8)])
def test_workspace_is_what_is_held(m, f, d, experts, top_k, dtype, scale):
    a = moe(scale, m=m, f=f, d=d, experts=experts, top_k=top_k, dtype=dtype, ldx=d, ldr=d, ldy=d, gate__ld=d, up__ld=d, down__ld=f,
            chosen=None, share=None)
    code, need = size(a)
    uses = m * top_k
    # act(..) * (..) in 32 bits or twice 16, its rows in whole eights; the routing; logits; in f32 the results of each use, or of
    # workgroups that share 64 rows and 32 columns, 256 in all
    each = uses * d if m > 64 and not scale and uses * d <= 64 << 20 else 0
    most = uses * ((f + 7) // 8 * 8 * 4 + 8) + (m * experts * 8 if m <= 256 else 0) + 4 * max(each, 256 * 64 * 32)
    assert code == embx.OK and uses * (4 * f + 8) <= need <= most + 8 * 256
