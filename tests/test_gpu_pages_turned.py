"""Keys turned on their way into the pages, with more heads than share a CTA (needs a B200)."""
import pytest
import torch

import paper_2608_22704_b200 as wnw
from pages_ref import E4M3, INT8
from test_gpu_pages import DEV, Both, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", [(E4M3, torch.bfloat16), (INT8, torch.float16)])
@pytest.mark.parametrize("heads,d,T,pairs,neighbours", [(5, 128, 64, 64, False), (8, 64, 16, 32, True), (9, 64, 128, 16, False), (4, 128, 256, 40, True)])
def test_prompts_and_tokens_turned_over_many_heads(heads, d, T, pairs, neighbours, fmt, dtype):
    """Groups of heads, the last one not whole; prompts, pieces that begin inside a page, single tokens; a scale that rises."""
    plan = wnw.wnw_rotary_init(pairs, 1e4, [pairs // 2, pairs - pairs // 2], neighbours=neighbours)
    width = 700 // T + 2
    b = Both(3 * width, heads, T, d, fmt, 3, width)
    for step, rows in enumerate([[3, 300, 70], [1, 1, 1], [40, 0, 260], [1, 1, 1]]):
        n = sum(rows)
        scale = (1.0, 20.0, 0.5, 300.0)[step]
        k, v = (randn(n, heads, d, seed=10 * step + s, dtype=dtype, scale=scale).to(DEV) for s in (1, 2))
        pos = torch.randint(0, 10 ** 6, (2, n), generator=torch.Generator().manual_seed(step), dtype=torch.int32).to(DEV)
        turned = torch.empty_like(k)
        wnw.wnw_rotate(plan, pos, k, turned)
        b.write(k, v, rows, rotary=plan, positions=pos, max_rows=(0, 1, max(rows), 0)[step], k_ref=turned)
        b.check()
