"""dora_decode_attn_window where there are segments enough for one workgroup each, around the 256 pages
that a workgroup takes at most: windows that fill it, pass it by a page, and take several."""
import numpy as np
import pytest
import torch

from cache_util import Cache, check, window_reference
from gpu_util import lib

pytestmark = pytest.mark.gpu

COPIES = 130  # of each row below: 1,040 segments


def _visible(L, P, window, sinks):
    n, s = -(-L // P), min(-(-sinks // P), -(-L // P))
    return s + n - max(s, max(0, L - window) // P)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("P", [16, 32])
@pytest.mark.parametrize("pages,sinks", [(255, 0), (256, 0), (256, 3), (257, 0), (520, 40)])
def test_windows_around_a_workgroups_pages(pages, sinks, P, dt):
    window = pages * P
    lens = [window + 5 * P, window + 5 * P + 7, window - 1, window, 256 * P, 130 * P + 3, 0, 1]
    print(f"[case] pages={pages} sinks={sinks} P={P} dt={dt}", flush=True)
    seen = {_visible(L, P, window, sinks) for L in lens}
    assert pages in seen and max(seen) > pages  # (what the sinks show is more)
    c = Cache(lens, 1, 64, P, dt, seed=pages + P)
    q = torch.randn(8, 4, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    want, spread = window_reference(c, q, window, sinks)
    dev = c.gpu()
    rows = torch.arange(8).repeat(COPIES).cuda()  # the same pages and queries, over and over
    many = q.cuda()[rows].contiguous()
    out = torch.full_like(many, 7.0)
    lib().dora_decode_attn_window(many, dev["k"], dev["v"], dev["bt"][rows].contiguous(), dev["lens"][rows].contiguous(), None, out,
                                  window=window, sinks=sinks, **dev["kw"])
    torch.cuda.synchronize()
    out = out.reshape(COPIES, 8, 4, 64)
    check(out[0], want, spread, "window")
    assert torch.equal(out.view(torch.int16), out[:1].expand_as(out).contiguous().view(torch.int16))
