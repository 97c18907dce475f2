"""The attention gradient stays inside the scratch it asks for, and does not depend on what lies there before."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF = torch.bfloat16


@pytest.mark.parametrize("n,length,heads,kv,hd", [(300, 1, 3, 1, 64), (129, 1, 2, 1, 128), (77, 8, 4, 2, 64), (10, 43, 2, 1, 128), (5, 64, 2, 2, 64),
                                                  (3, 65, 2, 1, 64), (2, 300, 4, 2, 128)])
def test_scratch(n, length, heads, kv, hd):
    g = torch.Generator().manual_seed(n + length)
    mk = lambda h: torch.randn(n * length, h, hd, generator=g).to(BF).cuda()  # noqa: E731
    q, k, v, dout = mk(heads), mk(kv), mk(kv), mk(heads)
    out, lse = rb.attention(q, k, v, n, length)
    want = rb.attention_grad(q, k, v, out, lse, dout, n, length)
    desc = rb.make_attn_desc(n, length, heads, kv, hd)
    size = rb.rapid_attention_bwd_workspace_bytes(desc)
    room = torch.full((size + (1 << 20),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN wherever nothing is written
    grads = [torch.empty_like(x) for x in (q, k, v)]
    stats = rb.alloc_stats()
    rb.rapid_attention_bwd(desc, q, k, v, None, out, lse, dout, *grads, stats, room[:size])
    assert rb.read_stats(stats)["status"] == 0
    assert (room[size:] == 0xFF).all()
    assert all(torch.equal(a, b) for a, b in zip(grads, (want.dq, want.dk, want.dv)))
