"""Rows whose offsets pass 32 bits: the policy operators on slices of one wide matrix of 66000 x 32768 bf16 (4.3 GB), whose last
rows begin beyond element 2^31 and byte 2^32, give the same bits as on compact copies of the slices."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF = torch.bfloat16
ROWS, PITCH = 66000, 32768


@pytest.fixture(scope="module")
def wide():
    m = torch.empty(ROWS, PITCH, dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    m[:, :1024] = torch.randn(ROWS, 1024, generator=g, device="cuda").to(BF)
    m[:, 1024:2048] = 7
    yield m
    del m
    torch.cuda.empty_cache()


def _heads(m, first, count, hd=64):
    return m[:, first * hd:(first + count) * hd].unflatten(1, (count, hd))


def test_embedding(wide):
    g = torch.Generator().manual_seed(2)
    tokens = torch.randint(0, ROWS, (5000,), generator=g, dtype=torch.int32)
    tokens[:3] = torch.tensor([ROWS - 1, 0, ROWS - 1])
    tokens = tokens.cuda()
    table = wide[:, :64]
    assert torch.equal(rb.embedding(table, tokens, scale=3.0), rb.embedding(table.contiguous(), tokens, scale=3.0))


@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_gradient(wide, accumulate):
    g = torch.Generator().manual_seed(3)
    tokens = torch.randint(0, ROWS, (ROWS,), generator=g, dtype=torch.int32)
    tokens[::2] = ROWS - 1
    tokens = tokens.cuda()
    dout = wide[:, 64:192]
    compact = dout.contiguous()
    if accumulate:
        want, near = torch.ones(2, ROWS, 128, dtype=BF, device="cuda")
        got = wide[:, 1024:1024 + 128]
        got.fill_(1)
        for rows, table in ((compact, want), (dout, near), (compact, got)):
            rb.embedding_grad(rows, tokens, None, ROWS, dtable=table)
    else:
        want, near = (rb.embedding_grad(x, tokens, None, ROWS, dtable_dtype=BF) for x in (compact, dout))
        got = wide[:, 1024:1024 + 128]
        desc = rb.make_embed_desc(ROWS, ROWS, 128, BF, PITCH, 128, flags=rb.EMBED_DTABLE_BF16)
        ws = torch.empty(rb.rapid_embedding_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        rb.rapid_embedding_bwd(desc, tokens, None, compact, got, ws)
    assert torch.equal(near, want) and torch.equal(got, want)
    assert (wide[:, 1024 + 128:1024 + 256] == 7).all()
    got.fill_(7)


def test_qk_norm_rope(wide):
    n, length = 2, ROWS // 2
    w = [torch.rand(64, device="cuda") + 0.5 for _ in range(2)]
    inv = 10000.0 ** (-torch.arange(0, 64, 2, device="cuda") / 64)
    q, k, dq_, dk_ = _heads(wide, 0, 2), _heads(wide, 2, 1), _heads(wide, 3, 2), _heads(wide, 5, 1)
    compact = [x.contiguous() for x in (q, k, dq_, dk_)]
    for a, b in zip(rb.qk_norm_rope(q, k, *w, inv, n, length), rb.qk_norm_rope(*compact[:2], *w, inv, n, length)):
        assert torch.equal(a, b)
    got = rb.qk_norm_rope_grad(q, k, *w, inv, dq_, dk_, n, length, dq=_heads(wide, 16, 2), dk=_heads(wide, 18, 1))
    want = rb.qk_norm_rope_grad(*compact[:2], *w, inv, *compact[2:], n, length)
    assert torch.equal(got.dq, want.dq) and torch.equal(got.dk, want.dk)
    assert torch.equal(got.dq_weight, want.dq_weight) and torch.equal(got.dk_weight, want.dk_weight)
    wide[:, 1024:2048] = 7


def test_attention(wide):
    n, length = 330, 200
    q, k, v, dout = _heads(wide, 0, 2), _heads(wide, 2, 1), _heads(wide, 3, 1), _heads(wide, 4, 2)
    compact = [x.contiguous() for x in (q, k, v)]
    desc = rb.make_attn_desc(n, length, 2, 1, 64, ld_q=PITCH, ld_k=PITCH, ld_v=PITCH, ld_out=PITCH)
    out = _heads(wide, 16, 2)
    lse = torch.empty(n, 2, length, device="cuda")
    stats = rb.alloc_stats()
    rb.rapid_attention_fwd(desc, q, k, v, None, out, lse, stats)
    want, lse_want = rb.attention(*compact, n, length)
    assert torch.equal(out, want) and torch.equal(lse, lse_want) and rb.read_stats(stats)["status"] == 0
    got = rb.attention_grad(q, k, v, out, lse, dout, n, length, dq=_heads(wide, 18, 2), dk=_heads(wide, 20, 1), dv=_heads(wide, 21, 1),
                            stats=stats)
    ref = rb.attention_grad(*compact, want, lse, dout.contiguous(), n, length)
    for name in ("dq", "dk", "dv"):
        assert torch.equal(getattr(got, name), getattr(ref, name)), name
    assert rb.read_stats(stats)["status"] == 0
    assert (wide[:, 22 * 64:2048] == 7).all()
    wide[:, 1024:2048] = 7
