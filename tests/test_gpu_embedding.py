"""Token embedding and its gradient on the GPU against the definition in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


def _half_ulp(dtype):
    return torch.finfo(dtype).eps / 2


def _pitched(x, extra):
    """x with `extra` further columns between rows, which hold a value that must never count."""
    step = 16 // x.element_size()
    pitch = -(-x.shape[1] // step) * step + extra * step
    wide = torch.full((x.shape[0], pitch), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide


def _tokens(T, V, kind, g):
    if kind == "same":
        t = torch.full((T,), V // 2)
    elif kind == "few":
        t = torch.randint(0, min(V, 3), (T,), generator=g)
    elif kind == "distinct":
        t = torch.randperm(max(V, T), generator=g)[:T] % V
    else:  # frequent tokens have low numbers
        t = (torch.exp(torch.rand(T, generator=g, dtype=torch.float64) * torch.log(torch.tensor(V + 1.0))).long() - 1).clamp(0, V - 1)
    return t.to(torch.int32)


def _mask(T, kind, g):
    if kind == "none":
        return None
    m = torch.zeros(T, dtype=torch.uint8) if kind == "dead" else (torch.rand(T, generator=g) < 0.7).to(torch.uint8) * 3
    return m


CASES = [  # T, V, D, tokens, mask
    (1, 1, 1, "same", "none"), (1, 600, 8, "zipf", "none"), (5, 7, 3, "few", "random"), (31, 40, 9, "same", "none"),
    (33, 40, 257, "same", "random"), (64, 151936, 64, "zipf", "none"), (200, 5, 1001, "few", "random"),
    (700, 1 << 18, 16, "zipf", "random"), (4096, 1000, 24, "same", "none"), (4097, 511, 40, "zipf", "random"),
    (5000, 512, 8, "distinct", "none"), (70001, 3000, 16, "zipf", "random"), (66000, 300, 8, "same", "random"),
    (333, 77, 2056, "zipf", "random"), (100, 50, 12, "zipf", "dead"),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,D,tok,mk", CASES)
def test_embedding_forward(T, V, D, tok, mk, dtype):
    g = torch.Generator().manual_seed(T + V + D)
    tokens, mask = _tokens(T, V, tok, g), _mask(T, mk, g)
    bad = torch.rand(T, generator=g) < 0.05
    tokens[bad] = torch.where(torch.rand(int(bad.sum()), generator=g) < 0.5, -1 - tokens[bad], V + tokens[bad])
    table = torch.randn(V, D, generator=g).to(dtype)
    scale = 1.7
    live = torch.ones(T, dtype=torch.bool) if mask is None else mask != 0
    ok = live & ~bad
    ref = torch.zeros(T, D, dtype=torch.float64)
    ref[ok] = table[tokens[ok].long()].double() * scale
    stats = rb.alloc_stats()
    got = rb.embedding(_pitched(table.cuda(), 1)[:, :D], tokens.cuda(), None if mask is None else mask.cuda(), scale, stats)
    assert got.shape == (T, D) and got.dtype == dtype
    # scale is rounded to float (2^-24), the product too, then the result once
    tol = ref.abs() * (_half_ulp(dtype) + 2 * 2.0 ** -24) + 1e-38
    assert ((got.cpu().double() - ref).abs() <= tol).all()
    st = rb.read_stats(stats)
    assert st["n_tokens"] == int(ok.sum()) and st["n_bad_token"] == int((live & bad).sum()) and st["status"] == 0


@pytest.mark.parametrize("dtype,grad", [(BF, F32), (BF, BF), (F32, F32)])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,D,tok,mk", CASES)
def test_embedding_gradient(T, V, D, tok, mk, dtype, grad, accumulate):
    g = torch.Generator().manual_seed(T + V + D)
    tokens, mask = _tokens(T, V, tok, g), _mask(T, mk, g)
    bad = torch.rand(T, generator=g) < 0.03
    tokens[bad] = V + tokens[bad]
    live = ~bad if mask is None else (mask != 0) & ~bad
    dout = torch.randn(T, D, generator=g).to(dtype)
    dout[~live] = float("nan")  # rows that do not count are never read
    scale = 0.3
    idx = tokens[live].long()
    x = dout[live].double()
    total = torch.zeros(V, D, dtype=torch.float64).index_add_(0, idx, x) * scale
    mass = torch.zeros(V, D, dtype=torch.float64).index_add_(0, idx, x.abs()) * scale
    count = torch.zeros(V, dtype=torch.float64).index_add_(0, idx, torch.ones(len(idx), dtype=torch.float64))[:, None]
    base = torch.randn(V, D, generator=g).to(grad) if accumulate else torch.zeros(V, D, dtype=grad)
    wide = _pitched(base.cuda(), 1) if accumulate else None
    mcuda = None if mask is None else mask.cuda()
    dcuda = _pitched(dout.cuda(), 2)[:, :D]
    got = rb.embedding_grad(dcuda, tokens.cuda(), mcuda, V, scale, grad, wide[:, :D] if accumulate else None)
    ref = base.double() + total
    # every addition of the float sum is off by 2^-24 of a partial sum (at most `mass`); scale and product two more; then
    # one rounding to the result's type
    tol = (count + 3) * 2.0 ** -24 * mass + ref.abs() * _half_ulp(grad) * 1.01 + 1e-38
    assert ((got.cpu().double() - ref).abs() <= tol).all()
    if accumulate:
        assert got.data_ptr() == wide.data_ptr() and torch.isnan(wide[:, D:]).all()
        assert torch.equal(got.cpu()[count[:, 0] == 0], base[count[:, 0] == 0])
    else:
        again = rb.embedding_grad(dcuda, tokens.cuda(), mcuda, V, scale, grad)
        assert torch.equal(got, again)  # the same bits


def test_embedding_gradient_overwrites_what_was_there():
    V, D = 37, 24
    dtable = torch.full((V, 32), float("nan"), device="cuda")
    d = rb.make_embed_desc(6, V, D, BF, ld_table=32)
    ws = torch.full((rb.rapid_embedding_bwd_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    tok = torch.tensor([3, 3, 36, 0, 3, 40], dtype=torch.int32, device="cuda")
    rb.rapid_embedding_bwd(d, tok, None, torch.ones(6, D, dtype=BF, device="cuda"), dtable, ws)
    want = torch.zeros(V, D)
    want[3], want[36], want[0] = 3, 1, 1
    assert torch.equal(dtable[:, :D].cpu(), want) and torch.isnan(dtable[:, D:]).all()


def test_embedding_gradient_captured_and_replayed():
    """One capture, replayed on new contents of its inputs."""
    T, V, D = 5000, 900, 40
    tok, dout = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, D, dtype=BF, device="cuda")
    desc = rb.make_embed_desc(T, V, D, BF)
    ws = torch.empty(rb.rapid_embedding_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    dtable = torch.empty(V, D, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rb.rapid_embedding_bwd(desc, tok, None, dout, dtable, ws)
    for seed in range(2):
        g = torch.Generator().manual_seed(seed)
        tok.copy_(_tokens(T, V, "zipf", g))
        dout.copy_(torch.randn(T, D, generator=g))
        graph.replay()
        assert torch.equal(dtable, rb.embedding_grad(dout, tok, None, V))


def test_empty_calls():
    e = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert rb.embedding(torch.zeros(4, 8, device="cuda"), e).shape == (0, 8)
    assert torch.equal(rb.embedding_grad(torch.zeros(0, 8, device="cuda"), e, None, 4), torch.zeros(4, 8, device="cuda"))
