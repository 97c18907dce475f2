"""The losses over the logits against their formulas in 64 bits: sizes, types, pitches, masks, lists and pairs where they can go wrong."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# N, L, V, type, pitch (None: the narrowest), lengths (None: no mask)
GRIDS = [
    (1, 1, 1, BF, None, None), (1, 1, 1, F32, None, None), (2, 1, 2, F32, None, None), (2, 3, 7, BF, 32, [0, 2]), (3, 5, 33, F32, None, [5, 0, 1]),
    (4, 9, 1000, BF, None, [9, 3, 0, 1]), (2, 40, 4096, F32, None, None), (3, 17, 4097, BF, 4160, [17, 1, 8]), (2, 16, 8191, F32, None, [16, 7]),
    (2, 9, 16385, BF, None, None), (2, 6, 32001, F32, None, [6, 2]), (2, 7, 50257, BF, None, [7, 3]), (2, 5, 151936, BF, None, [5, 2]),
    (1, 3, 151936, F32, None, None), (1, 4, 155649, BF, None, None), (2, 3, 262147, BF, None, [3, 1]), (1, 2, 300001, F32, None, None),
    (300, 4, 512, BF, None, [i % 5 for i in range(300)]),
]


def _ids(g):
    return f"{g[0]}x{g[1]}x{g[2]}-{'bf16' if g[3] == BF else 'f32'}"


def _clip_inputs(lu_grid, n_seq, g, by_token=False, ref=True):
    z, targets, mask, _ = lu_grid
    T = z.shape[0]
    live = lu.rows_that_count(targets, mask, z.shape[1])
    lp, _, _ = lu._token_logp(z, targets, live)
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    old = (lp + 0.3 * r(T)).float()
    return old, r(T if by_token else n_seq), (lp + 0.5 * r(T)).float() if ref else None


def _away_from_corners(old, lp, low, high):
    """Ratios within 1e-3 of a corner are moved off it: there the sign of a rounding decides."""
    for c in (1 - low, 1 + high):
        near = ((lp - old.double()).exp() - c).abs() < 1e-3
        old = torch.where(near, old + 0.01, old)
    return old


@pytest.mark.parametrize("shape", GRIDS, ids=_ids)
def test_clip(shape):
    n, length, v, dtype, pitch, lens = shape
    made = lu.grid(n, length, v, dtype, seed=v + n, pitch=pitch, lens=lens)
    z, targets, mask, g = made
    by_token, by_seq = v % 2 == 1, length % 2 == 1
    old, adv, ref = _clip_inputs(made, n, g, by_token)
    live = lu.rows_that_count(targets, mask, v)
    old = _away_from_corners(old, lu._token_logp(z, targets, live)[0], 0.2, 0.3)
    want = lu.clip(z, targets, mask, old, adv, n, ref, 0.2, 0.3, 0.05, 2.0, by_seq)
    assert not want["near"]
    stats = rb.alloc_stats()
    got = rb.clip_loss(z, targets, mask, old, adv, n, length, ref, 0.2, 0.3, 0.05, 2.0, rb.LOSS_NORM_SEQ if by_seq else 0, stats=stats)
    st = rb.read_loss_stats(stats)
    lu.check(want, got, st, dtype)
    assert st["n_clipped"] == want["cut"] and st["n_bad"] == 0
    assert abs(st["mean_log_ratio"] - want["mean_log_ratio"]) <= lu.LSE and abs(st["mean_kl"] - want["mean_kl"]) <= 20 * lu.LSE
    only = rb.clip_loss(z, targets, mask, old, adv, n, length, ref, 0.2, 0.3, 0.05, 2.0, rb.LOSS_NORM_SEQ if by_seq else 0, want_grad=False, stats=stats)
    lu.check(want, only, rb.read_loss_stats(stats), dtype, grad=False)


@pytest.mark.parametrize("shape", GRIDS, ids=_ids)
@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "squared"])
def test_preference(shape, kind):
    n, length, v, dtype, pitch, lens = shape
    z, targets, mask, g = lu.grid(n, length, v, dtype, seed=v + n + 1, pitch=pitch, lens=lens)
    live = lu.rows_that_count(targets, mask, v)
    ref = (lu._token_logp(z, targets, live)[0] + 0.3 * torch.randn(n * length, generator=g).cuda()).float() if v % 2 == 0 else None
    # every generation with the next, one pair twice, one with itself, two that are not valid
    pairs = [(i, (i + 1) % n) for i in range(n)] + [(0, n - 1), (0, n - 1), (n // 2, n // 2), (0, n), (-1, 0)]
    pairs = torch.tensor(pairs, dtype=torch.int32, device="cuda")
    mean = ref is None or length % 2 == 1
    kw = dict(beta=0.3 if mean else 0.1, margin=0.25)
    smoothing = 0.1 if kind == "sigmoid" else 0.0
    want = lu.preference(z, targets, mask, pairs, n, ref, smoothing=smoothing, kind=kind, mean=mean, scale=1.5, **kw)
    assert not want["near"]
    flags = {"sigmoid": 0, "hinge": rb.PREF_HINGE, "squared": rb.PREF_SQUARED}[kind] | (rb.PREF_TOKEN_MEAN if mean else 0)
    stats = rb.alloc_stats()
    for grad in (True, False):
        got = rb.preference_loss(z, targets, mask, pairs, n, length, ref, label_smoothing=smoothing, scale=1.5, flags=flags, want_grad=grad,
                                 stats=stats, **kw)
        st = rb.read_loss_stats(stats)
        lu.check(want, got, st, dtype, grad)
        assert st["n_pairs"] == want["valid"] and abs(st["mean_kl"] - want["won"] / want["valid"]) < 1e-12
        ok = ~want["margins"].isnan()
        assert torch.equal(got.margins.isnan(), ~ok)
        assert bool(((got.margins[ok].double() - want["margins"][ok]).abs() <= want["margins_tol"] + 2.0 ** -24 * want["margins"][ok].abs()).all())


def _lists(z, k, g, ragged=False, spread=2.0):
    """k different columns of each row, with a teacher's logits near the student's."""
    T, V = z.shape
    index = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(T)]).to(torch.int32)
    near = torch.nan_to_num(z.float().cpu(), nan=0.0).gather(1, index.long())
    logit = near + spread * torch.randn(T, k, generator=g) + 6.0
    if ragged:
        index[torch.rand(T, k, generator=g) < 0.3] = -1
        logit[index < 0] = math.nan
    return index.cuda(), logit.cuda()


@pytest.mark.parametrize("shape", GRIDS, ids=_ids)
@pytest.mark.parametrize("tail", [False, True])
def test_distill(shape, tail):
    n, length, v, dtype, pitch, lens = shape
    z, _, mask, g = lu.grid(n, length, v, dtype, seed=v + n + 2, pitch=pitch, lens=lens)
    k = min(v, [1, 5, 32, 33, 64, 200, 256][v % 7])
    index, logit = _lists(z, k, g, ragged=v % 3 == 0)
    tau = [1.0, 2.0, 0.7][v % 3]
    top_lse = None
    if tail:
        part = torch.where(index >= 0, logit.double() / tau, -math.inf)
        rest = torch.rand(n * length, generator=g).cuda().double() * 0.8 + 0.001
        top_lse = torch.logsumexp(torch.cat([part, torch.full_like(part[:, :1], -30.0)], 1), 1) + torch.log1p(rest)
        top_lse = top_lse.float()
    want = lu.distill(z, index, logit, mask, top_lse, tau, 3.0)
    stats = rb.alloc_stats()
    got = rb.distill_loss(z, index, logit, mask, top_lse, tau, 3.0, stats=stats)
    lu.check(want, got, rb.read_loss_stats(stats), dtype)
    only = rb.distill_loss(z, index, logit, mask, top_lse, tau, 3.0, want_grad=False, stats=stats)
    lu.check(want, only, rb.read_loss_stats(stats), dtype, grad=False)
    assert rb.read_loss_stats(stats)["n_bad"] == want["bad"] == 0


# ---- rows, lists and pairs that do not count -----------------------------------------------------------------------

def test_clip_tokens_out_of_range():
    made = lu.grid(3, 8, 500, BF, seed=1)
    z, targets, mask, g = made
    old, adv, ref = _clip_inputs(made, 3, g)
    targets[3], targets[10], targets[23] = -1, 500, 2 ** 31 - 1
    old = _away_from_corners(old, lu._token_logp(z, targets, lu.rows_that_count(targets, mask, 500))[0], 0.2, 0.2)
    for by_seq in (False, True):
        want = lu.clip(z, targets, mask, old, adv, 3, ref, beta=0.1, by_seq=by_seq)
        stats = rb.alloc_stats()
        got = rb.clip_loss(z, targets, mask, old, adv, 3, 8, ref, kl_beta=0.1, flags=rb.LOSS_NORM_SEQ if by_seq else 0, stats=stats)
        st = rb.read_loss_stats(stats)
        lu.check(want, got, st, BF)
        assert st["n_bad"] == 3 and st["n_tokens"] == 21


@pytest.mark.parametrize("kind", ["clip", "preference", "distill"])
def test_nothing_counts(kind):
    z, targets, _, g = lu.grid(2, 5, 300, F32, seed=2)
    mask = torch.zeros(10, dtype=torch.uint8, device="cuda")
    z.fill_(math.nan)
    stats = rb.alloc_stats()
    if kind == "clip":
        got = rb.clip_loss(z, targets, mask, torch.zeros(10).cuda(), torch.ones(2).cuda(), 2, 5, flags=rb.LOSS_NORM_SEQ, stats=stats)
        want = 0.0
    elif kind == "preference":
        got = rb.preference_loss(z, targets, mask, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), 2, 5, flags=rb.PREF_TOKEN_MEAN, stats=stats)
        want = math.log(2.0)
    else:
        got = rb.distill_loss(z, torch.zeros(10, 3, dtype=torch.int32).cuda(), torch.zeros(10, 3).cuda(), mask, stats=stats)
        want = 0.0
    assert abs(float(got.loss) - want) < 1e-7 and bool((got.dlogits == 0).all())
    st = rb.read_loss_stats(stats)
    assert st["n_tokens"] == 0 and st["status"] == 0 and st["n_bad"] == 0


def test_preference_without_a_valid_pair():
    z, targets, mask, g = lu.grid(2, 5, 300, BF, seed=3)
    got = rb.preference_loss(z, targets, mask, torch.tensor([[0, 2], [-5, 1]], dtype=torch.int32).cuda(), 2, 5)
    assert float(got.loss) == 0.0 and bool((got.dlogits == 0).all()) and bool(got.margins.isnan().all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_lists_that_are_not_valid(dtype, tail):
    z, _, mask, g = lu.grid(1, 14, 1000, dtype, seed=4)
    index, logit = _lists(z, 40, g)
    index[1] = -1                       # nothing in it: masked
    index[2, 39] = index[2, 0]          # one twice
    index[3, 5], index[3, 6] = 77, 77   # the same beside one another
    index[4, 7] = 1000                  # out of range
    logit[5, 3] = math.nan
    logit[6, 0] = math.inf
    logit[7] = -math.inf                # no finite logit: masked, or (with a bucket) all of the mass in it
    logit[8, 1:] = -math.inf            # one entry of all the list's mass
    index[9, 1:] = -1
    index[10, :39] = -1
    logit[11, 2] = -3.0e38
    top_lse = None
    if tail:
        top_lse = (torch.logsumexp(torch.cat([torch.where(index >= 0, logit.double(), -math.inf), torch.full_like(logit[:, :1], -20.0).double()], 1), 1) + 0.2).float()
        top_lse[5], top_lse[6] = 3.0, 3.0
        top_lse[12] = math.nan
        top_lse[13] = math.inf
    want = lu.distill(z, index, logit, mask, top_lse)
    stats = rb.alloc_stats()
    got = rb.distill_loss(z, index, logit, mask, top_lse, stats=stats)
    st = rb.read_loss_stats(stats)
    lu.check(want, got, st, dtype)
    assert st["n_bad"] == want["bad"] == (7 if tail else 5)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_whole_vocabulary_listed(dtype):
    """Nothing is left for the bucket: K = V, with the teacher's mass all in the list (and, rounded, a little more)."""
    z, _, mask, g = lu.grid(1, 6, 200, dtype, seed=5)
    index, logit = _lists(z, 200, g)
    exact = torch.logsumexp(logit.double(), 1)
    top_lse = torch.nextafter(exact.float(), torch.tensor(-math.inf, device="cuda"))
    top_lse = torch.where(top_lse.double() > exact, torch.nextafter(top_lse, torch.tensor(-math.inf, device="cuda")), top_lse)
    want = lu.distill(z, index, logit, mask, top_lse)
    stats = rb.alloc_stats()
    lu.check(want, rb.distill_loss(z, index, logit, mask, top_lse, stats=stats), rb.read_loss_stats(stats), dtype)
    want = lu.distill(z, index, logit, mask)
    lu.check(want, rb.distill_loss(z, index, logit, mask, stats=stats), rb.read_loss_stats(stats), dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_hardly_anything_beside_the_list(dtype):
    """A student that puts all but 1e-9 of its mass on the list: the rest is summed by itself, not as a difference from one."""
    z, _, mask, g = lu.grid(1, 5, 4000, dtype, seed=6, std=1.0, boost=0.0)
    index, logit = _lists(z, 8, g)
    z.scatter_(1, index.long(), (torch.randn(5, 8, generator=g) + 30.0).cuda().to(dtype))
    top_lse = (torch.logsumexp(logit.double(), 1) + math.log1p(1e-4)).float()
    want = lu.distill(z, index, logit, mask, top_lse)
    stats = rb.alloc_stats()
    lu.check(want, rb.distill_loss(z, index, logit, mask, top_lse, stats=stats), rb.read_loss_stats(stats), dtype)


# ---- masked vocabulary, extreme values --------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
@pytest.mark.parametrize("v", [100, 5000, 40000, 152000])
def test_masked_vocabulary(dtype, low, v):
    made = lu.grid(2, 4, v, dtype, seed=7)
    z, targets, mask, g = made
    value = -math.inf if low == "-inf" else torch.finfo(dtype).min
    dead = torch.rand(8, v, generator=g).cuda() < 0.9
    dead[0] = True                      # all but the token
    dead[1, : v // 2], dead[1, v // 2:] = True, False
    dead.scatter_(1, targets.long()[:, None], False)
    z[dead] = value
    old, adv, ref = _clip_inputs(made, 2, g)
    old = _away_from_corners(old, lu._token_logp(z, targets, lu.rows_that_count(targets, mask, v))[0], 0.2, 0.2)
    want = lu.clip(z, targets, mask, old, adv, 2, ref, beta=0.1)
    stats = rb.alloc_stats()
    got = rb.clip_loss(z, targets, mask, old, adv, 2, 4, ref, kl_beta=0.1, stats=stats)
    lu.check(want, got, rb.read_loss_stats(stats), dtype)
    assert bool((got.dlogits[dead] == 0).all())
    pairs = torch.tensor([[0, 1]], dtype=torch.int32).cuda()
    want = lu.preference(z, targets, mask, pairs, 2)
    lu.check(want, rb.preference_loss(z, targets, mask, pairs, 2, 4, stats=stats), rb.read_loss_stats(stats), dtype)
    index = targets[:, None].repeat(1, 1).contiguous()
    logit = torch.zeros(8, 1).cuda()
    top_lse = torch.full((8,), 0.05).cuda()
    top_lse[0] = 0.0                    # no mass where the student has none
    for lse in (None, top_lse):
        want = lu.distill(z, index, logit, mask, lse)
        got = rb.distill_loss(z, index, logit, mask, lse, stats=stats)
        lu.check(want, got, rb.read_loss_stats(stats), dtype)
        assert bool((got.dlogits[dead] == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_far_logits(dtype):
    """Logits of some hundreds, all equal ones, and a row whose first half is far below the second."""
    made = lu.grid(1, 5, 3000, dtype, seed=8, std=1.0, boost=2.0)
    z, targets, mask, g = made
    z[0] += 40.0
    z[1] -= 40.0
    z[2] = 1.5
    z[3, :1500] = -60.0
    z[4] *= 8.0
    old, adv, ref = _clip_inputs(made, 1, g)
    old = _away_from_corners(old, lu._token_logp(z, targets, lu.rows_that_count(targets, mask, 3000))[0], 0.2, 0.2)
    want = lu.clip(z, targets, mask, old, adv, 1, ref, beta=0.1)
    stats = rb.alloc_stats()
    lu.check(want, rb.clip_loss(z, targets, mask, old, adv, 1, 5, ref, kl_beta=0.1, stats=stats), rb.read_loss_stats(stats), dtype)


def test_clip_without_a_clip_and_without_an_advantage():
    made = lu.grid(2, 6, 700, F32, seed=9)
    z, targets, mask, g = made
    old, adv, _ = _clip_inputs(made, 2, g)
    inf = math.inf
    want = lu.clip(z, targets, mask, old, adv, 2, low=inf, high=inf)
    stats = rb.alloc_stats()
    lu.check(want, rb.clip_loss(z, targets, mask, old, adv, 2, 6, eps_low=inf, eps_high=inf, stats=stats), rb.read_loss_stats(stats), F32)
    old[0], adv[0] = -2000.0, 0.0       # a ratio that overflows, times nothing
    got = rb.clip_loss(z, targets, mask, old, adv, 2, 6)
    assert bool((got.dlogits[:6] == 0).all()) and math.isfinite(float(got.loss))


# ---- pitches, in place, other streams, graphs, the same bits ------------------------------------------------------------

def _calls(z, targets, mask, g, n, length):
    T, v = z.shape
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    old, ref, adv = r(T) - 8.0, r(T) - 8.0, r(n)
    pairs = torch.tensor([(i, (i + 1) % n) for i in range(n)], dtype=torch.int32).cuda()
    index, logit = _lists(z, 12, g)
    lse = torch.logsumexp(logit, 1) + 0.3
    return {"clip": lambda z, **kw: rb.clip_loss(z, targets, mask, old, adv, n, length, ref, kl_beta=0.1, **kw),
            "preference": lambda z, **kw: rb.preference_loss(z, targets, mask, pairs, n, length, ref, **kw),
            "distill": lambda z, **kw: rb.distill_loss(z, index, logit, mask, lse, 1.5, **kw)}


def _same(a, b, grads=True):
    for x, y in zip(vars(a).values(), vars(b).values()):
        if x is not None and (grads or x.dim() < 2):
            assert torch.equal(x, y)


@pytest.mark.parametrize("v,dtype", [(77, BF), (4099, F32), (20001, BF), (60000, F32), (151937, BF), (200001, F32)])
def test_in_place_and_what_lies_around(v, dtype):
    n, length = 2, 7
    step = 16 // dtype.itemsize
    pitch = (-(-v // step) + 3) * step
    z, targets, mask, g = lu.grid(n, length, v, dtype, seed=10, pitch=pitch, lens=[7, 4])
    room = torch.full((n * length + 4, pitch), 55.0, dtype=dtype, device="cuda")
    for name, call in _calls(z, targets, mask, g, n, length).items():
        apart = call(z)
        room.fill_(55.0)
        room[2:-2, :v] = z
        inside = call(room[2:-2, :v], in_place=True)
        _same(apart, inside)
        assert bool((room[:2] == 55).all()) and bool((room[-2:] == 55).all()) and bool((room[2:-2, v:] == 55).all()), name
        # a gradient of another pitch, between rows that stay
        wide = torch.full((n * length + 2, pitch + step), 33.0, dtype=dtype, device="cuda")
        _into(name, call, z, wide[1:-1, :v])
        assert torch.equal(wide[1:-1, :v], apart.dlogits), name
        assert bool((wide[0] == 33).all()) and bool((wide[-1] == 33).all()) and bool((wide[1:-1, v:] == 33).all()), name


def _into(name, call, z, out):
    """The wrapper with its gradient's place given."""
    keep = rb._loss_grad
    rb._loss_grad = lambda *a: out
    try:
        return call(z)
    finally:
        rb._loss_grad = keep


@pytest.mark.parametrize("v,dtype", [(300, F32), (4096, BF), (50000, BF), (151936, BF)])
def test_same_bits_and_another_stream(v, dtype):
    n, length = 6, 50
    z, targets, mask, g = lu.grid(n, length, v, dtype, seed=11, lens=[50, 3, 20, 50, 0, 49])
    for name, call in _calls(z, targets, mask, g, n, length).items():
        first = call(z)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            with torch.cuda.stream(side):
                again = call(z)
            torch.cuda.current_stream().wait_stream(side)
            _same(first, again)


@pytest.mark.parametrize("v,dtype", [(1000, F32), (33000, BF), (151936, BF)])
def test_captured_and_replayed(v, dtype):
    n, length = 4, 16
    z, targets, mask, g = lu.grid(n, length, v, dtype, seed=12, lens=[16, 5, 9, 16])
    other = lu.grid(n, length, v, dtype, seed=13, lens=[16, 5, 9, 16])[0]
    calls = _calls(z, targets, mask, g, n, length)
    place = torch.empty_like(other)
    for name, call in calls.items():
        place.copy_(z)
        call(place)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = call(place)
            twice = call(place)
        for x in (z, other, z):
            place.copy_(x)
            graph.replay()
            torch.cuda.synchronize()
            now = call(x)
            _same(now, held)
            _same(now, twice)


def test_two_streams_at_once():
    """Calls with workspaces of their own run beside one another."""
    n, length, v = 8, 100, 32000
    made = [lu.grid(n, length, v, BF, seed=20 + i, lens=[100, 7, 60, 100, 33, 0, 80, 99]) for i in range(2)]
    calls = [_calls(z, t, m, g, n, length) for z, t, m, g in made]
    alone = [[c(m[0]) for c in cs.values()] for cs, m in zip(calls, made)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    results = [[], []]
    for k in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                results[i].append(list(calls[i].values())[k](made[i][0]))
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in zip(alone[i], results[i]):
            _same(a, b)


# ---- parts of a mini-batch, differences, a training step ---------------------------------------------------------------------

def test_parts_with_a_given_number_add_up():
    n, length, v = 6, 20, 3000
    z, targets, mask, g = lu.grid(n, length, v, F32, seed=14, lens=[20, 3, 9, 20, 1, 15])
    old, adv = torch.randn(n * length, generator=g).cuda() - 9.0, torch.randn(n, generator=g).cuda()
    half = n * length // 2
    parts = [slice(0, half), slice(half, None)]
    for flags, norm in ((0, 68.0), (rb.LOSS_NORM_SEQ, 6.0)):
        whole = rb.clip_loss(z, targets, mask, old, adv, n, length, flags=flags)
        got = [rb.clip_loss(z[p], targets[p], mask[p], old[p], a, 3, length, flags=flags | rb.LOSS_NORM_GIVEN, norm_z=norm)
               for p, a in zip(parts, (adv[:3], adv[3:]))]
        # the weight and the loss are rounded once each on either side
        assert abs(float(got[0].loss) + float(got[1].loss) - float(whole.loss)) <= 4 * 2.0 ** -24 * (abs(float(got[0].loss)) + abs(float(got[1].loss)))
        assert torch.equal(torch.cat([x.dlogits for x in got]), whole.dlogits)
    index, logit = _lists(z, 6, g)
    whole = rb.distill_loss(z, index, logit, mask)
    got = [rb.distill_loss(z[p], index[p], logit[p], mask[p], flags=rb.LOSS_NORM_GIVEN, norm_z=68.0) for p in parts]
    assert torch.equal(torch.cat([x.dlogits for x in got]), whole.dlogits)
    pairs = torch.tensor([[0, 1], [1, 2], [3, 5]], dtype=torch.int32).cuda()
    whole = rb.preference_loss(z, targets, mask, pairs, n, length)
    got = [rb.preference_loss(z[p], targets[p], mask[p], q, 3, length, flags=rb.LOSS_NORM_GIVEN, norm_z=3.0)
           for p, q in zip(parts, (pairs[:2].contiguous(), (pairs[2:] - 3).contiguous()))]
    assert torch.equal(torch.cat([x.dlogits for x in got]), whole.dlogits)


def test_gradients_against_differences():
    """Central differences of the library's own loss in one column at a time; the losses' third derivatives by a logit are below
    |loss terms| ~ 10, so the step's error is 10 h^2 / 6, and the loss in double is good to LSE a row."""
    n, length, v, h = 2, 3, 40, 0.03125
    z, targets, mask, g = lu.grid(n, length, v, F32, seed=15, std=1.0, boost=1.0, lens=[3, 2])
    live = lu.rows_that_count(targets, mask, v)
    lp = lu._token_logp(z, targets, live)[0]
    old, ref, adv = (lp - 0.05).float(), (lp + 0.1).float(), torch.tensor([1.0, -0.7]).cuda()
    pairs = torch.tensor([[0, 1]], dtype=torch.int32).cuda()
    index, logit = _lists(z, 5, g, spread=0.5)
    lse = torch.logsumexp(logit, 1) + 0.5
    stats = rb.alloc_stats()
    for call in (lambda x: rb.clip_loss(x, targets, mask, old, adv, n, length, ref, kl_beta=0.3, stats=stats),
                 lambda x: rb.preference_loss(x, targets, mask, pairs, n, length, ref, beta=0.5, stats=stats),
                 lambda x: rb.distill_loss(x, index, logit, mask, lse, 1.5, stats=stats)):
        d = call(z).dlogits
        for r in (0, 2, 3):
            for c in sorted({0, int(targets[r]), int(index[r, 0]), v - 1}):
                value = []
                for sign in (1, -1):
                    x = z.clone()
                    x[r, c] += sign * h
                    call(x)
                    value.append(rb.read_loss_stats(stats)["loss"])
                slope = (value[0] - value[1]) / (2 * h)
                assert abs(slope - float(d[r, c])) <= 10 * h * h / 6 + 10 * lu.LSE / h


def test_a_training_step_of_each_kind_on_one_head():
    """The three losses one after the other on the logits of one head, in place, the gradients taken back to hidden states and
    weight, as a script does that warms a policy up on a teacher, aligns it and trains it on."""
    n, length, v, dim = 4, 12, 6000, 64
    _, targets, mask, g = lu.grid(n, length, v, BF, seed=16, lens=[12, 5, 12, 9])
    hidden = torch.randn(n * length, dim, generator=g).cuda().to(BF)
    weight = (torch.randn(dim, v, generator=g) * 0.3).cuda().to(BF)
    old, ref, adv = (torch.randn(k, generator=g).cuda() - s for k, s in ((n * length, 9.0), (n * length, 9.0), (n, 0.0)))
    pairs = torch.tensor([[0, 1], [3, 2]], dtype=torch.int32).cuda()
    z = hidden @ weight
    index, logit = _lists(z, 16, g)
    lse = torch.logsumexp(logit, 1) + 0.2
    steps = {
        "distill": (lambda x: rb.distill_loss(x, index, logit, mask, lse, in_place=True), lambda x: lu.distill(x, index, logit, mask, lse)),
        "preference": (lambda x: rb.preference_loss(x, targets, mask, pairs, n, length, ref, in_place=True), lambda x: lu.preference(x, targets, mask, pairs, n, ref)),
        "clip": (lambda x: rb.clip_loss(x, targets, mask, old, adv, n, length, ref, kl_beta=0.01, in_place=True),
                 lambda x: lu.clip(x, targets, mask, old, adv, n, ref, beta=0.01)),
    }
    for name, (own, plain) in steps.items():
        z = hidden @ weight
        want = plain(z)
        got = own(z)
        assert got.dlogits is z
        dw, dh = hidden.T.double() @ got.dlogits.double(), got.dlogits.double() @ weight.T.double()
        room = want["grad_tol"] + (lu.HALF[BF] + lu.P) * want["grad"].abs() + 1e-30
        assert bool(((dw - hidden.T.double() @ want["grad"]).abs() <= hidden.T.double().abs() @ room).all()), name
        assert bool(((dh - want["grad"] @ weight.T.double()).abs() <= room @ weight.T.double().abs()).all()), name


def test_rows_past_32_bits():
    """Offsets of elements and bytes beyond 2^32: 40 000 rows of 160 000 columns, of which a few count."""
    T, v = 40000, 160000
    z = torch.empty(T, v, dtype=BF, device="cuda")
    mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
    rows = [0, 13421, 26844, T - 1]
    mask[rows] = 1
    small, t4, _, g = lu.grid(1, 4, v, BF, seed=17)
    z[rows] = small
    targets = torch.zeros(T, dtype=torch.int32, device="cuda")
    targets[rows] = t4
    old = torch.full((T,), -8.0, device="cuda")
    adv = torch.tensor([1.3], device="cuda")
    whole = rb.clip_loss(z, targets, mask, old, adv, 1, T, in_place=True)
    four = rb.clip_loss(small, t4, None, old[:4].contiguous(), adv, 1, 4)
    assert torch.equal(whole.dlogits[rows], four.dlogits) and torch.equal(whole.token_logp[rows], four.token_logp)
    dead = mask == 0
    assert not bool(z[:, 7][dead].any()) and not bool(z[13420].any()) and not bool(z[T - 2].any())
