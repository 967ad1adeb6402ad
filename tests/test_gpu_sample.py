"""dc_sample_tokens against its definition in 64 bits: every rule alone and together, ties, masked and odd logits, rows that leave nothing, odd and
large vocabularies, strides, and random numbers at the ends of their range."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def dc():
    import paper_2609_35115_b200 as dc
    dc.load_library()
    return dc


def pick(l, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, probability) of one row of float64 logits."""
    l = np.where(np.isnan(l), -np.inf, l) + 0.0
    if not (l > -np.inf).any():
        return -1, 0.0
    if not T > 0:
        return int(np.argmax(l)), 1.0
    order = np.argsort(-l, kind="stable")
    order = order[l[order] > -np.inf]
    if k > 0:
        order = order[:k]
    top = l[order[0]]
    with np.errstate(invalid="ignore", over="ignore"):
        weight = lambda x: np.where(x == np.inf, 1.0, 0.0) if np.isinf(top) else np.exp((x - top) / T)
    w = weight(l[order])
    many = len(order)
    if p < 1:
        many = 1 + min(int(np.searchsorted(np.cumsum(w), p * w.sum())), many - 1)
    kept = order[:many]
    kept = np.sort(kept[weight(l[kept]) >= m])
    w = weight(l[kept])
    mass = np.cumsum(w)
    i = int(np.searchsorted(mass, u * mass[-1], side="right"))
    if i == len(kept):       # u >= 1
        i = int(np.nonzero(w)[0][-1])
    return int(kept[i]), w[i] / mass[-1]


def check(dc, logits, u, T=None, k=None, p=None, m=None):
    n = logits.shape[0]
    dev = lambda x, t: None if x is None else torch.tensor(x, dtype=t, device="cuda")
    probs = torch.full((n,), 9.0, device="cuda")
    uu = dev(u, torch.float32)
    rules = dict(temperature=dev(T, torch.float32), top_k=dev(k, torch.int32), top_p=dev(p, torch.float32), min_p=dev(m, torch.float32))
    tokens = dc.sample_tokens(logits, uu, probs=probs, **rules)
    again = dc.sample_tokens(logits, uu, **rules)
    assert torch.equal(tokens, again)
    host = logits.double().cpu().numpy()
    f = lambda name, off: np.full(n, off) if rules[name] is None else rules[name].double().cpu().numpy()
    T, k, p, m, u = f("temperature", 1.0), f("top_k", 0), f("top_p", 1.0), f("min_p", 0.0), uu.double().cpu().numpy()
    for r in range(n):
        want, share = pick(host[r], u[r], T[r], int(k[r]), p[r], m[r])
        assert int(tokens[r]) == want, (r, int(tokens[r]), want, T[r], k[r], p[r], m[r], u[r])
        # fp64 inside, one rounding to fp32 at the end
        assert abs(float(probs[r]) - share) <= 2.0 ** -24 * share * 1.001, (r, float(probs[r]), share)


def logits_of(rng, n, vocab, dtype, spread=2.0, peaks=24):
    l = spread * rng.standard_normal((n, vocab))
    for r in range(n):
        at = rng.integers(0, vocab, min(peaks, vocab))
        l[r, at] += 6 + 2 * rng.standard_normal(len(at))
    return torch.tensor(l, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 7, 64, 1000, 4097, 16384, 16385, 32001, 100003])
def test_rules_together(dc, vocab, dtype):
    rng = np.random.default_rng(vocab + len(dtype))
    n = 24
    l = logits_of(rng, n, vocab, TYPES[dtype])
    u = rng.random(n)
    r = np.arange(n)
    check(dc, l, u)
    check(dc, l, u, T=0.5 + 0.25 * (r % 5))
    check(dc, l, u, k=1 + (r * r) % 60)
    check(dc, l, u, p=(r % 12) / 11)
    check(dc, l, u, m=(r % 6) / 5)
    check(dc, l, u, T=np.where(r % 7 == 6, 0.0, 0.4 + 0.1 * r), k=np.where(r % 3 == 0, 0, 5 * r), p=np.where(r % 4 == 0, 1.0, 0.3 + 0.025 * r), m=np.where(r % 5 == 0, 0.0, 0.01 * r))


@pytest.mark.parametrize("n", [1, 3, 200])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_and_few_rows_of_the_largest_vocabulary(dc, n, dtype):
    rng = np.random.default_rng(n)
    vocab = 262144 if n < 200 else 131072
    l = logits_of(rng, n, vocab, TYPES[dtype])
    r = np.arange(n)
    check(dc, l, rng.random(n), T=np.full(n, 0.8), k=np.where(r % 2 == 0, 0, 1000), p=np.where(r % 4 < 2, 0.95, 1.0))
    with pytest.raises(dc.DCError):
        dc.sample_tokens(torch.zeros(1, 262145, device="cuda"), torch.zeros(1, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
def test_ties(dc, dtype):
    """Equal logits: whole rows of them, and groups that a rule cuts through."""
    t = TYPES[dtype]
    rng = np.random.default_rng(3)
    for vocab in (5, 300, 20001, 70000):
        n = 16
        u = rng.random(n)
        r = np.arange(n)
        flat = torch.full((n, vocab), -3.0, dtype=t, device="cuda")
        check(dc, flat, u)
        check(dc, flat, u, k=1 + r * vocab // 17)
        check(dc, flat, u, p=(r + 1) / 17)
        check(dc, flat, u, k=1 + r * vocab // 17, p=np.full(n, 0.37), T=np.full(n, 0.3))
        steps = torch.tensor(rng.integers(-4, 3, (n, vocab)) * 0.5, device="cuda").to(t)
        check(dc, steps, u, k=1 + r * vocab // 40)
        check(dc, steps, u, p=(r + 1) / 17, m=np.full(n, 0.2))
        check(dc, steps, u, k=1 + r * vocab // 20, p=(r + 1) / 17)
        check(dc, steps, u, T=np.zeros(n))
        zeros = torch.where(torch.tensor(rng.random((n, vocab)) < 0.5, device="cuda"), -0.0, 0.0).to(t)     # one logit, two zeros
        check(dc, zeros, u, k=1 + r * vocab // 17)
        check(dc, zeros, u, T=np.zeros(n))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 5000, 40001])
def test_masked_and_odd_logits(dc, vocab, dtype):
    t = TYPES[dtype]
    rng = np.random.default_rng(vocab)
    n = 12
    l = logits_of(rng, n, vocab, t)
    l[0] = -torch.inf                                   # nothing left
    l[1] = torch.nan
    l[2, : vocab - 1] = -torch.inf                      # one token left, the last
    l[3, vocab // 2:] = torch.finfo(t).min              # the type's lowest value
    l[4] = torch.finfo(t).min                           # a whole row of it: a row like any other
    l[5, 3] = torch.nan
    l[6, [1, vocab - 2]] = torch.inf                    # two infinities
    l[7, ::2] = -torch.inf
    l[8] = torch.finfo(t).max
    l[9, 4], l[9, 5] = torch.finfo(t).max, torch.finfo(t).min
    l[10, 0], l[10, 1:] = torch.inf, -torch.inf
    l[11, :-2] = torch.nan
    u = rng.random(n)
    r = np.arange(n)
    for rules in ({}, dict(T=np.full(n, 0.7)), dict(k=np.full(n, 3)), dict(k=np.full(n, vocab + 5)), dict(p=np.full(n, 0.6)), dict(m=np.full(n, 0.5)), dict(T=np.zeros(n)),
                  dict(k=np.full(n, 4), p=np.full(n, 0.9), m=np.full(n, 0.01), T=1 + r % 2)):
        check(dc, l, u, **rules)


def test_rules_and_random_numbers_at_their_ends(dc):
    rng = np.random.default_rng(11)
    n, vocab = 8, 3001
    l = logits_of(rng, n, vocab, torch.float32)
    below = float(np.nextafter(np.float32(1), np.float32(0)))
    for u in (0.0, below, 1.0, 2.0, 1e-30):
        check(dc, l, np.full(n, u))
        check(dc, l, np.full(n, u), k=np.full(n, 40), p=np.full(n, 0.9))
    u = rng.random(n)
    for rules in (dict(k=np.full(n, -1)), dict(k=np.full(n, vocab)), dict(k=np.full(n, vocab - 1)), dict(k=np.full(n, 2 ** 31 - 1)), dict(p=np.full(n, 0.0)), dict(p=np.full(n, -1.0)),
                  dict(p=np.full(n, 5.0)), dict(p=np.full(n, below)), dict(p=np.full(n, 1e-20)), dict(m=np.full(n, 1.0)), dict(m=np.full(n, -1.0)), dict(T=np.full(n, 1e-3)),
                  dict(T=np.full(n, 1e-30)), dict(T=np.full(n, 1e-44)), dict(T=np.full(n, 100.0)), dict(T=np.full(n, 1e30)), dict(T=np.full(n, -1.0)), dict(T=np.full(n, np.nan))):
        check(dc, l, u, **rules)
    tokens = dc.sample_tokens(l, torch.full((n,), float("nan"), device="cuda"))      # no random number: the first token that weighs anything
    assert torch.equal(tokens, dc.sample_tokens(l, torch.zeros(n, device="cuda")))


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_rows_that_are_not_aligned(dc, dtype):
    rng = np.random.default_rng(5)
    for vocab, stride in ((1003, 1003), (1003, 1009), (501, 4096), (33333, 33335), (4, 5)):
        n = 9
        wide = logits_of(rng, n, stride, TYPES[dtype])
        wide[:, vocab:] = 50.0                               # larger than any logit of the rows
        check(dc, wide[:, :vocab], rng.random(n), k=np.arange(n) * 7, p=np.full(n, 0.8))


def test_what_is_not_written_and_what_is_refused(dc):
    l = torch.zeros(4, 100, device="cuda")
    u = torch.zeros(4, device="cuda")
    tokens = torch.full((6,), 77, dtype=torch.int32, device="cuda")
    assert dc.sample_tokens(l, u, tokens=tokens[1:5]).tolist() == [0] * 4 and tokens[0] == 77 and tokens[5] == 77
    for call in (lambda: dc.sample_tokens(l[0], u), lambda: dc.sample_tokens(l.cpu(), u), lambda: dc.sample_tokens(l.T, u), lambda: dc.sample_tokens(l, u[:3]),
                 lambda: dc.sample_tokens(l, u.double()), lambda: dc.sample_tokens(l, u, top_k=u), lambda: dc.sample_tokens(l, u, top_p=u.cpu()),
                 lambda: dc.sample_tokens(l, u, tokens=u), lambda: dc.sample_tokens(l, u, probs=tokens)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        dc.sample_tokens(l.double(), u)
    with pytest.raises(dc.DCError):
        dc.sample_tokens(torch.zeros(500, device="cuda")[1:401].view(4, 100), u)      # not 16-byte aligned
    assert dc.sample_tokens(l, u).tolist() == [0] * 4


def test_a_captured_draw_reads_its_rules_and_numbers_when_it_runs(dc):
    rng = np.random.default_rng(8)
    n, vocab = 5, 20000
    l = logits_of(rng, n, vocab, torch.float32)
    u, T, tokens = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        dc.sample_tokens(l, u, temperature=T, tokens=tokens)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        dc.sample_tokens(l, u, temperature=T, tokens=tokens)
    for _ in range(4):
        u.copy_(torch.tensor(rng.random(n), dtype=torch.float32))
        T.copy_(torch.tensor(0.5 + rng.random(n), dtype=torch.float32))
        g.replay()
        assert torch.equal(tokens, dc.sample_tokens(l, u, temperature=T))
    torch.cuda.synchronize()


def test_shares_of_many_draws(dc):
    """Evenly spaced random numbers take every token its share of times, to one."""
    n, vocab = 4000, 50
    row = torch.tensor(np.random.default_rng(2).standard_normal(vocab), dtype=torch.float32, device="cuda")
    u = (torch.arange(n, device="cuda") + 0.5) / n
    got = torch.bincount(dc.sample_tokens(row.repeat(n, 1), u).long(), minlength=vocab).double()
    assert (got - n * torch.softmax(row.double(), 0)).abs().max() <= 1.0 + n * 2.0 ** -24      # (u is rounded to fp32)


@pytest.mark.parametrize("T", [np.inf, 1e30, 1e38, 3e4, 50.0])
def test_scores_closer_than_weights_can_tell(dc, T):
    """High temperatures: neighbouring logits have equal weights, and their order still decides who is kept."""
    rng = np.random.default_rng(17)
    n, vocab = 6, 9001
    u = rng.random(n)
    l = torch.tensor(rng.standard_normal((n, vocab)), dtype=torch.float32, device="cuda")
    check(dc, l, u, T=np.full(n, T), k=1 + np.arange(n) * 1700)
    check(dc, l, u, T=np.full(n, T), p=(np.arange(n) + 0.5) / n)
    l[:, ::3] *= 1e38
    l[0, 7], l[0, 8] = torch.finfo(torch.float32).max, torch.finfo(torch.float32).min
    check(dc, l, u, T=np.full(n, T), k=1 + np.arange(n) * 1700, p=np.full(n, 0.8))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,stride", [(8200, 8200), (9001, 9003), (30000, 30002)])
def test_many_rows(dc, vocab, stride, dtype):
    """Rows enough for every SM: a row is streamed by one CTA."""
    t = TYPES[dtype]
    rng = np.random.default_rng(vocab)
    n = 150
    wide = logits_of(rng, n, stride, t)
    wide[:, vocab:] = 60.0
    l = wide[:, :vocab]
    u = rng.random(n)
    r = np.arange(n)
    check(dc, l, u, T=np.where(r % 7 == 6, 0.0, 0.4 + 0.02 * r), k=np.where(r % 3 == 0, 0, 5 * r), p=np.where(r % 4 == 0, 1.0, 0.3 + 0.004 * r), m=np.where(r % 5 == 0, 0.0, 0.001 * r))
    l[:40] = torch.tensor(rng.integers(-4, 3, (40, vocab)) * 0.5, device="cuda").to(t)      # ties
    l[40:50] = 1.0
    l[50] = -torch.inf
    l[51, : vocab - 1] = torch.nan
    l[52:56, 3::7] = torch.inf
    l[56:60, ::2] = -torch.inf
    l[60], l[61] = torch.finfo(t).max, torch.finfo(t).min
    l[62:66, 5:] = -torch.inf
    check(dc, l, u, T=0.5 + 0.01 * r, k=np.where(r % 2 == 0, 0, 1 + r * vocab // 300), p=np.where(r % 4 < 2, 1.0, (r + 1) / 151))
    check(dc, l, u, p=np.full(n, 0.5), T=np.where(r % 2 == 0, 1e30, 0.7))
    check(dc, l, u, T=np.zeros(n))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9000, 100003])
def test_flat_rows(dc, vocab, dtype):
    """Cuts in the middle of a broad distribution: many logits share the last bin, more than one CTA has some."""
    rng = np.random.default_rng(vocab + 1)
    n = 12
    l = torch.tensor(rng.standard_normal((n, vocab)), device="cuda").to(TYPES[dtype])
    u = rng.random(n)
    r = np.arange(n)
    check(dc, l, u, p=(r + 0.5) / n, T=0.3 + 0.3 * r)
    check(dc, l, u, k=1 + r * vocab // n, T=0.3 + 0.3 * r)
    check(dc, l, u, k=1 + r * vocab // n, p=np.full(n, 0.6), T=0.3 + 0.3 * r, m=np.full(n, 0.001))
