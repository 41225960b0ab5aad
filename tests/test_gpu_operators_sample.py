"""he_sample against its definition in numpy's float64: ids equal, log-probabilities to a float's rounding."""
import numpy as np
import pytest
import torch

from paper_2308_01320_amd import binding as B
from tests import operators_ref as R

pytestmark = pytest.mark.gpu


def run(z, u, **f):
    def up(x, dt):
        return None if x is None else torch.tensor(x, dtype=dt).cuda()

    ids, lp = B.he_sample(z if z.is_cuda else z.cuda(), up(u, torch.float32), temperature=up(f.get("temperature"), torch.float32), top_k=up(f.get("top_k"), torch.int32),
                          top_p=up(f.get("top_p"), torch.float32), min_p=up(f.get("min_p"), torch.float32))
    return ids.cpu().numpy(), lp.cpu().numpy()


def check(z, u, **f):
    ids, lp = run(z, u, **f)
    zs, f32 = z.double().cpu().numpy(), np.float32
    for r in range(len(u)):
        one = {k: (int(v[r]) if k == "top_k" else float(f32(v[r]))) for k, v in f.items() if v is not None}
        i, want = R.sample_row(zs[r], float(f32(u[r])), **one)
        assert ids[r] == i, (r, ids[r], i, one, u[r])
        # a sum in 64 bits, its logarithm, one rounding to float (and one unit of 2^-23 to spare)
        assert lp[r] == want or abs(lp[r] - want) <= 2.0 ** -23 * max(1.0, abs(want)), (r, lp[r], want)


def logits(rows, vocab, dt, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g) * spread).to(dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 1000, 1025, 50272, 131071])
@pytest.mark.parametrize("spread", [0.5, 3.0])
def test_matches_the_definition(dtype, vocab, spread):
    rows = 12
    rng = np.random.default_rng(vocab)
    z = logits(rows, vocab, R.DTYPES[dtype], vocab, spread)
    u = rng.random(rows).astype(np.float32).tolist()
    t = rng.uniform(0.3, 2.0, rows).tolist()
    k = [0, -1, 1, 2, 5, 50, 1000, vocab, vocab - 1, vocab + 1, 100, 40]
    p = [1.0, 0.9, 0.5, 0.95, 0.99, 0.1, 0.0, -1.0, 2.0, 0.7, 0.999, 0.8]
    m = [0.0, 0.1, 0.01, -1.0, 1.0, 2.0, 0.05, 0.5, 0.001, 0.0, 0.02, 0.0]
    check(z, u)
    check(z, u, temperature=t)
    check(z, u, top_k=k)
    check(z, u, top_p=p)
    check(z, u, min_p=m, temperature=t)
    check(z, u, temperature=t, top_k=k, top_p=p, min_p=m)


@pytest.mark.parametrize("vocab", [100, 5000, 70000])
def test_equal_logits(vocab):
    """All equal, or of a few values: order by id decides what is kept, in one group of equal values as large as the row."""
    z = torch.zeros(6, vocab, dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(1)
    z[3:] = torch.randint(0, 3, (3, vocab), generator=g).bfloat16()
    z[1, ::2] = -0.0  # (equal to +0)
    u = [0.0, 0.5, 0.999, 0.3, 0.77, 0.999]
    check(z, u)
    check(z, u, top_k=[1, 7, vocab // 2, 3, vocab // 3 + 5, vocab - 1])
    check(z, u, top_p=[0.25, 0.5, 0.75, 0.125, 0.9, 0.6])
    check(z, u, top_k=[50] * 6, top_p=[0.5] * 6, min_p=[1.0, 0.5, 0.9, 0.4, 0.3, 0.2], temperature=[0.5, 1, 2, 1, 2, 4])


def test_numbers_at_the_ends():
    z = logits(8, 3001, torch.float32, 5)
    check(z, [0.0, 1.0, 1.5, -0.5, float(np.nextafter(np.float32(1), np.float32(0))), 1e-38, 0.5, 2.0], top_p=[0.9] * 8)
    check(z, [0.0, 1.0, 1.5, -0.5, float(np.nextafter(np.float32(1), np.float32(0))), 1e-38, 0.5, 2.0])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_greedy_and_extreme_temperatures(dtype):
    z = logits(7, 2000, R.DTYPES[dtype], 6)
    z[1, 7] = z[1, 1999] = z[1].max() + 1  # a tie: the lower id
    u = [0.1, 0.9, 0.5, 0.3, 0.7, 0.9999, 0.2]
    check(z, u, temperature=[0.0, -1.0, 0.0, 1e-38, 1e-3, 1e30, 3e38])
    ids, _ = run(z, u, temperature=[float("nan")] * 7, top_p=[0.5] * 7, top_k=[9] * 7)
    first = z.float().argmax(1)
    first[1] = 7
    assert np.array_equal(ids, first.numpy())


def test_masked_logits():
    """-infinity, NaN and the type's lowest value in masked places, rows of nothing, +infinity."""
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        z = logits(9, 700, dt, 8)
        z[0, 1:] = -float("inf")
        z[1, :] = -float("inf")
        z[2, :] = float("nan")
        z[3, 100:] = float("nan")
        z[4, :650] = torch.finfo(dt).min
        z[5, :] = torch.finfo(dt).min
        z[6, 5] = z[6, 9] = float("inf")
        z[7, ::2] = -float("inf")
        u = [0.99, 0.5, 0.5, 0.99, 0.999, 0.5, 0.7, 0.01, 0.5]
        check(z, u)
        check(z, u, temperature=[0.7] * 9, top_k=[600] * 9, top_p=[0.95] * 9, min_p=[0.001] * 9)
        check(z, u, temperature=[0.0] * 9)
        ids, lp = run(z, u)
        assert ids[1] == ids[2] == -1 and lp[1] == lp[2] == -np.inf and ids[6] == 9


def test_rows_in_a_wider_matrix():
    wide = logits(5, 4097, torch.float16, 11).cuda()
    for lo, hi in ((0, 4000), (1, 4001), (3, 4097)):  # rows that begin on any element
        check(wide[:, lo:hi], [0.1, 0.4, 0.6, 0.8, 0.95], top_p=[0.9] * 5, temperature=[0.8] * 5)
    one = logits(1, 999, torch.float32, 12).cuda().expand(4, 999)  # a row for everybody
    check(one, [0.1, 0.4, 0.6, 0.8], top_k=[3, 30, 300, 900])


def test_distribution_of_many_draws():
    """Every number of a fine grid: each token is drawn as often as its share of the kept weight says, to one draw."""
    z = logits(1, 40, torch.float32, 13, 1.0)
    n = 20000
    ids, _ = run(z.expand(n, 40).contiguous(), ((np.arange(n) + 0.5) / n).astype(np.float32).tolist(), top_k=[12] * n, temperature=[0.9] * n)
    zs = z[0].double().numpy()
    w = np.exp((zs - zs.max()) / np.float64(np.float32(0.9)))
    w[np.lexsort((np.arange(40), -zs))[12:]] = 0
    assert np.abs(np.bincount(ids, minlength=40) - n * w / w.sum()).max() <= 1.01


def test_replays_and_repeats():
    z = logits(16, 50272, torch.bfloat16, 14).cuda()
    u = torch.rand(16).cuda()
    p = torch.full((16,), 0.9).cuda()
    B.he_sample(z, u, top_p=p)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        ids, lp = B.he_sample(z, u, top_p=p)
    for s in range(4):
        u.copy_(torch.rand(16))
        z.copy_(logits(16, 50272, torch.bfloat16, 20 + s))
        torch.cuda.synchronize()
        g.replay()
        a, b = B.he_sample(z, u, top_p=p)
        torch.cuda.synchronize()
        assert torch.equal(a, ids) and torch.equal(b, lp)
    check(z, u.cpu().tolist(), top_p=[float(np.float32(0.9))] * 16)


@pytest.mark.parametrize("vocab", [1, 3, 5, 7, 9, 512, 513])
def test_small_vocabularies(vocab):
    """Fewer logits than a lane reads at a time, with every filter, infinities, and temperatures next to nothing."""
    for dt in (torch.float32, torch.bfloat16):
        z = logits(6, vocab, dt, 30 + vocab)
        z[3, vocab // 2] = float("inf")
        z[4, 1:] = -float("inf")
        u = [0.1, 0.5, 0.9, 0.3, 0.7, 1.0]
        check(z, u)
        for t in (1.0, 1e-30, 1e-38):
            check(z, u, temperature=[t] * 6, top_k=[2, 3, 4, 5, 6, 2], top_p=[0.9, 0.5, 0.99, 0.7, 0.3, 0.8], min_p=[0.0, 0.1, 0.01, 0.0, 0.0, 0.5])
            check(z, u, temperature=[t] * 6, top_k=[2, 3, 4, 5, 6, 2])


def test_deep_borders():
    """Filters that keep far more of a row than its largest few thousand tokens, and rows whose largest tokens are many and equal."""
    z = logits(8, 60000, torch.float32, 40, 1.0)
    z[5, ::3] = 5.0
    z[6, 1000:9000] = 7.5
    z[7, :4096] = 3.25
    u = [0.05, 0.3, 0.5, 0.7, 0.9, 0.2, 0.6, 0.99]
    check(z, u, top_p=[0.99, 0.95, 0.9, 0.8, 0.999, 0.9, 0.97, 0.95], temperature=[1.3, 1.0, 2.0, 0.8, 1.0, 1.0, 0.7, 5.0])
    check(z, u, top_k=[20000, 9000, 50000, 6000, 59999, 15000, 4000, 30000], top_p=[0.9, 0.99, 0.5, 0.7, 0.98, 0.6, 0.95, 0.9])
    check(z, u, min_p=[0.01, 0.001, 1e-4, 0.05, 0.02, 0.5, 0.3, 0.1], top_p=[0.99] * 8, top_k=[30000] * 8)
    check(z, u, temperature=[0.0] * 8)
