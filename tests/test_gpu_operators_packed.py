"""he_packed_attention against its definition in 64 bits."""
import pytest
import torch

from paper_2308_01320_amd import binding as B
from tests import operators_ref as R

pytestmark = pytest.mark.gpu


def weight_step(dt):
    # a weight may be rounded to the type once before it multiplies its value
    return R.half_step(dt) if dt != torch.float32 else 0.0


def check(got, q, k, v, starts, dt, causal, scale):
    for a, b in zip(starts, starts[1:]):
        n = b - a
        if n == 0:
            continue
        seen = torch.ones(n, n, dtype=torch.bool).tril() if causal else None
        want, mag, most = R.attend(q[a:b], k[a:b], v[a:b], scale, seen)
        R.check_attended(got[a:b], want, mag, most, n, dt, weight_step(dt))


def make(dt, nh, nk, d, n, seed=0):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(n, (nh + 2 * nk) * d, generator=g).to(dt)
    return qkv, [t.view(n, -1, d) for t in qkv.split([nh * d, nk * d, nk * d], 1)]


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nh,nk,d", [(2, 2, 64), (4, 2, 128), (3, 1, 80), (2, 1, 96), (2, 1, 256), (5, 1, 16), (2, 2, 112)])
@pytest.mark.parametrize("lens,causal", [((1,), True), ((33, 0, 5, 64), True), ((65, 127, 1, 32), False), ((130, 3), True)])
def test_matches_the_definition(dtype, nh, nk, d, lens, causal):
    dt = R.DTYPES[dtype]
    qkv, (q, k, v) = make(dt, nh, nk, d, sum(lens))
    starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
    dq, dk, dv = (t.view(sum(lens), -1, d) for t in qkv.cuda().split([nh * d, nk * d, nk * d], 1))
    got = B.he_packed_attention(dq, dk, dv, ints(starts), causal=causal)
    check(got.cpu(), q, k, v, starts, dt, causal, d ** -0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts_of_many_tiles(dtype, causal):
    """One prompt over many tiles of keys and several of queries, some rows of it checked."""
    dt, n, nh, nk, d = R.DTYPES[dtype], 1187, 4, 2, 128
    qkv, (q, k, v) = make(dt, nh, nk, d, n + 40)
    got = B.he_packed_attention(q.cuda(), k.cuda(), v.cuda(), ints([0, 40, 40 + n]), causal=causal).cpu()
    at = torch.tensor([0, 1, 31, 32, 63, 64, 127, 128, 255, 256, 500, 511, 512, 640, 1023, 1024, 1151, 1186])
    seen = (torch.arange(n)[None] <= at[:, None]) if causal else None
    want, mag, most = R.attend(q[40 + at], k[40:], v[40:], d ** -0.5, seen)
    R.check_attended(got[40 + at], want, mag, most, n, dt, weight_step(dt))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, bad):
    """The last keys of a sequence and all of its neighbour are NaN or infinite: the rows before them, and the other neighbour, stay what they were."""
    dt, nh, nk, d = R.DTYPES[dtype], 2, 1, 64
    lens = (70, 45, 50)
    starts = [0, 70, 115, 165]
    _, (q, k, v) = make(dt, nh, nk, d, 165)
    k, v = k.clone(), v.clone()
    clean = B.he_packed_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts))
    v[40:70:3], k[41:70:5] = bad, bad
    k[70:115], v[70:115] = bad, bad
    got = B.he_packed_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts))
    assert torch.isfinite(got[:40]).all() and torch.isfinite(got[115:]).all()
    tol = 4 * (R.half_step(dt) + weight_step(dt) + 1e-5)  # the same sums, perhaps taken another way; values of a few units
    assert (got[:40].float() - clean[:40].float()).abs().max() <= tol * 4 and torch.equal(got[115:], clean[115:])
    assert not torch.isfinite(got[40:70]).any()
    # one bad value in one dimension: the other dimensions of the rows that see it are as before
    _, (q, k, v) = make(dt, nh, nk, d, 165)
    v = v.clone()
    v[20, 0, 7] = bad
    got = B.he_packed_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts))
    other = [i for i in range(d) if i != 7]
    assert torch.isfinite(got[:20]).all() and torch.isfinite(got[20:, :, other]).all() and not torch.isfinite(got[20:70, :, 7]).any()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_rows_of_no_sequence_and_wider_rows(dtype):
    dt, nh, nk, d = R.DTYPES[dtype], 4, 2, 64
    _, (q, k, v) = make(dt, nh, nk, d, 200)
    starts = [5, 5, 60, 190]
    wide = torch.full((200, nh * d + 48), 9.0, dtype=dt).cuda()
    B.he_packed_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts), out=wide[:, 16:16 + nh * d].unflatten(1, (nh, d)), scale=0.3)
    got = wide.cpu()
    check(got[:, 16:16 + nh * d].unflatten(1, (nh, d)), q, k, v, starts, dt, True, 0.3)
    assert (got[:5] == 9).all() and (got[190:] == 9).all() and (got[:, :16] == 9).all() and (got[:, 16 + nh * d:] == 9).all()


def test_no_rows_and_many_sequences():
    q = torch.zeros(0, 2, 64, device="cuda")
    assert B.he_packed_attention(q, q, q, ints([0])).shape == (0, 2, 64)
    g = torch.Generator().manual_seed(9)
    lens = torch.randint(0, 4, (3000,), generator=g)
    starts = [0] + lens.cumsum(0).tolist()
    _, (q, k, v) = make(torch.float16, 2, 1, 64, starts[-1], seed=2)
    got = B.he_packed_attention(q.cuda(), k.cuda(), v.cuda(), ints(starts)).cpu()
    pick = list(range(0, 3000, 97))
    for b in pick:
        check(got, q, k, v, starts[b:b + 2], torch.float16, True, 64 ** -0.5)
    assert torch.isfinite(got).all()


def test_repeats_bit_for_bit_and_replays():
    _, (q, k, v) = make(torch.bfloat16, 8, 2, 128, 777)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    starts = ints([0, 300, 301, 777])
    first = B.he_packed_attention(q, k, v, starts)
    side = torch.cuda.Stream()
    out = torch.empty_like(first)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        B.he_packed_attention(q, k, v, starts, out=out)
    for s in ([0, 300, 301, 777], [0, 1, 2, 3], [0, 777, 777, 777], [10, 100, 500, 600]):
        starts.copy_(ints(s))
        out.fill_(5.0)
        torch.cuda.synchronize()
        g.replay()
        want = torch.full_like(out, 5.0)
        B.he_packed_attention(q, k, v, starts, out=want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    starts.copy_(ints([0, 300, 301, 777]))
    assert torch.equal(B.he_packed_attention(q, k, v, starts), first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-0.3, 0.0])
def test_scales_that_turn_or_level_the_scores(dtype, scale):
    dt = R.DTYPES[dtype]
    _, (q, k, v) = make(dt, 4, 2, 64, 90)
    got = B.he_packed_attention(q.cuda(), k.cuda(), v.cuda(), ints([0, 70, 90]), scale=scale)
    check(got.cpu(), q, k, v, [0, 70, 90], dt, True, scale)
    pages = torch.randperm(12, generator=torch.Generator().manual_seed(1)).int().view(2, 6)
    kp, vp = (torch.zeros(12, 2, 16, 64, dtype=dt).cuda() for _ in range(2))
    B.he_paged_append(k.cuda(), v.cuda(), kp, vp, pages.cuda(), ints([0, 0]), seq_starts=ints([0, 70, 90]))
    got = B.he_paged_attention(q[[69, 89]].cuda(), kp, vp, pages.cuda(), ints([70, 20]), scale=scale).cpu()
    for i, (a, b) in enumerate(((0, 70), (70, 90))):
        want, mag, most = R.attend(q[b - 1:b], k[a:b], v[a:b], scale)
        R.check_attended(got[i:i + 1], want, mag, most, b - a, dt, 2.0 ** -16)
