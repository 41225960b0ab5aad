"""he_paged_attention against its definition in 64 bits."""
import pytest
import torch

from paper_2308_01320_amd import binding as B
from tests import operators_ref as R

pytestmark = pytest.mark.gpu

# A weight multiplies its value as two terms of the type at least (or in float): 2^-16 of it is lost at most with bf16
WEIGHT_STEP = 2.0 ** -16


def build(dt, nk, d, page, lens, capacity=None, seed=0, fill=float("nan")):
    """Keys and values [len, nk, d] of each sequence, pages that hold them in no order and `fill` everywhere else, the table."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(n, 0) // page) for n in lens]
    width = max(max(need), 1) + 1 if capacity is None else capacity
    order = torch.randperm(sum(need) + 2, generator=g)
    table = torch.full((len(lens), width), -7, dtype=torch.int32)
    kp, vp = (torch.full((sum(need) + 2, nk, page, d), fill, dtype=dt) for _ in range(2))
    ks, vs, at = [], [], 0
    for b, n in enumerate(lens):
        k, v = (torch.randn(max(n, 0), nk, d, generator=g).to(dt) for _ in range(2))
        ks.append(k), vs.append(v)
        for i in range(need[b]):
            p = int(order[at + i])
            m = min(page, n - i * page)
            kp[p, :, :m], vp[p, :, :m] = k[i * page:i * page + m].transpose(0, 1), v[i * page:i * page + m].transpose(0, 1)
            table[b, i] = p
        at += need[b]
    return ks, vs, kp, vp, table


def check(got, q, ks, vs, dt, scale):
    for b in range(q.shape[0]):
        want, mag, most = R.attend(q[b:b + 1], ks[b], vs[b], scale)
        R.check_attended(got[b:b + 1], want, mag, most, len(ks[b]), dt, WEIGHT_STEP)


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nh,nk,d,page", [(4, 4, 64, 16), (8, 2, 128, 8), (5, 1, 128, 1), (6, 2, 80, 64), (3, 1, 96, 4), (8, 1, 256, 32), (2, 2, 16, 2), (20, 1, 64, 256), (34, 2, 128, 16),
                                          (2, 1, 112, 16), (2, 2, 208, 128)])
@pytest.mark.parametrize("lens,max_len", [((1, 0, 77), 0), ((16, 64, 65, 63), 64), ((129, 300, 2, 31, 1), 4000)])
def test_matches_the_definition(dtype, nh, nk, d, page, lens, max_len):
    """Lengths from none on, pages that end inside a tile, whatever the launch is shaped for; rows of a page behind the length hold NaN."""
    dt = R.DTYPES[dtype]
    ks, vs, kp, vp, table = build(dt, nk, d, page, lens)
    q = torch.randn(len(lens), nh, d, generator=torch.Generator().manual_seed(1)).to(dt)
    got = B.he_paged_attention(q.cuda(), kp.cuda(), vp.cuda(), table.cuda(), ints(lens), max_len=max_len)
    check(got.cpu(), q, ks, vs, dt, d ** -0.5)
    for b, n in enumerate(lens):
        if n == 0:
            assert (got[b] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nh,nk,d,page,lens", [(8, 2, 128, 16, (4999, 17)), (2, 2, 64, 64, (9001,)), (32, 8, 64, 32, (1500, 2047, 640))])
def test_long_caches_are_split(dtype, nh, nk, d, page, lens):
    dt = R.DTYPES[dtype]
    ks, vs, kp, vp, table = build(dt, nk, d, page, lens, seed=4)
    q = torch.randn(len(lens), nh, d, generator=torch.Generator().manual_seed(5)).to(dt)
    args = (q.cuda(), kp.cuda(), vp.cuda(), table.cuda(), ints(lens))
    outs = [B.he_paged_attention(*args, max_len=m) for m in (0, 1, 300, 5000)]  # one workgroup to a head, and many
    for o in outs:
        check(o.cpu(), q, ks, vs, dt, d ** -0.5)
    again = B.he_paged_attention(*args, max_len=5000)
    assert torch.equal(again, outs[3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores in the hundreds, one of them far above the rest and at the end: the running maximum moves late and far."""
    dt = R.DTYPES[dtype]
    ks, vs, kp, vp, table = build(dt, 2, 64, 16, (700,), seed=6)
    q = (torch.randn(1, 4, 64, generator=torch.Generator().manual_seed(7)) * 20).to(dt)
    kp[table[0, 690 // 16], :, 690 % 16] = (q[0, ::2] / 4).to(dt)
    ks[0][690] = (q[0, ::2] / 4).to(dt)
    got = B.he_paged_attention(q.cuda(), kp.cuda(), vp.cuda(), table.cuda(), ints((700,)), scale=0.5)
    check(got.cpu(), q, ks, vs, dt, 0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_that_are_none(dtype):
    """A table entry outside the pool takes its positions out; a sequence of nothing else gets zeros.  Lengths past the table count up to its end."""
    dt = R.DTYPES[dtype]
    lens = (50, 40, 24, 64)
    ks, vs, kp, vp, table = build(dt, 2, 64, 8, lens, capacity=8, seed=8)
    table[0, 2], table[0, 5], table[1, :] = -1, kp.shape[0], 2 ** 31 - 1
    table[2, 0] = -2 ** 31
    keep = [torch.tensor([t for t in range(50) if t // 8 not in (2, 5)]), torch.tensor([], dtype=torch.long), torch.arange(8, 24), torch.arange(64)]
    q = torch.randn(4, 4, 64).to(dt)
    got = B.he_paged_attention(q.cuda(), kp.cuda(), vp.cuda(), table.cuda(), ints((50, 40, 24, 2 ** 31 - 1)), max_len=0).cpu()
    check(got, q, [k[i] for k, i in zip(ks, keep)], [v[i] for v, i in zip(vs, keep)], dt, 64 ** -0.5)
    assert (got[1] == 0).all()


def test_negative_lengths_are_none():
    ks, vs, kp, vp, table = build(torch.float16, 1, 64, 8, (5, 9))
    got = B.he_paged_attention(torch.randn(2, 2, 64).half().cuda(), kp.cuda(), vp.cuda(), table.cuda(), ints((-2 ** 31, -1)))
    assert (got == 0).all()


def test_rows_in_wider_matrices_and_shared_pages():
    """Queries and results inside wider rows, K and V in one pool, two sequences that share their first pages."""
    dt, nh, nk, d, page = torch.float16, 6, 3, 64, 16
    ks, vs, kp, vp, table = build(dt, nk, d, page, (40, 40))
    table[1, :2] = table[0, :2]
    ks[1], vs[1] = torch.cat([ks[0][:32], ks[1][32:]]), torch.cat([vs[0][:32], vs[1][32:]])
    pool = torch.stack([kp, vp], 1).cuda()
    wide = torch.randn(2, nh * d + 200).half()
    out = torch.full((2, nh * d + 72), 3.0, dtype=dt).cuda()
    q = wide[:, 8:8 + nh * d].unflatten(1, (nh, d))
    dev = wide.cuda()
    B.he_paged_attention(dev[:, 8:8 + nh * d].unflatten(1, (nh, d)), pool[:, 0], pool[:, 1], table.cuda(), ints((40, 40)), out=out[:, 16:16 + nh * d].unflatten(1, (nh, d)))
    got = out.cpu()
    check(got[:, 16:16 + nh * d].unflatten(1, (nh, d)), q, ks, vs, dt, d ** -0.5)
    assert (got[:, :16] == 3).all() and (got[:, 16 + nh * d:] == 3).all()


def test_on_another_stream_and_captured():
    """Two captured graphs with workspaces of their own, replayed in turn with other lengths and contents, and eager calls in between."""
    dt, nh, nk, d, page = torch.bfloat16, 8, 2, 128, 16
    ks, vs, kp, vp, table = build(dt, nk, d, page, (900, 333), capacity=64, fill=0.0)
    side = torch.cuda.Stream()
    dev = [t.cuda() for t in (kp, vp, table)]
    q = torch.randn(2, nh, d).to(dt).cuda()
    lens = ints((900, 333))
    torch.cuda.synchronize()
    graphs, outs = [], []
    with torch.cuda.stream(side):
        B.he_paged_attention(q, *dev, lens)  # (code is loaded before the capture)
        for _ in range(2):
            ws = torch.empty(B.he_paged_attention_workspace(*dev, nh), dtype=torch.uint8, device="cuda")
            out = torch.empty_like(q)
            side.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                B.he_paged_attention(q, *dev, lens, out=out, workspace=ws)
            graphs.append((g, ws)), outs.append(out)
    torch.cuda.synchronize()
    for step, (a, b) in enumerate(((900, 333), (5, 0), (64, 321), (899, 1))):
        lens.copy_(ints((a, b)))
        q.copy_(torch.randn(2, nh, d).to(dt))
        torch.cuda.synchronize()
        eager = B.he_paged_attention(q, *dev, lens)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], eager) and torch.equal(outs[1], eager), step
        check(eager.cpu(), q.cpu(), [ks[0][:a], ks[1][:b]], [vs[0][:a], vs[1][:b]], dt, d ** -0.5)


def test_calls_on_two_streams_at_once():
    dt, nh, nk, d, page = torch.float16, 8, 8, 64, 16
    ks, vs, kp, vp, table = build(dt, nk, d, page, (3000,))
    dev = [t.cuda() for t in (kp, vp, table)]
    qs = [torch.randn(1, nh, d).to(dt).cuda() for _ in range(2)]
    lens = ints((3000,))
    want = [B.he_paged_attention(q, *dev, lens) for q in qs]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(B.he_paged_attention(qs[i], *dev, lens))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in (0, 1) for o in outs[i])
