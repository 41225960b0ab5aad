"""he_paged_append against its definition in 64 bits: rows into pages, keys and queries rotated."""
import pytest
import torch

from paper_2308_01320_amd import binding as B
from tests import operators_ref as R

pytestmark = pytest.mark.gpu


def make(dt, nh, nk, d, page, before, new, seed=0, spare=1, page_gap=0):
    """A pool of pages full of numbers, a table in no order, and rows side by side as the fused weights leave them."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-(a + b) // page) for a, b in zip(before, new)]
    table = torch.full((len(new), max(need) + spare), -1, dtype=torch.int32)
    order = torch.randperm(sum(need) + 2, generator=g).int()
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    pool = torch.randn(sum(need) + 2, 2, nk * page * d + page_gap, generator=g).to(dt)
    qkv = torch.randn(sum(new), (nh + 2 * nk) * d, generator=g).to(dt)
    return table, pool, qkv


def split(qkv, nh, nk, d):
    return (t.view(qkv.shape[0], -1, d) for t in qkv.split([nh * d, nk * d, nk * d], 1))


def pages_of(pool, nk, page, d):
    n = nk * page * d
    return (pool[:, i, :n].unflatten(1, (nk, page, d)) for i in (0, 1))


def expect(table, pool, k_rot, v, before, new, nk, page, d):
    """The pool afterwards, K in float64."""
    kp, vp = (t.double().clone() for t in pages_of(pool, nk, page, d))
    i = 0
    for b, n in enumerate(new):
        for t in range(before[b], before[b] + n):
            if t >= 0 and t // page < table.shape[1] and 0 <= int(table[b, t // page]) < pool.shape[0]:
                p = int(table[b, t // page])
                kp[p, :, t % page], vp[p, :, t % page] = k_rot[i], v[i].double()
            i += 1
    return kp, vp


def positions(before, new):
    return torch.cat([torch.arange(a, a + n) for a, n in zip(before, new)]).long()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nh,nk,d,page,dim,inter", [
    (4, 4, 64, 16, 64, False), (8, 2, 128, 8, 128, True), (5, 1, 128, 1, 32, False), (6, 2, 80, 64, 80, False), (3, 3, 96, 4, 48, True), (2, 1, 256, 32, 256, False),
    (4, 2, 16, 2, 16, True), (40, 8, 128, 16, 128, False), (4, 2, 64, 128, None, False)])
@pytest.mark.parametrize("before,new", [((0,), (1,)), ((7, 0, 33), (20, 0, 5)), ((15, 16, 17, 1), (1, 1, 1, 1)), ((0, 3), (131, 64))])
def test_rows_go_to_their_pages(dtype, nh, nk, d, page, dim, inter, before, new):
    dt = R.DTYPES[dtype]
    table, pool, qkv = make(dt, nh, nk, d, page, before, new, page_gap=16)
    q, k, v = split(qkv, nh, nk, d)
    pos = positions(before, new)
    want_k, mag_k = R.rotate(k, pos, dim or 0, interleaved=inter)
    want_q, mag_q = R.rotate(q, pos, dim or 0, interleaved=inter)
    dev_pool, dev = pool.cuda(), qkv.cuda()
    dq, dk, dv = split(dev, nh, nk, d)
    kp, vp = pages_of(dev_pool, nk, page, d)  # K and V of a page side by side: a page stride of its own
    q_out, k_out = torch.zeros_like(q).cuda(), torch.zeros_like(k).cuda()
    starts = None
    if any(n != 1 for n in new):
        starts = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda()
    B.he_paged_append(dk, dv, kp, vp, table.cuda(), torch.tensor(before, dtype=torch.int32).cuda(), seq_starts=starts, q=dq, q_out=q_out, k_out=k_out,
                      rope=B.rope(dim, interleaved=inter) if dim else None)
    torch.cuda.synchronize()
    R.check_rotated(q_out, want_q, mag_q, dt)
    R.check_rotated(k_out, want_k, mag_k, dt)
    wk, wv = expect(table, pool, k_out.cpu().double(), v, before, new, nk, page, d)
    assert torch.equal(kp.cpu().double(), wk) and torch.equal(vp.cpu().double(), wv)  # and everything else as it was
    if page * nk:
        assert torch.equal(dev_pool[:, :, nk * page * d:].cpu(), pool[:, :, nk * page * d:])
    assert torch.equal(dev.cpu(), qkv)


@pytest.mark.parametrize("pos", [100_000, 1_000_003, 2 ** 24 + 1])
@pytest.mark.parametrize("base,scale", [(10000.0, 1.0), (500000.0, 0.25)])
def test_angles_of_far_positions(pos, base, scale):
    d, page = 128, 32768
    table = torch.full((1, pos // page + 1), -1, dtype=torch.int32)
    table[0, -1] = 0
    k = torch.randn(1, 1, d)
    kp, vp = torch.zeros(1, 1, page, d).cuda(), torch.zeros(1, 1, page, d).cuda()
    B.he_paged_append(k.cuda(), k.cuda(), kp, vp, table.cuda(), torch.tensor([pos], dtype=torch.int32).cuda(), rope=B.rope(d, base, scale))
    want, mag = R.rotate(k, torch.tensor([pos]), d, base, scale)
    R.check_rotated(kp[0, :, pos % page][None], want, mag, torch.float32)
    assert int((vp != 0).any(-1).sum()) == 1


def test_queries_and_keys_in_place():
    table, pool, qkv = make(torch.bfloat16, 8, 2, 64, 16, (5, 2), (9, 30))
    outs = []
    for in_place in (False, True):
        dev, dp = qkv.cuda(), pool.cuda()
        q, k, v = split(dev, 8, 2, 64)
        kp, vp = pages_of(dp, 2, 16, 64)
        qo, ko = (q, k) if in_place else (torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format))
        B.he_paged_append(k, v, kp, vp, table.cuda(), torch.tensor([5, 2], dtype=torch.int32).cuda(), seq_starts=torch.tensor([0, 9, 39], dtype=torch.int32).cuda(), q=q, q_out=qo,
                          k_out=ko, rope=B.rope(64))
        outs.append((qo.cpu().contiguous(), ko.cpu().contiguous(), dp.cpu()))
        if in_place:
            assert torch.equal(v.cpu(), qkv[:, 640:].view(39, 2, 64))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_rows_of_no_sequence_and_positions_of_no_page():
    """Rows before the first start and behind the last are left alone; a position past the table, before it, or under a table entry that is no page
    is rotated but not kept."""
    nk, d, page = 2, 64, 8
    table = torch.tensor([[1, -1, 2], [0, 99, -2147483648], [3, 2147483647, 4]], dtype=torch.int32)
    pool = torch.randn(5, 2, nk * page * d)
    before, new = (20, 6, -3), (7, 12, 9)  # up to 26 of 24 positions; page 99 of 5; from -3 on
    n = sum(new)
    qkv = torch.randn(n + 5, 4 * d * 2)
    q, k, v = (t.view(n + 5, -1, d) for t in qkv.split([4 * d, 2 * d, 2 * d], 1))
    starts = torch.tensor([2, 9, 21, 30], dtype=torch.int32)
    dp = pool.cuda()
    kp, vp = pages_of(dp, nk, page, d)
    q_out, k_out = torch.full((n + 5, 4, d), 7.0).cuda(), torch.full((n + 5, 2, d), 7.0).cuda()
    B.he_paged_append(k.cuda(), v.cuda(), kp, vp, table.cuda(), torch.tensor(before, dtype=torch.int32).cuda(), seq_starts=starts.cuda(), q=q.cuda(), q_out=q_out, k_out=k_out,
                      rope=B.rope(32))
    pos = positions(before, new)
    want, mag = R.rotate(q[2:30], pos, 32)
    R.check_rotated(q_out[2:30], want, mag, torch.float32)
    assert (q_out[:2] == 7).all() and (q_out[30:] == 7).all() and (k_out[:2] == 7).all() and (k_out[30:] == 7).all()
    wk, wv = expect(table, pool, k_out[2:30].cpu().double(), v[2:30], before, new, nk, page, d)
    assert torch.equal(kp.cpu().double(), wk) and torch.equal(vp.cpu().double(), wv)


def test_many_sequences_find_their_rows():
    """Five thousand sequences, most of them empty or of one row: the search over the starts takes more than two steps."""
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 3, (5000,), generator=g)
    starts = torch.cat([torch.zeros(1, dtype=torch.long), lens.cumsum(0)]).int()
    n = int(starts[-1])
    table = torch.arange(5000, dtype=torch.int32)[:, None].contiguous()
    k = torch.randn(n, 1, 16, generator=g)
    kp, vp = torch.zeros(5000, 1, 4, 16).cuda(), torch.zeros(5000, 1, 4, 16).cuda()
    B.he_paged_append(k.cuda(), k.cuda(), kp, vp, table.cuda(), torch.ones(5000, dtype=torch.int32).cuda(), seq_starts=starts.cuda())
    want = torch.zeros(5000, 1, 4, 16)
    for b in range(5000):
        for i in range(int(lens[b])):
            want[b, 0, 1 + i] = k[int(starts[b]) + i, 0]
    assert torch.equal(kp.cpu(), want) and torch.equal(vp.cpu(), want)


def test_pages_beyond_32_bits():
    """Pages whose elements lie past 2^32 of the first."""
    d, page, nk = 64, 16, 1
    stride = 3 * 2 ** 31 // 16 * 16
    base = torch.empty(stride + nk * page * d, dtype=torch.bfloat16, device="cuda")
    kp = base.as_strided((2, nk, page, d), (stride, page * d, d, 1))
    kp.zero_()
    vp = torch.empty(stride + nk * page * d, dtype=torch.bfloat16, device="cuda").as_strided((2, nk, page, d), (stride, page * d, d, 1))
    vp.zero_()
    k = torch.randn(1, 1, d).bfloat16()
    B.he_paged_append(k.cuda(), k.cuda(), kp, vp, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), torch.tensor([18], dtype=torch.int32).cuda())
    assert torch.equal(kp[1, 0, 2].cpu(), k[0, 0]) and torch.equal(vp[1, 0, 2].cpu(), k[0, 0]) and int((kp != 0).any(-1).sum()) == 1
    q = torch.randn(1, 2, d).bfloat16()
    got = B.he_paged_attention(q.cuda(), kp, vp, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), torch.tensor([19], dtype=torch.int32).cuda())
    kk = torch.zeros(19, 1, d)
    kk[18] = k[0].float()
    want, mag, most = R.attend(q, kk, kk, d ** -0.5)
    R.check_attended(got, want, mag, most, 19, torch.bfloat16, 2.0 ** -16)
