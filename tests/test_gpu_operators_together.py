"""The operators as a serving loop uses them: prompts appended and attended to, then token after token over the pages, and a token drawn from logits."""
import numpy as np
import pytest
import torch

from paper_2308_01320_amd import binding as B
from paper_2308_01320_amd import synth
from tests import operators_ref as R
from tests import util

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nh,nk,d,page", [(8, 2, 64, 16), (4, 4, 128, 8)])
def test_a_prompt_and_its_answer_attend_to_everything_before(dtype, nh, nk, d, page):
    dt, lens, steps = R.DTYPES[dtype], [23, 1, 70], 6
    B_, g = len(lens), torch.Generator().manual_seed(0)
    per = 8 if page == 16 else 16
    table = torch.randperm(B_ * per, generator=g).int().view(B_, per).cuda()
    kp, vp = (torch.zeros(B_ * per, nk, page, d, dtype=dt).cuda() for _ in range(2))
    starts = torch.tensor([0, 23, 24, 94], dtype=torch.int32).cuda()
    have = torch.zeros(B_, dtype=torch.int32).cuda()
    rope = B.rope(d)

    def fresh(n):
        qkv = torch.randn(n, (nh + 2 * nk) * d, generator=g).to(dt)
        return qkv, qkv.cuda()

    def views(t):
        return (x.view(t.shape[0], -1, d) for x in t.split([nh * d, nk * d, nk * d], 1))

    host, dev = fresh(94)
    q, k, v = views(dev)
    B.he_paged_append(k, v, kp, vp, table, have, seq_starts=starts, q=q, q_out=q, k_out=k, rope=rope)  # rotated in place
    prompt = B.he_packed_attention(q, k, v, starts)
    have += torch.tensor(lens, dtype=torch.int32).cuda()
    rot_q, rot_k = q.cpu().clone(), k.cpu().clone()
    keys = [rot_k[a:b] for a, b in ((0, 23), (23, 24), (24, 94))]
    vals = [v.cpu()[a:b] for a, b in ((0, 23), (23, 24), (24, 94))]
    hq, hk, hv = views(host)
    pos = torch.cat([torch.arange(n) for n in lens])
    R.check_rotated(rot_q, *R.rotate(hq, pos, d), dt)
    R.check_rotated(rot_k, *R.rotate(hk, pos, d), dt)
    step_w = R.half_step(dt) if dtype != "f32" else 0.0
    for b, (a, e) in enumerate(((0, 23), (23, 24), (24, 94))):
        n = e - a
        want, mag, most = R.attend(rot_q[a:e], keys[b], vals[b], d ** -0.5, torch.ones(n, n, dtype=torch.bool).tril())
        R.check_attended(prompt[a:e], want, mag, most, n, dt, step_w)
    for _ in range(steps):
        host, dev = fresh(B_)
        q, k, v = views(dev)
        q_out = torch.empty(B_, nh, d, dtype=dt).cuda()
        B.he_paged_append(k, v, kp, vp, table, have, q=q, q_out=q_out, rope=rope)
        old = have.cpu().long()
        have += 1
        out = B.he_paged_attention(q_out, kp, vp, table, have)
        hq, hk, hv = views(host)
        R.check_rotated(q_out, *R.rotate(hq, old, d), dt)
        for b in range(B_):
            p, r = int(table[b, int(old[b]) // page]), int(old[b]) % page
            new_k = kp[p, :, r].cpu()[None]
            R.check_rotated(new_k, *R.rotate(hk[b:b + 1], old[b:b + 1], d), dt)
            keys[b], vals[b] = torch.cat([keys[b], new_k]), torch.cat([vals[b], hv[b:b + 1]])
            want, mag, most = R.attend(q_out[b:b + 1].cpu(), keys[b], vals[b], d ** -0.5)
            R.check_attended(out[b:b + 1], want, mag, most, len(keys[b]), dt, 2.0 ** -16)


def test_the_last_row_of_a_prompt_is_a_step():
    """A prompt's last row, through the prompt's attention and as a single token over pages: the same to rounding."""
    dt, nh, nk, d, n = torch.bfloat16, 8, 2, 128, 333
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(n, h, d, generator=g).to(dt).cuda() for h in (nh, nk, nk))
    kp, vp = (torch.zeros(24, nk, 16, d, dtype=dt).cuda() for _ in range(2))
    table = torch.randperm(24, generator=g).int()[None].cuda()
    starts, zero, all_ = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([0, n], [0], [n]))
    B.he_paged_append(k, v, kp, vp, table, zero, seq_starts=starts)
    a = B.he_packed_attention(q, k, v, starts)[-1:].cpu()
    b = B.he_paged_attention(q[-1:], kp, vp, table, all_).cpu()
    want, mag, most = R.attend(q[-1:].cpu(), k.cpu(), v.cpu(), d ** -0.5)
    R.check_attended(a, want, mag, most, n, dt, R.half_step(dt))
    R.check_attended(b, want, mag, most, n, dt, 2.0 ** -16)


def test_tokens_drawn_from_the_engines_logits():
    """An answer of the engine with nucleus sampling: its logits through he_sample, the token back into he_decode_step."""
    d = synth.CONFIGS["tiny"]
    eng = util.make_engine(d, synth.make_weights(d, seed=3))
    prompts = torch.from_numpy(synth.make_prompts(d, seed=4)).cuda()
    rng = np.random.default_rng(5)
    n = prompts.shape[0]
    f = {"temperature": torch.full((n,), 0.8), "top_k": torch.full((n,), 40, dtype=torch.int32), "top_p": torch.full((n,), 0.9), "min_p": torch.full((n,), 0.01)}
    f = {k: v.cuda() for k, v in f.items()}
    samp = B.sampling("greedy")
    _, _, z = eng.he_prefill(prompts, samp, want_logits=True)
    for _ in range(8):
        u = rng.random(n).astype(np.float32)
        ids, lp = B.he_sample(z, torch.from_numpy(u).cuda(), **f)
        rows = z.double().cpu().numpy()
        for r in range(n):
            i, want = R.sample_row(rows[r], float(u[r]), float(np.float32(0.8)), 40, float(np.float32(0.9)), float(np.float32(0.01)))
            assert int(ids[r]) == i and abs(float(lp[r]) - want) <= 2.0 ** -23 * max(1.0, abs(want))
        _, _, z = eng.he_decode_step(ids, samp, want_logits=True)
    eng.he_destroy()
