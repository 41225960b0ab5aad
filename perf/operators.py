"""The operators of a serving loop over a paged key-value cache, as cases that can be timed and checked.

  append   he_paged_append: new tokens' keys and values go into the pages of their sequences, keys and queries rotated by their positions on the way
  decode   he_paged_attention: one new token per sequence attends to everything its sequence has in the pages
  prompt   he_packed_attention: prompts of different lengths laid end to end, causal, query heads sharing key-value heads
  sample   he_sample: a token per row of logits from a given random number, after temperature, top-k, top-p and min-p

Where `own` is false, run() computes them in elementary torch operations, in 32 bits (angles, the sums that a token is picked by and the values
next to a threshold in 64); where it is true it makes the framework's calls.  A case is a dict:

  op       one of the four;  dtype "bf16", "f16" or "f32"
  heads, kv_heads, dim (append, decode, prompt)
  seqs, longest, ragged: sequences and their lengths (positions in the cache, tokens of a prompt); page: positions to a page
  append:  new (tokens per sequence at most; 1: a decode step), rotary (rotated dimensions), interleaved, base
  sample:  rows, vocab, filtered (all four parameters, else temperature and top-p), spread (standard deviation of the logits)
"""
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases


def _append(dtype, heads, kv_heads, dim, seqs, longest, new, page, rotary, interleaved=False, base=10000.0, ragged=True):
    return {"op": "append", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "longest": longest, "ragged": ragged,
            "new": new, "page": page, "rotary": rotary, "interleaved": interleaved, "base": base}


def _decode(dtype, heads, kv_heads, dim, seqs, longest, page, ragged=True):
    return {"op": "decode", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "longest": longest, "ragged": ragged, "page": page}


def _prompt(dtype, heads, kv_heads, dim, seqs, longest, ragged=True):
    return {"op": "prompt", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "longest": longest, "ragged": ragged}


def _sample(dtype, rows, vocab, filtered, spread):
    return {"op": "sample", "dtype": dtype, "rows": rows, "vocab": vocab, "filtered": filtered, "spread": spread}


def listed():
    return [
        # the step of a batch of 32 answers: one token each, grouped heads, somewhere in pages of 16; a few hundred KB, so latency
        dict(_append("bf16", 40, 8, 128, 32, 511, 1, 16, 128), name="append_step_b32"),
        # the prompts of the headline workload, 32 of up to 256 tokens, a key-value head to every head, rotated in interleaved pairs
        dict(_append("f16", 40, 40, 128, 32, 0, 256, 64, 128, interleaved=True), name="append_prompts_b32"),
        # one user's next token with little behind it: the smallest call
        dict(_decode("f16", 32, 32, 64, 1, 77, 16), name="decode_b1_short"),
        # the headline workload's step: 32 answers of the 13B-shaped actor, a key-value head to every head
        dict(_decode("bf16", 40, 40, 128, 32, 511, 16), name="decode_b32"),
        # long documents: few sequences, a long cache in pages of 64, five query heads to a key-value head
        dict(_decode("bf16", 40, 8, 128, 4, 100003, 64), name="decode_long"),
        # the same step in float, as the float models have it
        dict(_decode("f32", 8, 2, 64, 8, 1500, 32), name="decode_f32"),
        # a single prompt of odd length: time to the first token
        dict(_prompt("f16", 32, 32, 128, 1, 250), name="prompt_b1"),
        # the headline workload's prompts, of different lengths
        dict(_prompt("bf16", 40, 40, 128, 32, 256), name="prompt_b32"),
        # one long document, four query heads to a key-value head: attention is what such a prompt costs
        dict(_prompt("bf16", 32, 8, 128, 1, 8189, ragged=False), name="prompt_long"),
        # prompts of a float model
        dict(_prompt("f32", 8, 2, 64, 4, 700), name="prompt_f32"),
        # one user's token out of the OPT vocabulary: latency
        dict(_sample("f32", 1, 50272, False, 2.5), name="sample_b1"),
        # experience generation at a large batch, logits as a 16-bit head leaves them (many of them equal), every filter in use
        dict(_sample("bf16", 256, 50272, True, 3.0), name="sample_b256"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (heads, key-value heads, head dimension): the configurations' attention, and grouped and narrower ones
_HEADS = [(32, 32, 64), (32, 32, 128), (40, 40, 128), (72, 72, 128), (40, 8, 128), (32, 4, 128), (16, 2, 128), (8, 1, 128), (4, 4, 64), (8, 2, 64),
          (10, 10, 64), (12, 3, 80), (6, 2, 96), (8, 1, 256), (20, 1, 64)]


def _draw(rng):
    op = rng.choice(("append", "decode", "decode", "prompt", "prompt", "sample"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f16", "f32"))
    heads, kv_heads, dim = rng.choice(_HEADS)
    page = 1 << rng.randint(3, 8)
    if op == "append":
        rotary = dim if rng.random() < 0.7 else 16 * rng.randint(1, dim // 16)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 4000)
        return _append(dtype, heads, kv_heads, dim, _log_int(rng, 1, 256 if new == 1 else 40), _log_int(rng, 1, 2000) if rng.random() < 0.7 else 0, new, page,
                       rotary, rng.random() < 0.4, rng.choice((10000.0, 500000.0)))
    if op == "decode":
        return _decode(dtype, heads, kv_heads, dim, _log_int(rng, 1, 200), _log_int(rng, 1, 120000), page)
    if op == "prompt":
        return _prompt(dtype, heads, kv_heads, dim, _log_int(rng, 1, 48), _log_int(rng, 1, 8000), ragged=rng.random() < 0.8)
    return _sample(dtype, _log_int(rng, 1, 256), _log_int(rng, 100, 131072), rng.random() < 0.6, rng.uniform(1.0, 4.0))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        b, f = most.get(c["op"], (0.0, 0.0))
        most[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    while True:
        c = _draw(rng)
        w = work(c)
        b, f = most[c["op"]]
        if c["op"] == "prompt" and c["dtype"] == "f32":
            f /= 16  # (what the matrix cores do in float they do in 16 bits sixteen times as fast)
        # (padded to the longest, the scores of a batch of prompts are what the plain form holds in memory)
        if w["bytes"] <= b and w["flops"] <= f and (c["op"] != "prompt" or c["seqs"] * c["heads"] * c["longest"] ** 2 <= 3e9):
            return c


# ------------------------------------------------------------------ inputs


def _lengths(case, longest):
    """Lengths of the case's sequences, the first the longest; they belong to the case, not to the seed."""
    r = random.Random(case["seqs"] * 100003 + longest)
    return [longest] + [r.randint((longest + 2) // 3, longest) if case["ragged"] else longest for _ in range(case["seqs"] - 1)]


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _pages(case, g, lens):
    """K and V pages in a pool with some to spare, and the table that says which belong to whom, in no order; unused entries of it are -1."""
    dev, page = _device(), case["page"]
    used = [-(-n // page) for n in lens]
    per_seq = max(max(used), 1) + 1
    n_pages = sum(used) + 3
    table = torch.full((len(lens), per_seq), -1, dtype=torch.int32, device=dev)
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (n_pages, case["kv_heads"], page, case["dim"])
    k, v = (torch.randn(shape, generator=g, device=dev).to(_TYPES[case["dtype"]]) for _ in range(2))
    return k, v, table


def prepare(case, seed):
    dev, dt = _device(), _TYPES[case["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=dev)

    state = {"case": case}
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        z = torch.randn(rows, vocab, generator=g, device=dev) * case["spread"]
        # a few tokens that the context calls for
        z.scatter_add_(1, torch.randint(0, vocab, (rows, 8), generator=g, device=dev), torch.rand(rows, 8, generator=g, device=dev) * 4 * case["spread"])

        def between(lo, hi):
            return torch.rand(rows, generator=g, device=dev) * (hi - lo) + lo

        state |= {"logits": z.to(dt), "uniform": torch.rand(rows, generator=g, device=dev), "temperature": between(0.6, 1.3), "top_p": between(0.8, 1.0),
                  "top_k": None, "min_p": None}
        if case["filtered"]:
            state |= {"top_k": torch.randint(0, min(vocab, 2000), (rows,), generator=g, device=dev, dtype=torch.int32), "min_p": between(0.0, 0.05)}
        return state
    nh, nk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "decode":
        lens = _lengths(case, case["longest"])
        k, v, table = _pages(case, g, lens)
        q = torch.randn(case["seqs"], nh, d, generator=g, device=dev).to(dt)
        return state | {"q": q, "k_pages": k, "v_pages": v, "pages": table, "lens": ints(lens), "max_len": max(lens), "out": torch.empty_like(q)}
    # rows as the product with the fused weights leaves them: queries, keys and values side by side
    new = _lengths(case, case["new"] if case["op"] == "append" else case["longest"])
    n = sum(new)
    qkv = torch.randn(n, (nh + 2 * nk) * d, generator=g, device=dev).to(dt)
    q, k, v = (t.view(n, -1, d) for t in qkv.split([nh * d, nk * d, nk * d], dim=1))
    starts = ints([sum(new[:b]) for b in range(len(new) + 1)])
    state |= {"qkv": qkv, "q": q, "k": k, "v": v, "seq_starts": starts, "q_out": torch.empty(n, nh, d, dtype=dt, device=dev)}
    if case["op"] == "append":
        before = _lengths(case, case["longest"])
        kp, vp, table = _pages(case, g, [a + b for a, b in zip(before, new)])
        state |= {"k_pages": kp, "v_pages": vp, "pages": table, "lens": ints(before)}
        if case["new"] == 1:
            state["seq_starts"] = None  # a token per sequence
    return state


# ------------------------------------------------------------------ the plain form


def _rotated(x, pos, case):
    """x [n, heads, d] with its first `rotary` dimensions turned by pos * base^(-2 i / rotary) in pair i."""
    r, half = case["rotary"], case["rotary"] // 2
    angle = pos.double()[:, None] * (case["base"] ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half))
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y = x.float().clone()
    if case["interleaved"]:
        a, b = x[..., 0:r:2].float(), x[..., 1:r:2].float()
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., :half].float(), x[..., half:r].float()
        y[..., :half], y[..., half:r] = a * c - b * s, a * s + b * c
    return y.to(x.dtype)


def _plain_append(s):
    case, page = s["case"], s["case"]["page"]
    n = s["q"].shape[0]
    tok = torch.arange(n, device=s["q"].device)
    if s["seq_starts"] is None:
        seq, pos = tok, s["lens"].long()
    else:
        seq = torch.bucketize(tok, s["seq_starts"][1:].long(), right=True)
        pos = s["lens"].long()[seq] + tok - s["seq_starts"].long()[seq]
    at, row = s["pages"].long()[seq, pos // page], pos % page
    s["q_out"].copy_(_rotated(s["q"], pos, case))
    s["k_pages"][at, :, row] = _rotated(s["k"], pos, case)
    s["v_pages"][at, :, row] = s["v"]
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _softmax(scores, seen):
    scores = torch.where(seen, scores, -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _plain_decode(s):
    q, page = s["q"], s["case"]["page"]
    b, nh, d = q.shape
    nk = s["case"]["kv_heads"]
    used = -(-s["max_len"] // page)
    at = s["pages"][:, :used].long().clamp_min(0)
    # [sequence, key-value head, position, dimension]
    k, v = (p[at].transpose(1, 2).reshape(b, nk, used * page, d).float() for p in (s["k_pages"], s["v_pages"]))
    seen = (torch.arange(used * page, device=q.device) < s["lens"][:, None])[:, None, None]
    scores = torch.matmul(q.float().reshape(b, nk, nh // nk, d), k.transpose(2, 3).contiguous()) * d ** -0.5
    return torch.matmul(_softmax(scores, seen), v).reshape(b, nh, d).to(q.dtype)


def _plain_prompt(s):
    q, starts = s["q"], s["seq_starts"].long()
    n, nh, d = q.shape
    nk, longest, seqs = s["case"]["kv_heads"], s["case"]["longest"], s["case"]["seqs"]
    t = torch.arange(longest, device=q.device)
    real = t < (starts[1:] - starts[:-1])[:, None]
    at = torch.where(real, starts[:-1, None] + t, 0)
    # padded to the longest: [sequence, key-value head, position (times the heads that share it), dimension]
    k, v = (x[at].transpose(1, 2).float().contiguous() for x in (s["k"], s["v"]))
    qp = q[at].view(seqs, longest, nk, nh // nk, d).permute(0, 2, 3, 1, 4).float().reshape(seqs, nk, nh // nk * longest, d)
    scores = torch.matmul(qp, k.transpose(2, 3).contiguous()).mul_(d ** -0.5).view(seqs, nk, nh // nk, longest, longest)
    p = _softmax(scores, t[None, :] <= t[:, None]).view(seqs, nk, nh // nk * longest, longest)
    o = torch.matmul(p, v).view(seqs, nk, nh // nk, longest, d).permute(0, 3, 1, 2, 4).reshape(seqs, longest, nh, d)
    return o[real].to(q.dtype)


def _plain_sample(s):
    z = s["logits"].double()
    rows, vocab = z.shape
    top, ids = torch.sort(z, dim=1, descending=True, stable=True)  # equal logits: the lower id first
    w = torch.exp((top - top[:, :1]) / s["temperature"].double()[:, None])
    upto = torch.cumsum(w, 1)
    rank = torch.arange(vocab, device=z.device)[None]
    k = torch.full((rows, 1), vocab, device=z.device) if s["top_k"] is None else s["top_k"].long()[:, None]
    k = torch.where((k <= 0) | (k > vocab), vocab, k)
    keep = (rank < k) & (upto - w < s["top_p"].double()[:, None] * upto.gather(1, k - 1))
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    keep |= rank == 0
    kept = torch.zeros_like(w).scatter_(1, ids, torch.where(keep, w, 0.0))
    upto = torch.cumsum(kept, 1)
    goal = s["uniform"].double()[:, None] * upto[:, -1:]
    last = torch.where(kept > 0, torch.arange(vocab, device=z.device)[None], -1).amax(1)
    chosen = torch.minimum((upto <= goal).sum(1), last)
    logprob = z.gather(1, chosen[:, None])[:, 0] - top[:, 0] - torch.log(torch.exp(top - top[:, :1]).sum(1))
    return {"ids": chosen.to(torch.int32), "logprobs": logprob.float()}


# ------------------------------------------------------------------ one pass


def run(state):
    op, case = state["case"]["op"], state["case"]
    if own:
        from paper_2308_01320_amd import binding

        if op == "append":
            binding.he_paged_append(state["k"], state["v"], state["k_pages"], state["v_pages"], state["pages"], state["lens"], seq_starts=state["seq_starts"],
                                    q=state["q"], q_out=state["q_out"], rope=binding.rope(case["rotary"], case["base"], interleaved=case["interleaved"]))
            return {"q": state["q_out"], "k_pages": state["k_pages"], "v_pages": state["v_pages"]}
        if op == "decode":
            return binding.he_paged_attention(state["q"], state["k_pages"], state["v_pages"], state["pages"], state["lens"], max_len=state["max_len"], out=state["out"])
        if op == "prompt":
            return binding.he_packed_attention(state["q"], state["k"], state["v"], state["seq_starts"], out=state["q_out"])
        ids, logprobs = binding.he_sample(state["logits"], state["uniform"], temperature=state["temperature"], top_k=state["top_k"], top_p=state["top_p"],
                                          min_p=state["min_p"])
        return {"ids": ids, "logprobs": logprobs}
    return {"append": _plain_append, "decode": _plain_decode, "prompt": _plain_prompt, "sample": _plain_sample}[op](state)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    el = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "sample":
        values = case["rows"] * case["vocab"]
        # read once; of every value a difference, a product and an exponential, twice (at the temperature, and without it), and the sums
        return {"bytes": float(values * el + case["rows"] * 28), "flops": float(values * 8)}
    nh, nk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "decode":
        lens = _lengths(case, case["longest"])
        return {"bytes": float(sum(lens) * 2 * nk * d * el + len(lens) * 2 * nh * d * el + sum(-(-n // case["page"]) for n in lens) * 4),
                "flops": 4.0 * sum(lens) * nh * d}
    if case["op"] == "prompt":
        lens = _lengths(case, case["longest"])
        return {"bytes": float(sum(lens) * 2 * (nh + nk) * d * el), "flops": 2.0 * sum(n * (n + 1) for n in lens) * nh * d}
    n = sum(_lengths(case, case["new"]))
    # queries, keys and values, in and out; three operations to a rotated value
    return {"bytes": float(n * 2 * (nh + 2 * nk) * d * el), "flops": 3.0 * n * (nh + nk) * case["rotary"]}


# ------------------------------------------------------------------ the same in 64 bits


def _exact_turn(x, pos, case):
    """Pairs as complex numbers, multiplied by exp(i pos base^(-2 i / rotary))."""
    r = case["rotary"]
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device=x.device),
                       torch.outer(pos, torch.exp(torch.arange(0, r, 2, dtype=torch.float64, device=x.device) * (-math.log(case["base"]) / r))))[:, None]
    y = x.double().clone()
    part = y[..., :r].reshape(*y.shape[:2], r // 2, 2) if case["interleaved"] else y[..., :r].reshape(*y.shape[:2], 2, r // 2).transpose(2, 3)
    part = torch.view_as_real(torch.complex(part[..., 0].contiguous(), part[..., 1].contiguous()) * turn)
    y[..., :r] = (part if case["interleaved"] else part.transpose(2, 3)).reshape(*y.shape[:2], r)
    return y


def _exact_append(s):
    case, page = s["case"], s["case"]["page"]
    starts = list(range(len(s["lens"]) + 1)) if s["seq_starts"] is None else s["seq_starts"].tolist()
    before, table = s["lens"].tolist(), s["pages"].tolist()
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    pos = torch.cat([torch.arange(m, m + b - a, dtype=torch.float64, device=kp.device) for m, a, b in zip(before, starts, starts[1:])])
    q, k = _exact_turn(s["q"], pos, case), _exact_turn(s["k"], pos, case)
    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        t = a
        while t < b:  # a page at a time
            p, row = divmod(before[i] + t - a, page)
            m = min(page - row, b - t)
            kp[table[i][p], :, row:row + m] = k[t:t + m].transpose(0, 1)
            vp[table[i][p], :, row:row + m] = s["v"][t:t + m].double().transpose(0, 1)
            t += m
    return {"q": q, "k_pages": kp, "v_pages": vp}


def _exact_attention(q, k, v, causal):
    """One sequence: q [m, heads, d], k and v [n, kv heads, d], in 64 bits, a head at a time."""
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    share = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        z = (q[:, h].double() / math.sqrt(q.shape[2])) @ k[:, h // share].double().t().contiguous()
        if causal:
            z.masked_fill_(torch.ones(z.shape, dtype=torch.bool, device=z.device).triu_(1), -math.inf)
        out[:, h] = torch.softmax(z, 1) @ v[:, h // share].double()
    return out


def _exact_sample(s):
    z = s["logits"].double().cpu().numpy()
    rows, vocab = z.shape
    get = {k: None if s[k] is None else s[k].double().cpu().numpy() for k in ("uniform", "temperature", "top_k", "top_p", "min_p")}
    ids, lps = np.empty(rows, np.int32), np.empty(rows)
    for r in range(rows):
        zr = z[r] - z[r].max()
        w = np.exp(zr / get["temperature"][r])
        order = np.lexsort((np.arange(vocab), -zr))
        n = vocab if get["top_k"] is None or not 0 < get["top_k"][r] <= vocab else int(get["top_k"][r])
        sums = np.cumsum(w[order[:n]])
        n = min(n, int(np.searchsorted(sums, get["top_p"][r] * sums[-1])) + 1)
        if get["min_p"] is not None:
            n = min(n, max(1, int((w >= get["min_p"][r]).sum())))
        kept = np.sort(order[:n])
        sums = np.cumsum(w[kept])
        ids[r] = kept[min(n - 1, int(np.searchsorted(sums, get["uniform"][r] * sums[-1], side="right")))]
        lps[r] = zr[ids[r]] - np.log(np.exp(zr).sum())
    return {"ids": torch.from_numpy(ids), "logprobs": torch.from_numpy(lps)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "sample":
        return _exact_sample(s)
    if case["op"] == "decode":
        out = []
        for b, n in enumerate(s["lens"].tolist()):
            at = s["pages"][b, :-(-n // case["page"])].long()
            k, v = (p[at].transpose(1, 2).reshape(-1, case["kv_heads"], case["dim"])[:n] for p in (s["k_pages"], s["v_pages"]))
            out.append(_exact_attention(s["q"][b:b + 1], k, v, False))
        return torch.cat(out)
    starts = s["seq_starts"].tolist()
    return torch.cat([_exact_attention(s["q"][a:b], s["k"][a:b], s["v"][a:b], True) for a, b in zip(starts, starts[1:])])
