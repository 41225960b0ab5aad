"""The operators of a serving loop: what they refuse, on the host, before anything touches a GPU.  (Pointers are numbers that no call here follows.)"""
import ctypes as C

import pytest

from paper_2308_01320_amd import binding as B

P = 1 << 20  # "device memory", on a 16-byte boundary


def cache(**kw):
    c = B.he_paged_cache(P, P, P, B.HE_BF16, 2, 64, 16, 8, 4, 2 * 16 * 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(data=P, stride=512):
    return B.he_rows(data, stride)


def append(c=None, rope=None, q=None, heads=0, q_out=None, k=None, k_out=None, v=None, starts=P, lens=P, seqs=2, n=5):
    return B.lib().he_paged_append(cache() if c is None else c, rope, q, heads, q_out, rows() if k is None else k, k_out, rows() if v is None else v, starts,
                                   lens, seqs, n, None)


def paged(c=None, q=None, heads=4, out=None, lens=P, seqs=2, max_len=64, scale=0.125, ws=P, nbytes=1 << 30):
    return B.lib().he_paged_attention(cache() if c is None else c, rows() if q is None else q, heads, rows() if out is None else out, lens, seqs, max_len, scale, ws,
                                      nbytes, None)


def packed(dtype=B.HE_F16, q=None, heads=4, k=None, v=None, kv=2, d=64, out=None, starts=P, seqs=2, n=5, causal=1, scale=0.125):
    return B.lib().he_packed_attention(dtype, rows() if q is None else q, heads, rows() if k is None else k, rows() if v is None else v, kv, d,
                                       rows() if out is None else out, starts, seqs, n, causal, scale, None)


def sample(dtype=B.HE_F32, z=None, n=2, vocab=100, f=None, u=P, ids=P, lp=P, ws=P, nbytes=1 << 30):
    return B.lib().he_sample(dtype, rows() if z is None else z, n, vocab, f, u, ids, lp, ws, nbytes, None)


BAD_CACHES = [
    (dict(k=None), 1), (dict(v=None), 1), (dict(pages=None), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(n_kv_heads=0), 2), (dict(head_dim=72), 2), (dict(head_dim=0), 2),
    (dict(head_dim=272), 2), (dict(page_size=0), 2), (dict(page_size=24), 2), (dict(page_size=65536), 2), (dict(n_pages=0), 1), (dict(pages_per_seq=0), 1),
    (dict(pages_per_seq=1 << 27), 2), (dict(page_stride=2047), 2), (dict(page_stride=2052), 2), (dict(k=P + 8), 2), (dict(v=P + 2), 2)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_caches_that_are_refused(bad, status):
    assert paged(cache(**bad)) == status and B.lib().he_operator_error()
    assert append(cache(**bad)) == status
    assert B.lib().he_paged_attention_workspace(cache(**bad), 4, 2, 0) == 0


def test_null_arguments_are_refused():
    L = B.lib()
    assert L.he_paged_append(None, None, None, 0, None, rows(), None, rows(), P, P, 2, 5, None) == 1
    assert L.he_paged_attention(None, rows(), 4, rows(), P, 2, 64, 0.1, None, 0, None) == 1
    assert L.he_paged_attention_workspace(None, 4, 2, 0) == 0
    assert append(k=rows(None)) == append(v=rows(None)) == append(lens=None) == 1
    assert append(q=rows(), heads=4) == append(q_out=rows(), heads=4) == 1  # one without the other
    assert paged(q=rows(None)) == paged(out=rows(None)) == paged(lens=None) == 1
    assert packed(q=rows(None)) == packed(k=rows(None)) == packed(v=rows(None)) == packed(out=rows(None)) == packed(starts=None) == 1
    assert sample(z=rows(None)) == sample(u=None) == sample(ids=None) == sample(lp=None) == 1


def test_append_refuses():
    assert append(seqs=-1) == append(n=-1) == 1
    assert append(starts=None, seqs=2, n=5) == 1
    assert b"5 rows, 2 sequences" in B.lib().he_operator_error()
    assert append(seqs=65536, n=65536) == 2 and append(n=(1 << 23) + 1) == 2
    assert append(k=rows(P + 4)) == append(k=rows(stride=129)) == append(v=rows(stride=-8)) == 2
    assert append(k_out=rows(stride=120)) == 2  # rows that would overlap
    assert append(q=rows(), q_out=rows(), heads=3) == 2
    for r, status in ((B.he_rope(8, 0, 1e4, 1.0), 2), (B.he_rope(80, 0, 1e4, 1.0), 2), (B.he_rope(24, 0, 1e4, 1.0), 2), (B.he_rope(64, 2, 1e4, 1.0), 1), (B.he_rope(64, 0, 0.0, 1.0), 1),
                      (B.he_rope(64, 0, float("nan"), 1.0), 1), (B.he_rope(64, 0, 1e4, float("inf")), 1)):
        assert append(rope=r) == status
    assert append(seqs=0, n=0) == 0 and append(seqs=0, n=5) == 0 and append(n=0) == 0  # nothing to do, nothing launched


def test_paged_attention_refuses():
    assert paged(heads=3) == paged(heads=0) == paged(q=rows(P + 2)) == paged(out=rows(stride=248)) == paged(out=rows(stride=260)) == paged(seqs=65536) == 2
    assert paged(seqs=-1) == paged(scale=float("nan")) == paged(scale=float("inf")) == 1
    need = B.lib().he_paged_attention_workspace(cache(pages_per_seq=1024, n_pages=4096), 4, 1, 0)
    assert need > 0
    big = cache(pages_per_seq=1024, n_pages=4096)
    assert paged(big, seqs=1, max_len=0, nbytes=need - 1) == 3 and paged(big, seqs=1, max_len=0, ws=None, nbytes=need) == 3
    assert paged(big, seqs=1, max_len=0, ws=P + 8, nbytes=need) == 2
    assert paged(seqs=0, ws=None, nbytes=0) == 0


def test_packed_attention_refuses():
    assert packed(dtype=3) == packed(causal=2) == packed(scale=float("nan")) == packed(seqs=-1) == packed(n=-1) == 1
    assert packed(heads=5) == packed(kv=0) == packed(d=40) == packed(d=512) == packed(q=rows(P + 8)) == packed(k=rows(stride=4)) == packed(out=rows(stride=128)) == 2
    assert packed(dtype=B.HE_F32, k=rows(stride=130)) == 2 and packed(seqs=65536) == 2
    assert packed(n=1 << 23, heads=128, kv=2, q=rows(stride=8192), out=rows(stride=8192)) == 2  # (more workgroups than a launch may have)
    assert packed(seqs=0) == packed(n=0) == 0


def test_sample_refuses():
    assert sample(dtype=9) == sample(n=-1) == sample(vocab=0) == 1
    assert sample(vocab=(1 << 20) + 1) == sample(z=rows(P + 2)) == sample(z=rows(stride=-1)) == 2
    assert sample(n=65536) == 2 and sample(ws=P + 8) == 2
    need = B.he_sample_workspace(2, 100)
    assert need > 0 and sample(nbytes=need - 1) == sample(ws=None) == 3 and B.he_sample_workspace(0, 5) == B.he_sample_workspace(1, (1 << 20) + 1) == 0
    assert sample(n=0) == 0


def test_engine_refuses_the_operators_own_dtype():
    from paper_2308_01320_amd import synth
    cfg = B.make_config(synth.CONFIGS["tiny"])
    cfg.dtype = B.HE_F16
    h = C.c_void_p()
    assert B.lib().he_create(C.byref(cfg), None, C.byref(h)) == 1


def test_binding_refuses_what_is_no_gpu_tensor():
    import torch
    z = torch.zeros(2, 8)
    with pytest.raises(B.HeError):
        B.he_sample(z, torch.zeros(2))
    x = torch.zeros(3, 4, 64)
    with pytest.raises(B.HeError):
        B.he_packed_attention(x, x, x, torch.tensor([0, 3], dtype=torch.int32))
