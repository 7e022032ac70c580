"""Arguments that the entry points of the paged cache in 4 bits refuse, on the host, before anything reaches a GPU."""
import ctypes

import pytest
import torch

from paper_2409_15104_amd import binding as pec

P = 0x10000          # never dereferenced: the calls fail validation, or have nothing to do
OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 0, -1, -2, -3, -4
REF = ctypes.byref


def shape(hq=8, hkv=2, d=128, dtype=0, scale=0.0, flags=0):
    return pec.PecShape(hq, hkv, d, dtype, scale, flags)


def cache(**kw):
    c = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=10, page_size=16, reserved=0, page_stride=16 * 2 * 64, row_stride=2 * 64, head_stride=64,
             scale_page_stride=2 * 64, scale_head_stride=64)
    c.update(kw)
    return pec.PecPagedCacheMx(**c)


def batch(**kw):
    b = dict(cu_seqlens_q=P, seqlens_k=P, block_table=P, batch=3, table_len=4, total_q=5, max_len_q=0, max_len_k=0)
    b.update(kw)
    return pec.PecPagedBatch(**b)


def append(s=None, n=None, c=None, b=None, q=P, qs=0, k=P, ks=0, v=P, vs=0, qo=P):
    return pec.lib().pec_paged_append_mx(REF(s or shape()), REF(n) if n is not None else None, REF(c or cache()), REF(b or batch()), q, qs,
                                         k, ks, v, vs, qo, None)


def read(s=None, c=None, b=None, k=P, v=P):
    return pec.lib().pec_paged_read_mx(REF(s or shape()), REF(c or cache()), REF(b or batch()), k, v, None)


def attn(s=None, c=None, b=None, q=P, qs=0, out=P, lse=P, ws=P, nbytes=0):
    return pec.lib().pec_attn_paged_mx(REF(s or shape()), REF(c or cache()), REF(b or batch()), q, qs, 1, out, lse, ws, nbytes, None)


@pytest.mark.parametrize("call", [append, read, attn])
def test_cache_and_batch_refusals(call):
    for bad in (cache(k=None), cache(v=None), cache(k_scale=None), cache(v_scale=None), cache(n_pages=0), cache(page_size=0),
                cache(page_size=-16), cache(reserved=3), cache(row_stride=48), cache(row_stride=-64), cache(head_stride=0), cache(page_stride=-16),
                cache(page_stride=48), cache(scale_page_stride=56), cache(scale_page_stride=-64), cache(scale_head_stride=56),
                cache(page_stride=(1 << 46) + 16), cache(row_stride=(1 << 31) + 16)):
        assert call(c=bad) == INVALID
    for bad in (cache(page_size=4), cache(page_size=24), cache(n_pages=1 << 31), cache(page_size=1 << 22, row_stride=1 << 10, scale_head_stride=1 << 24,
                                                                                     scale_page_stride=1 << 25),
                cache(scale_head_stride=(1 << 31) - 64)):
        assert call(c=bad) == UNSUPPORTED
    for bad in (cache(k=P + 8), cache(v_scale=P + 8), cache(row_stride=2 * 64 + 8), cache(head_stride=72), cache(page_stride=16 * 2 * 64 + 4),
                cache(scale_page_stride=132), cache(scale_head_stride=68)):
        assert call(c=bad) == MISALIGNED
    for bad in (batch(batch=-1), batch(total_q=-1), batch(table_len=-1), batch(cu_seqlens_q=None), batch(seqlens_k=None),
                batch(block_table=None), batch(max_len_q=-1), batch(max_len_k=-1)):
        assert call(b=bad) == INVALID
    assert call(b=batch(total_q=(1 << 30) + 1)) == UNSUPPORTED
    for bad in (batch(cu_seqlens_q=P + 2), batch(seqlens_k=P + 1), batch(block_table=P + 2)):
        assert call(b=bad) == MISALIGNED
    for nothing in (batch(batch=0), batch(total_q=0), batch(total_q=0, cu_seqlens_q=None, seqlens_k=None, block_table=None)):
        assert call(b=nothing) == OK
    assert call(s=shape(hq=7)) == INVALID and call(s=shape(d=64)) == UNSUPPORTED and call(s=shape(flags=2)) == UNSUPPORTED


def test_one_head_or_one_page_needs_no_stride():
    one = dict(head_stride=0, scale_head_stride=0)
    assert append(s=shape(hkv=1), c=cache(**one), b=batch(total_q=0)) == OK
    assert read(c=cache(n_pages=1, page_stride=0, scale_page_stride=0), b=batch(total_q=0)) == OK


def test_append_refusals():
    assert append(k=None) == INVALID and append(v=None) == INVALID and append(qo=None) == INVALID
    assert append(v=P + 4) == MISALIGNED and append(ks=100) == INVALID and append(vs=8) == INVALID and append(qs=-8) == INVALID
    assert append(s=shape(flags=1)) == UNSUPPORTED
    assert append(n=pec.PecNormRope(P, P, P, 100, 8, 0, 1e-6, 0)) == UNSUPPORTED


def test_read_refusals():
    assert read(k=None) == INVALID and read(v=None) == INVALID and read(k=P + 8) == MISALIGNED and read(v=P + 2) == MISALIGNED


def test_attention_refusals():
    need = pec.pec_paged_mx_workspace_bytes(8, 2, 3, 5)
    assert need > 0
    assert attn(nbytes=need - 1) == WORKSPACE and attn(ws=None, nbytes=need) == WORKSPACE
    assert attn(q=None) == INVALID and attn(out=None) == INVALID and attn(lse=None) == INVALID
    assert attn(out=P + 8) == MISALIGNED and attn(lse=P + 2) == MISALIGNED and attn(ws=P + 8) == MISALIGNED and attn(q=P + 8) == MISALIGNED
    assert attn(s=shape(scale=-1.0)) == INVALID and attn(s=shape(dtype=9)) == UNSUPPORTED
    assert attn(qs=-8) == INVALID and attn(qs=1025) == INVALID


def test_workspace_never_falls():
    f = pec.pec_paged_mx_workspace_bytes
    for hq, hkv in ((8, 2), (32, 8), (40, 40)):
        for b, t in ((1, 1), (4, 4), (64, 64), (64, 5000), (500, 100000)):
            for k in (0, 1000, 100000):
                n = f(hq, hkv, b, t, k)
                assert n <= f(hq, hkv, b + 7, t, k) and n <= f(hq, hkv, b, t + 333, k) and n <= f(hq, hkv, b, t, k + 77)
    assert f(8, 3, 1, 1) == 0 and f(8, 2, -1, 1) == 0 and f(8, 2, 1, -1) == 0 and f(8, 2, 1, 1, -1) == 0


def test_binding_refuses_tensors_of_the_cpu_and_of_other_shapes():
    z, s = torch.zeros(2, 16, 2, 64, dtype=torch.uint8), torch.zeros(2, 2, 4, 16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        pec.PagedCacheMx(z, z, s, s)
