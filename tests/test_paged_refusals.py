"""Arguments that the paged entry points refuse, on the host, before anything reaches a GPU."""
import ctypes

import pytest
import torch

from paper_2409_15104_amd import binding as pec

P = 0x10000          # never dereferenced: the calls fail validation, or have nothing to do
OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 0, -1, -2, -3, -4


def shape(hq=8, hkv=2, d=128, dtype=0, scale=0.0, flags=0):
    return pec.PecShape(hq, hkv, d, dtype, scale, flags)


def cache(**kw):
    c = dict(k=P, v=P, n_pages=10, page_size=16, reserved=0, page_stride=16 * 2 * 128, row_stride=2 * 128, head_stride=128)
    c.update(kw)
    return pec.PecPagedCache(**c)


def batch(**kw):
    b = dict(cu_seqlens_q=P, seqlens_k=P, block_table=P, batch=3, table_len=4, total_q=5, max_len_q=0, max_len_k=0)
    b.update(kw)
    return pec.PecPagedBatch(**b)


def turn(**kw):
    n = dict(q_weight=P, k_weight=P, cos_sin=P, n_positions=100, rotary_dim=128, interleaved=0, eps=1e-6, reserved=0)
    n.update(kw)
    return pec.PecNormRope(**n)


REF = ctypes.byref


def rope(s=None, n=None, q=P, qs=0, k=P, ks=0, pos=P, pos0=0, tokens=5, qo=P, ko=P):
    return pec.lib().pec_qk_norm_rope(REF(s or shape()), REF(n) if n is not None else None, q, qs, k, ks, pos, pos0, tokens, qo, ko, None)


def append(s=None, n=None, c=None, b=None, q=P, qs=0, k=P, ks=0, v=P, vs=0, qo=P):
    return pec.lib().pec_paged_append(REF(s or shape()), REF(n) if n is not None else None, REF(c or cache()), REF(b or batch()), q, qs,
                                      k, ks, v, vs, qo, None)


def attn(s=None, c=None, b=None, q=P, qs=0, out=P, lse=P, ws=P, nbytes=0):
    return pec.lib().pec_attn_paged(REF(s or shape()), REF(c or cache()), REF(b or batch()), q, qs, 1, out, lse, ws, nbytes, None)


def test_norm_rope_refusals():
    assert rope(n=None) == INVALID and rope(n=turn(), tokens=0) == OK
    assert rope(shape(hkv=3), turn()) == INVALID and rope(shape(d=64), turn()) == UNSUPPORTED
    assert rope(shape(flags=1), turn()) == UNSUPPORTED
    for bad in (turn(eps=-1.0), turn(eps=float("nan")), turn(n_positions=-1), turn(rotary_dim=-16), turn(cos_sin=None), turn(n_positions=0),
                turn(reserved=1)):
        assert rope(n=bad) == INVALID
    for bad in (turn(rotary_dim=24), turn(rotary_dim=144)):
        assert rope(n=bad) == UNSUPPORTED
    assert rope(n=turn(cos_sin=P + 4)) == MISALIGNED and rope(n=turn(q_weight=P + 2)) == MISALIGNED
    assert rope(n=turn(), q=None, k=None) == INVALID
    assert rope(n=turn(), qo=None) == INVALID and rope(n=turn(), ko=None) == INVALID
    assert rope(n=turn(), tokens=-1) == INVALID and rope(n=turn(), tokens=(1 << 30) + 1) == UNSUPPORTED
    assert rope(n=turn(), pos=None, pos0=96) == INVALID and rope(n=turn(), pos=None, pos0=-1) == INVALID
    for bad in (8 * 128 - 8, 8 * 128 + 4, -1):
        assert rope(n=turn(), qs=bad) == INVALID
    assert rope(n=turn(), ks=128) == INVALID
    assert rope(n=turn(), q=P + 8) == MISALIGNED and rope(n=turn(), ko=P + 2) == MISALIGNED and rope(n=turn(), pos=P + 1) == MISALIGNED


@pytest.mark.parametrize("call", [append, attn])
def test_cache_and_batch_refusals(call):
    for bad in (cache(k=None), cache(v=None), cache(n_pages=0), cache(page_size=0), cache(page_size=-16), cache(reserved=3),
                cache(row_stride=64), cache(head_stride=0), cache(page_stride=-8), cache(page_stride=64)):
        assert call(c=bad) == INVALID
    for bad in (cache(page_size=4), cache(page_size=24), cache(n_pages=1 << 31), cache(page_size=1 << 22, row_stride=1 << 10)):
        assert call(c=bad) == UNSUPPORTED
    for bad in (cache(k=P + 8), cache(row_stride=2 * 128 + 4), cache(head_stride=132), cache(page_stride=16 * 2 * 128 + 2)):
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
    assert call(qs=-8) == INVALID and call(qs=1025) == INVALID and call(q=P + 8) == MISALIGNED


def test_append_refusals():
    assert append(k=None) == INVALID and append(v=None) == INVALID and append(qo=None) == INVALID
    assert append(v=P + 4) == MISALIGNED and append(ks=100) == INVALID and append(vs=8) == INVALID
    assert append(n=turn(rotary_dim=8)) == UNSUPPORTED and append(s=shape(flags=1)) == UNSUPPORTED


def test_attention_refusals():
    need = pec.pec_paged_workspace_bytes(8, 2, 3, 5)
    assert need > 0
    assert attn(nbytes=need - 1) == WORKSPACE and attn(ws=None, nbytes=need) == WORKSPACE
    assert attn(q=None) == INVALID and attn(out=None) == INVALID and attn(lse=None) == INVALID
    assert attn(out=P + 8) == MISALIGNED and attn(lse=P + 2) == MISALIGNED and attn(ws=P + 8) == MISALIGNED
    assert attn(s=shape(scale=-1.0)) == INVALID and attn(s=shape(dtype=9)) == UNSUPPORTED


def test_head_rows_of_the_binding():
    z = torch.zeros(6, 5, 128, dtype=torch.bfloat16)
    assert pec._rows(z, "q", -1) == 640 and pec._rows(z[:, :2], "q", -1) == 640 and pec._rows(z[::2], "q", -1) == 1280
    assert pec._rows(z[:1, 1:2], "q", -1) == 0 and pec._rows(z[:0], "q", -1) == 0
    for bad in (z[:1].expand(6, 5, 128), z.transpose(0, 1), z.float(), z[:, ::2], z[..., :64], z[0]):
        with pytest.raises(ValueError):
            pec._rows(bad, "q", -1)
    with pytest.raises(ValueError):
        pec._rows(z, "q", 0)


def test_calls_that_no_count_holds():
    """More sequences than are added up, more rows or tile steps than have a number, more KV heads than wavefronts."""
    big = 1 << 60
    assert attn(b=batch(batch=65537, total_q=65537), nbytes=big) == UNSUPPORTED
    assert attn(s=shape(64, 1), b=batch(total_q=1 << 26), nbytes=big) == UNSUPPORTED
    assert attn(s=shape(2, 2), b=batch(batch=60000, total_q=60000, table_len=1 << 24, max_len_q=1), nbytes=big) == UNSUPPORTED
    wide = shape(2100, 2100)
    c = cache(row_stride=2100 * 128, page_stride=16 * 2100 * 128)
    assert attn(s=wide, c=c, b=batch(batch=2, total_q=2, max_len_q=1, table_len=1 << 10), nbytes=big) == UNSUPPORTED


def test_workspace_never_falls():
    for hq, hkv in ((8, 2), (32, 8), (40, 40)):
        for b, t in ((1, 1), (4, 4), (64, 64), (64, 5000), (500, 100000)):
            n = pec.pec_paged_workspace_bytes(hq, hkv, b, t)
            assert n <= pec.pec_paged_workspace_bytes(hq, hkv, b + 7, t) and n <= pec.pec_paged_workspace_bytes(hq, hkv, b, t + 333)


def test_binding_refuses_tensors_of_the_cpu_and_of_other_shapes():
    z = torch.zeros(2, 16, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        pec.PagedCache(z, z)
    with pytest.raises(ValueError):
        pec.NormRope(torch.zeros(4, 128))
    with pytest.raises(ValueError):
        pec.pec_qk_norm_rope(z[0], None, pec.NormRope())
    with pytest.raises(ValueError):
        pec.pec_qk_norm_rope(None, None, pec.NormRope())
