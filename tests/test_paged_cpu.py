"""What the paged calls refuse, on the CPU: every refusal comes before the first launch, so no device is needed."""
import ctypes

import pytest
import torch

from paper_2502_02617_amd import Context, PQ_BF16, PolarQuantError, Rotary, library
from paper_2502_02617_amd.binding import PQ_F32

EINVAL, EUNSUPPORTED, EALIGN, ENOMEM = -1, -2, -3, -5
P = 1 << 20  # stands for a device address, 16-byte aligned; never read


@pytest.fixture(scope="module")
def ctx():
    c = Context(seed=0)
    yield c
    c.close()


def rotary(cs=P, n_pos=10, dim=128, interleaved=0):
    r = Rotary.__new__(Rotary)
    ctypes.Structure.__init__(r)
    r.cos_sin, r.n_pos, r.dim, r.interleaved = cs, n_pos, dim, interleaved
    return ctypes.byref(r)


def append(ctx, **kw):
    a = dict(handle=ctx._h, xk=P, xv=P, xt=PQ_BF16, n_rows=4, n_heads=2, ld_token=256, ld_head=128, rot=None, positions=None, kc=P, kr=P, vc=P, vr=P,
             pool=640, pages=P, ld_pages=3, row_start=P, ctx_len=P, n_seq=2, stream=None)
    a.update(kw)
    return library().pq_append_paged(*a.values())


def decode(ctx, **kw):
    a = dict(handle=ctx._h, kc=P, kr=P, vc=P, vr=P, pool=640, pages=P, ld_pages=3, row_start=P, ctx_len=P, n_seq=2, n_rows=4, n_heads=2, ok=P, ov=P,
             ot=PQ_F32, ld_token=256, ld_head=128, stream=None)
    a.update(kw)
    return library().pq_decode_paged(*a.values())


def attend(ctx, **kw):
    a = dict(handle=ctx._h, q=P, out=P, ot=PQ_F32, rot=None, positions=None, kc=P, kr=P, vc=P, vr=P, pool=640, pages=P, ld_pages=10, ctx_len=P, B=2, M=1,
             Hq=8, Hkv=2, max_ctx=600, scale=0.1, ws=P, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return library().pq_attn_paged(*a.values())


def attend_prefix(ctx, **kw):
    a = dict(handle=ctx._h, q=P, out=P, ot=PQ_F32, rot=None, positions=None, kc=P, kr=P, vc=P, vr=P, pool=640, pages=P, ld_pages=10, ctx_len=P, B=2, M=1,
             Hq=8, Hkv=2, max_ctx=600, pre_pages=P, pre_ld=5, pre_len=P, start=P, groups=1, max_prefix=300, scale=0.1, ws=P, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return library().pq_attn_prefix_paged(*a.values())


@pytest.mark.parametrize("call", [append, decode])
@pytest.mark.parametrize("kw,code", [
    (dict(handle=None), EINVAL), (dict(kc=None), EINVAL), (dict(vr=None), EINVAL), (dict(pages=None), EINVAL), (dict(row_start=None), EINVAL),
    (dict(ctx_len=None), EINVAL), (dict(n_rows=-1), EINVAL), (dict(n_seq=-1), EINVAL), (dict(n_heads=0), EINVAL), (dict(pool=0), EINVAL),
    (dict(pool=100), EINVAL), (dict(ld_pages=0), EINVAL), (dict(ld_token=-8), EINVAL), (dict(ld_head=-8), EINVAL), (dict(kc=P + 8), EALIGN),
    (dict(vr=P + 2), EALIGN)])
def test_refusals_of_ragged_rows(ctx, call, kw, code):
    assert call(ctx, **kw) == code


@pytest.mark.parametrize("call", [append, decode])
@pytest.mark.parametrize("kw", [dict(n_rows=0), dict(n_seq=0)])
def test_nothing_to_do(ctx, call, kw):
    kw = dict(kw, kc=None, pages=None, row_start=None)
    assert call(ctx, **kw) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(xk=None), EINVAL), (dict(xv=None), EINVAL), (dict(xt=7), EINVAL), (dict(xk=P + 4), EALIGN), (dict(ld_token=260), EALIGN),
    (dict(ld_head=4), EALIGN), (dict(xt=PQ_F32, ld_head=6), EALIGN), (dict(n_rows=1 << 30), EUNSUPPORTED),
    (dict(rot=rotary(cs=None)), EINVAL), (dict(rot=rotary(n_pos=0)), EINVAL), (dict(rot=rotary(dim=0)), EINVAL),
    (dict(rot=rotary(dim=144)), EINVAL), (dict(rot=rotary(dim=40)), EUNSUPPORTED), (dict(rot=rotary(cs=P + 4)), EALIGN)])
def test_refusals_of_append(ctx, kw, code):
    assert append(ctx, **kw) == code


@pytest.mark.parametrize("kw,code", [(dict(ok=None, ov=None), EINVAL), (dict(ot=7), EINVAL), (dict(ok=P + 8), EALIGN), (dict(ov=P + 8), EALIGN),
                                     (dict(n_rows=1 << 31), EUNSUPPORTED)])
def test_refusals_of_decode(ctx, kw, code):
    assert decode(ctx, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(handle=None), EINVAL), (dict(q=None), EINVAL), (dict(pages=None), EINVAL), (dict(ctx_len=None), EINVAL), (dict(ws=None), EINVAL),
    (dict(B=0), EINVAL), (dict(Hq=7), EINVAL), (dict(max_ctx=-1), EINVAL), (dict(max_ctx=641), EINVAL), (dict(ld_pages=0), EINVAL),
    (dict(ld_pages=9), EINVAL), (dict(M=0), EUNSUPPORTED), (dict(M=5), EUNSUPPORTED), (dict(ot=5), EINVAL), (dict(q=P + 8), EALIGN),
    (dict(ws_bytes=100), ENOMEM), (dict(rot=rotary(dim=24)), EUNSUPPORTED), (dict(rot=rotary(cs=P + 8)), EALIGN),
    (dict(ld_pages=1 << 24, max_ctx=(1 << 26) + 1), EUNSUPPORTED)])
def test_refusals_of_attention(ctx, kw, code):
    assert attend(ctx, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(handle=None), EINVAL), (dict(pre_pages=None), EINVAL), (dict(pre_len=None), EINVAL), (dict(start=None), EINVAL), (dict(groups=-1), EINVAL),
    (dict(max_prefix=-1), EINVAL), (dict(pre_ld=0), EINVAL), (dict(pre_ld=4), EINVAL), (dict(groups=(1 << 24) + 1), EUNSUPPORTED),
    (dict(pre_ld=1 << 21, max_prefix=(1 << 26) + 1), EUNSUPPORTED), (dict(pre_ld=1 << 20, max_prefix=1 << 26, groups=2000, ws_bytes=1 << 60), EUNSUPPORTED),
    (dict(max_ctx=641), EINVAL), (dict(M=5), EUNSUPPORTED), (dict(q=P + 8), EALIGN), (dict(ws_bytes=1000), ENOMEM),
    (dict(ws_bytes=Context.attn_prefix_paged_workspace_bytes(2, 1, 8, 2, 600, 1, 300) - 1), ENOMEM), (dict(rot=rotary(n_pos=-1)), EINVAL)])
def test_refusals_of_attention_with_prefixes(ctx, kw, code):
    assert attend_prefix(ctx, **kw) == code


def test_workspace_with_prefixes():
    own = Context.attn_paged_workspace_bytes(4, 1, 32, 8, 100)
    assert Context.attn_prefix_paged_workspace_bytes(4, 1, 32, 8, 100, 0, 0) == own
    sizes = [Context.attn_prefix_paged_workspace_bytes(B, 1, 32, 8, 100, 2, n) for B, n in ((4, 0), (4, 100), (4, 5000), (64, 5000))]
    assert own < sizes[0] <= sizes[1] <= sizes[2] <= sizes[3]
    assert Context.attn_prefix_paged_workspace_bytes(4, 1, 7, 2, 100, 1, 100) == 0


def test_workspace_is_that_of_several_query_tokens():
    for args in ((1, 1, 32, 8, 1000), (16, 4, 32, 8, 12700)):
        assert Context.attn_paged_workspace_bytes(*args) == Context.attn_mq_workspace_bytes(*args) > 0
    assert Context.attn_paged_workspace_bytes(0, 1, 8, 2, 10) == 0


def test_the_binding_refuses_tensors_of_another_kind(ctx):
    """Host tensors, wrong types and shapes never reach the library (whose kernels would read them as device addresses)."""
    cache = ctx.alloc_cache_for(2, 128, "cpu") + ctx.alloc_cache_for(2, 128, "cpu")
    x = torch.zeros(3, 2, 128)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(PolarQuantError):
        ctx.append_paged(x, x, i, i[:1], *cache, i.view(1, 2))
    with pytest.raises(PolarQuantError):
        ctx.append_paged(x, x[:2], i, i[:1], *cache, i.view(1, 2))
    with pytest.raises(PolarQuantError):
        ctx.decode_paged(*cache, i.view(1, 2), i, i[:1], x, x)
    with pytest.raises(PolarQuantError):
        ctx.decode_paged(*cache, i.view(1, 2), i, i[:1])
    q = torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(PolarQuantError):
        ctx.attn_paged(q, q.clone(), *cache, i.view(1, 2), i[:1], 10, 0.1, torch.zeros(1 << 20, dtype=torch.uint8))
    for bad in (torch.zeros(4, 128), torch.zeros(4, 128, dtype=torch.bfloat16)):
        with pytest.raises(PolarQuantError):
            Rotary(bad)
