"""The paged calls' binding refuses tensors that do not hold what the call would read or write: on the CPU, where a call that has
passed every such check is refused for its device."""
import pytest
import torch

from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd.inputs import LayerShape

H, HKV, D, PAGES, B, NEW, KEEP, ROWS = 4, 2, 64, 5, 3, 2, 4, 7
I32, I64, F32, BF16 = torch.int32, torch.int64, torch.float32, torch.bfloat16


def _desc(**kw):
    return qb.make_desc(LayerShape(**{**dict(d_model=H * D, n_q_heads=H, n_kv_heads=HKV, head_dim=D, rope_base=10000.0, dtype="f32"), **kw}))


def _cache(dtype=F32, heads=HKV, d=D):
    pool = torch.zeros(PAGES, 16, heads, d, dtype=dtype)
    c = qb.PageCacheDesc(4096, 4096, 4096, 4096, 16 * heads * d, heads * d, d, PAGES, 16, 5, 0)
    return qb.PageCache(c, (pool, pool, None, torch.zeros(B, 5, dtype=I32)))


def _z(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype)


def _append(cache=None, desc=None, **kw):
    a = dict(q=_z(ROWS, H, D), k=_z(ROWS, HKV, D), v=_z(ROWS, HKV, D), row_off=_z(B + 1, dtype=I64), total_rows=ROWS, lens=_z(B, dtype=I32),
             pos=_z(ROWS, dtype=I32), q_out=_z(ROWS, H, D))
    a.update(kw)
    qb.qcf_page_append(desc or _desc(), cache or _cache(), B, **a)


def _select(cache=None, desc=None, **kw):
    a = dict(q=_z(B, NEW, H, D), seen=_z(B, NEW, dtype=I32), n_keep=KEEP, n_first=1, n_last=1, pages=_z(B, NEW, HKV, KEEP, dtype=I32),
             workspace=_z(1 << 16, dtype=torch.uint8))
    a.update(kw)
    qb.qcf_page_select(desc or _desc(), cache or _cache(), B, NEW, **a)


def _attn(cache=None, desc=None, **kw):
    a = dict(q=_z(B, NEW, H, D), seen=_z(B, NEW, dtype=I32), pages=_z(B, NEW, HKV, KEEP, dtype=I32), n_keep=KEEP, o_out=_z(B, NEW, H, D),
             lse_out=_z(B, NEW, H), workspace=_z(1 << 16, dtype=torch.uint8))
    a.update(kw)
    qb.qcf_page_attn(desc or _desc(), cache or _cache(), B, NEW, **a)


@pytest.mark.parametrize("call", [_append, _select, _attn])
def test_what_fits_is_only_refused_for_its_device(call):
    with pytest.raises(qb.QcfError, match="current device"):
        call()


def test_what_fits_with_less_or_with_room():
    with pytest.raises(qb.QcfError, match="current device"):
        _append(q=None, q_out=None, pos=None, k=_z(ROWS + 3, HKV, D), row_off=_z(B + 9, dtype=I64))
    rows = _z(ROWS, (H + 2 * HKV) * D)
    q, k, v = (t.unflatten(1, (-1, D)) for t in rows.split([H * D, HKV * D, HKV * D], 1))
    with pytest.raises(qb.QcfError, match="current device"):
        _append(q=q, k=k, v=v)
    with pytest.raises(qb.QcfError, match="current device"):
        _attn(pages=None, n_keep=0, lse_out=None, q=_z(B * NEW, H * D), seen=_z(B * NEW, dtype=I32), workspace=_z(1 << 12))


@pytest.mark.parametrize("call", [_append, _select, _attn])
@pytest.mark.parametrize("cache", [dict(dtype=BF16), dict(heads=4), dict(d=128), dict(dtype=torch.float16)])
def test_pages_of_another_layer(call, cache):
    with pytest.raises(qb.QcfError, match="for a layer of 2 heads of 64"):
        call(cache=_cache(**cache))


@pytest.mark.parametrize("change,word", [
    (dict(q=_z(ROWS, H, D, dtype=BF16)), "rows of"), (dict(k=_z(ROWS, HKV, D, dtype=torch.float64)), "rows of"),
    (dict(k=_z(ROWS, 4, D)), "2 heads of 64"), (dict(v=_z(ROWS, 1, 128)), "2 heads of 64"), (dict(q=_z(ROWS, 2, D)), "4 heads of 64"),
    (dict(q=_z(ROWS - 1, H, D)), "rows, 7 wanted"), (dict(k=_z(ROWS - 1, HKV, D)), "rows, 7 wanted"),
    (dict(row_off=_z(B, dtype=I64)), "row_off"), (dict(row_off=_z(B + 1, dtype=I32)), "row_off"), (dict(lens=_z(B - 1, dtype=I32)), "lens"),
    (dict(lens=_z(B, dtype=I64)), "lens"), (dict(pos=_z(ROWS - 1, dtype=I32)), "pos"), (dict(pos=_z(ROWS, dtype=I64)), "pos"),
    (dict(q_out=_z(ROWS - 1, H, D)), "q_out"), (dict(q_out=_z(ROWS, H, D, dtype=BF16)), "q_out"),
    (dict(q_out=_z(ROWS, H, 2 * D)[..., :D]), "q_out"), (dict(lens=_z(2 * B, dtype=I32)[::2]), "lens")])
def test_appends_that_do_not_fit(change, word):
    with pytest.raises(qb.QcfError, match=word):
        _append(**change)


@pytest.mark.parametrize("change,word", [
    (dict(pages=_z(B, NEW, HKV, KEEP - 1, dtype=I32)), "n_keep is 4"), (dict(pages=_z(B, NEW, HKV, KEEP + 1, dtype=I32)), "n_keep is 4"),
    (dict(pages=_z(B - 1, NEW, HKV, KEEP, dtype=I32)), "pages"), (dict(pages=_z(B, NEW, HKV, KEEP, dtype=I64)), "pages"),
    (dict(seen=_z(B, dtype=I32)), "seen"), (dict(seen=_z(B, NEW, dtype=I64)), "seen"), (dict(q=_z(B, H, D)), "q"),
    (dict(q=_z(B, NEW, H, D, dtype=BF16)), "q"), (dict(q=_z(NEW, B, H, D).transpose(0, 1)), "q"),
    (dict(workspace=_z(512, dtype=torch.uint8)[::2]), "workspace")])
def test_selections_and_attention_that_do_not_fit(change, word):
    for call in (_select, _attn):
        with pytest.raises(qb.QcfError, match=word):
            call(**change)


@pytest.mark.parametrize("change,word", [
    (dict(o_out=_z(B, NEW, H, D, dtype=BF16)), "o_out"), (dict(o_out=_z(B, 1, H, D)), "o_out"), (dict(lse_out=_z(B, NEW, H, dtype=BF16)), "lse_out"),
    (dict(lse_out=_z(B, H)), "lse_out"), (dict(lse_out=_z(B, NEW, 2 * H)[..., ::2]), "lse_out")])
def test_results_that_do_not_fit(change, word):
    with pytest.raises(qb.QcfError, match=word):
        _attn(**change)
