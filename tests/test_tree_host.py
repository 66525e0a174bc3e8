"""What the entry points of drafted trees, of slot copies and of adjusted logits refuse, without a GPU: every check stands in front of the first call of the runtime."""
import ctypes as C

import pytest
import torch

from paper_2602_16760_amd import binding as B

EINVAL, ENOMEM, ERANGE = -1, -2, -3
P = 1 << 20  # an address that is aligned and never followed
lib = B.lib


def refused(rc, code, text=None):
    assert rc == code, (rc, lib.la_last_error())
    if text:
        assert text in lib.la_last_error().decode(), lib.la_last_error()


def pages(**change):
    d = dict(k=P, v=P, n_layers=2, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, dtype=B.LA_BF16)
    d.update(change)
    return C.byref(B.la_pages_desc(*d.values()))


BAD_PAGES = [dict(k=None), dict(v=None), dict(n_layers=0), dict(n_pages=0), dict(page_size=0), dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=4), dict(head_dim=12),
             dict(head_dim=264), dict(dtype=3), dict(dtype=-1), dict(n_pages=1 << 27, page_size=16), dict(k=P + 8), dict(v=P + 2)]
LAYOUT = dict(parent=P, first=P, len=P, R=3, B=9, pos=P, vis=P, stream=None)
ACCEPT = dict(parent=P, tok=P, ids=P, slot=P, first=P, len=P, limit=None, R=3, B=9, max_path=4, n_new=P, new_len=P, last=P, out=P, frm=P, to=P, stream=None)
COPY = dict(pages=None, begin=0, end=2, frm=P, to=P, n=6, run=2, stream=None)
ATTEND = dict(pages=None, layer=0, q=P, ldq=256, Hq=4, scale=0.125, table=P, ldt=8, n_req=3, blocks=8, first=P, len=P, vis=P, max_rows=8, B=9, out=P, ldo=256, ws=P, ws_bytes=1 << 40,
              stream=None)


@pytest.mark.parametrize("change", [{k: None} for k in ("parent", "first", "len", "pos", "vis")] + [dict(R=-1), dict(B=-1), dict(R=0), dict(R=(1 << 20) + 1), dict(B=(1 << 20) + 1), dict(vis=P + 4)])
def test_layout_refuses(change):
    refused(lib.la_tree_layout(*{**LAYOUT, **change}.values()), EINVAL)


@pytest.mark.parametrize("change", [{k: None} for k in ("parent", "tok", "ids", "slot", "first", "len", "n_new", "new_len", "last", "out", "frm", "to")] +
                         [dict(R=-1), dict(B=-1), dict(R=(1 << 20) + 1), dict(B=(1 << 20) + 1), dict(max_path=0), dict(max_path=65), dict(max_path=-1)])
def test_accept_refuses(change):
    refused(lib.la_tree_accept(*{**ACCEPT, **change}.values()), EINVAL)


@pytest.mark.parametrize("change,code", [(dict(begin=-1), ERANGE), (dict(end=3), ERANGE), (dict(begin=2, end=1), ERANGE), (dict(n=-1), EINVAL), (dict(run=0), EINVAL), (dict(run=65), EINVAL),
                                         (dict(frm=None), EINVAL), (dict(to=None), EINVAL)] + [(dict(pages=pages(**b)), EINVAL) for b in BAD_PAGES])
def test_copy_refuses(change, code):
    refused(lib.la_paged_copy(*{**COPY, "pages": pages(), **change}.values()), code)


@pytest.mark.parametrize("n,run,heads,dh", [(2 ** 31 - 1, 1, 64, 256), (2 ** 31 - 1, 64, 8192, 256), (100, 1, 65536, 64)])
def test_copy_takes_no_more_than_a_launch_has(n, run, heads, dh):
    refused(lib.la_paged_copy(*{**COPY, "pages": pages(n_kv_heads=heads, head_dim=dh), "n": n, "run": run}.values()), EINVAL, "more than one launch")


@pytest.mark.parametrize("change,code", [
    (dict(layer=2), ERANGE), (dict(layer=-1), ERANGE), (dict(q=None), EINVAL), (dict(table=None), EINVAL), (dict(first=None), EINVAL), (dict(len=None), EINVAL), (dict(vis=None), EINVAL),
    (dict(out=None), EINVAL), (dict(Hq=0), EINVAL), (dict(Hq=5), EINVAL), (dict(Hq=-2), EINVAL), (dict(B=-1), EINVAL), (dict(n_req=0), EINVAL), (dict(blocks=0), EINVAL), (dict(ldt=7), EINVAL),
    (dict(q=P + 8), EINVAL), (dict(out=P + 8), EINVAL), (dict(vis=P + 4), EINVAL), (dict(ldq=252), EINVAL), (dict(ldo=257), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(blocks=1 << 27, ldt=1 << 27), EINVAL), (dict(B=(1 << 20) + 1), EINVAL), (dict(n_req=(1 << 20) + 1), EINVAL), (dict(max_rows=0), EINVAL),
    (dict(max_rows=65), EINVAL)] + [(dict(pages=pages(**b)), EINVAL) for b in BAD_PAGES])
def test_attend_refuses(change, code):
    refused(lib.la_paged_tree_attend(*{**ATTEND, "pages": pages(), **change}.values()), code)


def test_attend_asks_for_its_workspace():
    size = lib.la_paged_tree_attend_workspace
    need = size(pages(), 4, 100, 3, 8)
    assert need > 0 and size(pages(), 4, 8, 3, 8) == 0  # (a short cache is not cut)
    long = dict(blocks=100, ldt=100)
    refused(lib.la_paged_tree_attend(*{**ATTEND, "pages": pages(), **long, "ws_bytes": need - 1}.values()), ENOMEM)
    refused(lib.la_paged_tree_attend(*{**ATTEND, "pages": pages(), **long, "ws": None}.values()), ENOMEM)
    refused(lib.la_paged_tree_attend(*{**ATTEND, "pages": pages(), **long, "ws": P + 8}.values()), EINVAL)
    for args in ((0, 100, 3, 8), (3, 100, 3, 8), (4, 0, 3, 8), (4, 100, 0, 8), (4, 100, 3, 0), (4, 100, 3, 65)):
        assert size(pages(), *args) == 0
    for bad in BAD_PAGES:
        assert size(pages(**bad), 4, 100, 3, 8) == 0


@pytest.mark.parametrize("heads,kv,dh,dtype,page", [(32, 8, 128, B.LA_BF16, 16), (32, 8, 128, B.LA_F16, 24), (4, 2, 64, B.LA_F32, 24), (16, 1, 256, B.LA_F16, 16), (128, 1, 128, B.LA_BF16, 16), (8, 8, 64, B.LA_BF16, 64)])
def test_attend_keeps_its_records_to_a_bound(heads, kv, dh, dtype, page):
    """64 MB, or six items' where those are more, at any number of requests, rows and positions; and what a request and a list of items take beside them."""
    p = pages(n_kv_heads=kv, head_dim=dh, dtype=dtype, page_size=page)
    for rows in (1, 2, 3, 8, 16, 17, 40, 64):
        record = heads * rows * (dh + 4) * 4
        for R in (1, 2, 5, 17, 64, 65, 1000):
            for blocks in (1, 20, 50, 300, 4000, 1 << 20):
                beside = 8 * R + 16 + (0 if R <= 64 else 36 * R + 32 * 4096)
                assert lib.la_paged_tree_attend_workspace(p, heads, blocks, R, rows) <= max(64 << 20, 6 * record) + beside


def test_attend_takes_no_more_workgroups_than_a_launch_has():
    call = {**ATTEND, "pages": pages(n_kv_heads=4096), "Hq": 4096, "B": 1 << 20, "n_req": 1 << 20}
    refused(lib.la_paged_tree_attend(*call.values()), EINVAL, "more than one launch")
    call = {**ATTEND, "pages": pages(), "B": 1 << 20, "n_req": 1 << 20, "max_rows": 64}
    refused(lib.la_paged_tree_attend(*call.values()), EINVAL, "more than one launch")


def test_model_calls_refuse_null():
    refused(lib.la_forward_tree(None, 0, 1, P, 1, P, P, P, P, P, 1, pages(), P, 8, 1, 8, None), EINVAL)


# ---- la_logits_adjust -------------------------------------------------------------------------------------
ADJUST = dict(logits=P, dtype=B.LA_F32, ld=100, B=4, V=100, how=None, out=2 * P, ldo=100, stream=None)


def how(**change):
    d = dict(req=P, repetition=P, presence=P, frequency=P, tokens=P, n_tokens=P, n_prompt=P, draft=P, first=P, vis=P, bias_token=P, bias=P, allowed=P, allowed_index=P, tokens_stride=50,
             bias_stride=7, allowed_stride=4, n_requests=3, max_tokens=50, n_bias=7, n_allowed=2)
    d.update(change)
    return C.byref(B.la_adjust(*d.values()))


@pytest.mark.parametrize("change", [
    dict(how=None), dict(logits=None), dict(out=None), dict(dtype=3), dict(V=0), dict(V=(1 << 19) + 1, ld=1 << 20, ldo=1 << 20), dict(ld=99), dict(ldo=99), dict(B=-1), dict(B=65536),
    dict(out=P, ldo=104), dict(how=how(req=None)), dict(how=how(n_requests=-1)), dict(how=how(max_tokens=-1)), dict(how=how(n_bias=-1)), dict(how=how(n_allowed=-1)),
    dict(how=how(n_tokens=None)), dict(how=how(tokens_stride=49)), dict(how=how(max_tokens=(1 << 24) + 1, tokens_stride=1 << 25)), dict(how=how(first=None)), dict(how=how(vis=None)),
    dict(how=how(bias=None)), dict(how=how(bias_token=None)), dict(how=how(bias_stride=6)), dict(how=how(n_bias=4097, bias_stride=5000)), dict(how=how(allowed_stride=3)),
    dict(how=how(allowed_index=None))])
def test_adjust_refuses(change):
    refused(lib.la_logits_adjust(*{**ADJUST, "how": how(), **change}.values()), EINVAL)


def test_no_rows_are_no_work():
    assert lib.la_tree_layout(*{**LAYOUT, "B": 0, "parent": None, "pos": None, "vis": None}.values()) == 0
    assert lib.la_tree_accept(*{**ACCEPT, "R": 0, "first": None, "out": None}.values()) == 0
    assert lib.la_paged_copy(*{**COPY, "pages": pages(), "n": 0, "frm": None, "to": None}.values()) == 0
    assert lib.la_paged_copy(*{**COPY, "pages": pages(), "begin": 1, "end": 1, "frm": None}.values()) == 0
    assert lib.la_paged_tree_attend(*{**ATTEND, "pages": pages(), "B": 0, "q": None, "out": None, "vis": None}.values()) == 0
    assert lib.la_logits_adjust(*{**ADJUST, "how": how(), "B": 0, "logits": None, "out": None}.values()) == 0


def test_descriptor_matches_the_header():
    assert C.sizeof(B.la_adjust) == 14 * 8 + 3 * 8 + 4 * 4


def test_binding_refuses_tensors_of_the_host():
    f, i, m = torch.zeros(4), torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int64)
    first, path = torch.zeros(5, dtype=torch.int32), torch.zeros(4, 3, dtype=torch.int32)
    for call in (lambda: B.la_tree_layout(i, first, i, i, m), lambda: B.la_tree_accept(i, i, i, i, first, i, i, i, i, path, path, path),
                 lambda: B.la_logits_adjust(torch.zeros(4, 10), torch.zeros(4, 10), repetition=f)):
        with pytest.raises(B.LaError) as e:
            call()
        assert e.value.code == EINVAL
