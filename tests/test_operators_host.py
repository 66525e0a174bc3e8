"""What the entry points of the shared cache, of sampling and of stored logits refuse, without a GPU: every check stands in front of the first call of the runtime."""
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


# ---- la_page_map ---------------------------------------------------------------------------------------
MAP = dict(old=P, new=P, R=4, page=16, table=P, ld=8, blocks=8, ring=P, n_pages=10, heads_in=P, heads_out=P + 16, slot=P, pos=P, req=P, rows=5, first=P, stream=None)


@pytest.mark.parametrize("change", [{k: None} for k in ("old", "new", "table", "ring", "heads_in", "heads_out", "slot", "pos", "req", "first")] +
                         [dict(heads_out=P), dict(R=0), dict(R=-1), dict(page=0), dict(blocks=0), dict(n_pages=0), dict(rows=0), dict(ld=7),
                          dict(n_pages=1 << 20, page=1 << 11)])
def test_page_map_refuses(change):
    refused(lib.la_page_map(*{**MAP, **change}.values()), EINVAL)


# ---- la_paged_write, la_paged_attend ------------------------------------------------------------------------
BAD_PAGES = [dict(k=None), dict(v=None), dict(n_layers=0), dict(n_pages=0), dict(page_size=0), dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=4), dict(head_dim=12),
             dict(head_dim=264), dict(dtype=3), dict(dtype=-1), dict(n_pages=1 << 27, page_size=16), dict(k=P + 8), dict(v=P + 2)]
WRITE = dict(pages=None, layer=0, k=P, v=P, ldk=128, ldv=128, slot=P, n=3, stream=None)


@pytest.mark.parametrize("bad", BAD_PAGES)
def test_write_and_attend_refuse_bad_pages(bad):
    refused(lib.la_paged_write(*{**WRITE, "pages": pages(**bad)}.values()), EINVAL)
    refused(lib.la_paged_attend(*{**ATTEND, "pages": pages(**bad)}.values()), EINVAL)
    assert lib.la_paged_attend_workspace(pages(**bad), 4, 8, 3) == 0


@pytest.mark.parametrize("change,code", [(dict(layer=-1), ERANGE), (dict(layer=2), ERANGE), (dict(n=-1), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(slot=None), EINVAL),
                                         (dict(k=P + 2), EINVAL), (dict(v=P + 8), EINVAL), (dict(ldk=127), EINVAL), (dict(ldv=132), EINVAL), (dict(n=2 ** 31 - 1, ), None)])
def test_write_refuses(change, code):
    if code is None:  # (more workgroups than a launch has)
        refused(lib.la_paged_write(*{**WRITE, "pages": pages(n_kv_heads=64, head_dim=256), **change}.values()), EINVAL, "more than one launch")
    else:
        refused(lib.la_paged_write(*{**WRITE, "pages": pages(), **change}.values()), code)


ATTEND = dict(pages=None, layer=0, q=P, ldq=256, Hq=4, scale=0.125, table=P, ldt=8, n_req=3, blocks=8, req=P, pos=P, B=3, out=P, ldo=256, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(layer=2), ERANGE), (dict(layer=-1), ERANGE), (dict(q=None), EINVAL), (dict(table=None), EINVAL), (dict(pos=None), EINVAL), (dict(out=None), EINVAL), (dict(Hq=0), EINVAL),
    (dict(Hq=5), EINVAL), (dict(Hq=-2), EINVAL), (dict(B=-1), EINVAL), (dict(n_req=0), EINVAL), (dict(blocks=0), EINVAL), (dict(ldt=7), EINVAL), (dict(req=None, B=4), EINVAL),
    (dict(q=P + 8), EINVAL), (dict(out=P + 8), EINVAL), (dict(ldq=252), EINVAL), (dict(ldo=257), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(blocks=1 << 27, ldt=1 << 27), EINVAL), (dict(B=(1 << 20) + 1), EINVAL), (dict(Hq=65536), EINVAL)])
def test_attend_refuses(change, code):
    refused(lib.la_paged_attend(*{**ATTEND, "pages": pages(), **change}.values()), code)


def test_attend_asks_for_its_workspace():
    need = lib.la_paged_attend_workspace(pages(), 4, 100, 3)
    assert need > 0 and lib.la_paged_attend_workspace(pages(), 4, 8, 3) == 0  # (a short cache is not cut)
    long = dict(blocks=100, ldt=100)
    refused(lib.la_paged_attend(*{**ATTEND, "pages": pages(), **long, "ws_bytes": need - 1}.values()), ENOMEM)
    refused(lib.la_paged_attend(*{**ATTEND, "pages": pages(), **long, "ws": None}.values()), ENOMEM)
    refused(lib.la_paged_attend(*{**ATTEND, "pages": pages(), **long, "ws": P + 8}.values()), EINVAL)
    for args in ((0, 100, 3), (3, 100, 3), (4, 0, 3), (4, 100, 0), (4, 100, -5)):
        assert lib.la_paged_attend_workspace(pages(), *args) == 0


# ---- la_sample ---------------------------------------------------------------------------------------------
SAMPLE = dict(logits=P, dtype=B.LA_F32, ld=100, B=4, V=100, how=None, ids=P, prob=P, ws=P, ws_bytes=1 << 40, stream=None)


def how(**change):
    d = dict(temperature=P, top_k=P, top_p=P, min_p=P, u=P, u_index=None, n_u=4)
    d.update(change)
    return C.byref(B.la_sampling(*d.values()))


@pytest.mark.parametrize("change,code", [
    (dict(how=None), EINVAL), (dict(logits=None), EINVAL), (dict(ids=None), EINVAL), (dict(how=how(u=None)), EINVAL), (dict(how=how(n_u=3)), EINVAL), (dict(how=how(u_index=P, n_u=0)), EINVAL),
    (dict(dtype=3), EINVAL), (dict(V=0), EINVAL), (dict(V=(1 << 19) + 1, ld=1 << 20), EINVAL), (dict(ld=99), EINVAL), (dict(B=-1), EINVAL), (dict(B=65536, how=how(n_u=65536)), EINVAL),
    (dict(ws=None), ENOMEM), (dict(ws_bytes=100), ENOMEM), (dict(ws=P + 8), EINVAL)])
def test_sample_refuses(change, code):
    refused(lib.la_sample(*{**SAMPLE, "how": how(), **change}.values()), code)


def test_sample_workspace_grows_with_what_it_holds():
    sizes = [lib.la_sample_workspace(b, v) for b, v in ((1, 1), (1, 32768), (1, 32769), (2, 40000), (64, 131072), (64, 1 << 19))]
    assert all(a < b for a, b in zip(sizes[:2], sizes[1:2])) and all(s > 0 for s in sizes) and sizes[5] > sizes[4]
    for bad in ((0, 5), (-1, 5), (3, 0), (3, (1 << 19) + 1)):
        assert lib.la_sample_workspace(*bad) == 0


# ---- calls with nothing to do -------------------------------------------------------------------------------
def test_no_rows_are_no_work():
    assert lib.la_paged_write(*{**WRITE, "pages": pages(), "n": 0, "k": None, "v": None, "slot": None}.values()) == 0
    assert lib.la_paged_attend(*{**ATTEND, "pages": pages(), "B": 0, "q": None, "out": None, "pos": None}.values()) == 0
    assert lib.la_sample(*{**SAMPLE, "how": how(), "B": 0, "logits": None, "ids": None}.values()) == 0


def test_model_calls_refuse_null():
    refused(lib.la_unembed_logits(None, P, 1, P, 10, None), EINVAL)
    refused(lib.la_forward_paged(None, 0, 1, P, 1, P, P, P, pages(), P, 8, 1, 8, None), EINVAL)


# ---- the binding ----------------------------------------------------------------------------------------------
def test_binding_refuses_tensors_of_the_host():
    f, i = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: B.la_sample(torch.zeros(4, 10), f, i), lambda: B.la_page_map(i, i, 16, torch.zeros(4, 2, dtype=torch.int32), i, i, i, i, i, i, torch.zeros(5, dtype=torch.int32)),
                 lambda: B.la_pages(torch.zeros(1, 2, 2, 16, 64), torch.zeros(1, 2, 2, 16, 64)), lambda: B.la_unembed_logits(None, torch.zeros(1, 8), torch.zeros(1, 8))):
        with pytest.raises(B.LaError) as e:
            call()
        assert e.value.code == EINVAL


def test_descriptors_match_the_header():
    assert C.sizeof(B.la_pages_desc) == 2 * 8 + 6 * 4 and C.sizeof(B.la_sampling) == 6 * 8 + 8


def test_write_takes_no_more_threads_than_a_launch_has():
    """A thread per 16 bytes of a row of K: 2^32 of them are refused, whatever their workgroups number."""
    rows = (1 << 32) // (64 * 32)
    refused(lib.la_paged_write(*{**WRITE, "pages": pages(n_kv_heads=64, head_dim=256), "n": rows}.values()), EINVAL, "more than one launch")


@pytest.mark.parametrize("rows,heads", [(1 << 20, 16), (1 << 20, 4096), (300, 65535)])
@pytest.mark.parametrize("blocks", [8, 1000])
def test_attend_takes_no_more_workgroups_than_a_launch_has(rows, heads, blocks):
    call = {**ATTEND, "pages": pages(n_kv_heads=heads), "Hq": heads, "B": rows, "blocks": blocks, "ldt": blocks, "ws_bytes": 1 << 62}
    refused(lib.la_paged_attend(*call.values()), EINVAL, "more than one launch")


@pytest.mark.parametrize("b,v", [(1, 1), (1, 2048), (1, 2049), (1, 32768), (1, 32769), (2, 40000), (64, 131072), (3, 1 << 19), (65535, 1000)])
def test_sample_workspace_holds_what_a_call_writes(b, v):
    """Per row and chunk: its first token (8 bytes), 520 sums (8) and counts (4), the bins in use (4), a place per token (2); and not much more."""
    chunk = 2048 if v <= 32768 else 8192
    need = b * -(-v // chunk) * (8 + 520 * 12 + 4 + 2 * chunk)
    assert need <= lib.la_sample_workspace(b, v) <= need + 64


@pytest.mark.parametrize("requests", [(1 << 30) + 1, (1 << 31) - 256, (1 << 31) - 1])
def test_page_map_takes_no_more_requests_than_its_threads_count(requests):
    """A thread goes from request to request in steps of a workgroup, in 32 bits: beyond 2^31 - 256 it would pass their end."""
    refused(lib.la_page_map(*{**MAP, "R": requests}.values()), EINVAL, "requests")
