"""Refusals of the paged 4-bit cache and of beam search over it: every call
that the header rules out returns its status before any launch (so this runs
without a GPU), and says which argument it was."""
import ctypes

import pytest
import torch

import paper_2609_32831_amd as uc

FAKE = 0x100000  # aligned non-null address; validation never dereferences it
FAR = 0x10000000000000  # and one that no other argument reaches
E, U, W = uc.UC_E_INVALID, uc.UC_E_UNSUPPORTED, uc.UC_E_WORKSPACE
L = uc.lib


def cache(**kw):
    d = dict(n_pages=40, page_rows=64, Hkv=4, D=128, group=64, codes_k=FAKE, codes_v=FAKE, scale_k=FAKE,
             scale_v=FAKE)
    d.update(kw)
    return uc.uc_page_cache(**d)


def call(f, args, **kw):
    """f with the arguments of `args` in order, some of them replaced."""
    assert set(kw) <= set(args), kw
    d = dict(args, **kw)
    for k, v in d.items():
        if isinstance(v, uc.uc_page_cache):
            d[k] = ctypes.byref(v)
        elif k == "sm_scale":
            d[k] = ctypes.c_float(v)
    return f(*d.values())


FREE = dict(S=3, page_rows=64, n_pages=40, table=FAKE, ld=8, len=FAKE, free_list=FAKE, pool=FAKE, ws=FAKE,
            ws_bytes=1 << 30, stream=None)
STEP = dict(S=3, page_rows=64, n_pages=40, len=FAKE, new_len=FAKE, table=FAKE, ld=8, free_list=FAKE, pool=FAKE,
            len_out=FAKE, q_start=FAKE, slots=FAKE, n_slots=16, pool_out=FAKE, refused=FAKE, stream=None)
APPEND = dict(cache=cache(), k=FAKE, v=FAKE, dt=uc.UC_BF16, ld=512, T=5, slots=FAKE, copies=FAKE, n_copies=2,
              stream=None)
READ = dict(cache=cache(), slots=FAKE, T=5, k=FAKE, v=FAKE, dt=uc.UC_BF16, ld=512, stream=None)
ATTEND = dict(cache=cache(), Hq=28, q=FAKE, dt=uc.UC_BF16, q_ld=28 * 128, T=5, S=3, max_q=3, q_start=FAKE, len=FAKE,
              table=FAKE, ld=8, sm_scale=0.1, o=FAR, lse=FAKE, ws=FAKE, ws_bytes=1 << 40, stream=None)
SELECT = dict(R=2, W=4, V=1000, logits=FAKE, dt=uc.UC_BF16, ld=1000, score=FAKE, done=FAKE, eos=2, pad=0,
              score_out=FAKE, parent=FAKE, token=FAKE, done_out=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None)
REORDER = dict(R=2, W=4, parent=FAKE, token=FAKE, table=FAKE, ld=8, len=FAKE, page_rows=64, table_out=FAKE,
               copies=FAKE, history=FAKE, history_out=FAKE, history_ld=20, n_history=19, stream=None)

PAGING = [(dict(page_rows=p), E) for p in (0, 8, 48, 2048, -64)]
PAGES = [(dict(n_pages=0), E), (dict(n_pages=1 << 25), E)]  # 2^25 pages of 64 rows pass 2^31


def ints(*names):
    return [({n: v}, E) for n in names for v in (None, FAKE + 2)]


def rows(*names):
    return [({n: v}, E) for n in names for v in (None, FAKE + 8)]


CASES = [
    ("uc_page_free", FREE, PAGING + PAGES + ints("table", "len", "free_list", "pool") +
     [(dict(S=0), E), (dict(ld=0), E), (dict(ws=None), W), (dict(ws=FAKE + 8), W), (dict(ws_bytes=39), W)]),
    ("uc_page_step", STEP, PAGING + PAGES + ints("len", "new_len", "table", "free_list", "pool", "len_out",
                                                 "q_start", "slots", "pool_out") +
     [(dict(S=0), E), (dict(ld=0), E), (dict(n_slots=-1), E), (dict(refused=None), E)]),
    ("uc_page_append", APPEND, rows("k", "v") + ints("slots", "copies") +
     [(dict(dt=7), E), (dict(dt=-1, T=0), E), (dict(ld=511), E), (dict(ld=516), E), (dict(T=-1), E),
      (dict(n_copies=-1), E), (dict(T=(1 << 25) + 1), U), (dict(n_copies=(1 << 20) + 1), U)]),
    ("uc_page_read", READ, rows("k", "v") + ints("slots") +
     [(dict(dt=3), E), (dict(ld=504), E), (dict(ld=514, dt=uc.UC_F32), E), (dict(T=-1), E),
      (dict(T=(1 << 25) + 1), U)]),
    ("uc_page_attend", ATTEND, rows("q", "o") + ints("q_start", "len", "table") +
     [(dict(Hq=0), E), (dict(Hq=30), E), (dict(dt=9), E), (dict(q_ld=28 * 128 - 8), E), (dict(q_ld=28 * 128 + 4), E),
      (dict(o=FAKE), E), (dict(o=FAKE + 5 * 28 * 256 - 16), E), (dict(o=FAKE - 16), E),
      (dict(q_ld=28 * 128 + 64, o=FAKE + 28 * 256), E),
      (dict(T=-1), E), (dict(S=0), E), (dict(max_q=0), E), (dict(ld=0), E), (dict(lse=FAKE + 2), E),
      (dict(sm_scale=0.0), E), (dict(sm_scale=-1.0), E), (dict(sm_scale=float("nan")), E),
      (dict(sm_scale=float("inf")), E), (dict(sm_scale=3e38), E), (dict(T=1 << 27), U), (dict(ld=1 << 30), U),
      (dict(S=1 << 30), U), (dict(T=1 << 22, ld=1 << 15), U), (dict(ws=None), W), (dict(ws=FAKE + 8), W),
      (dict(ws_bytes=16), W)]),
    ("uc_beam_select", SELECT, ints("score", "score_out", "parent", "token") +
     [(dict(R=0), E), (dict(W=0), E), (dict(W=33), E), (dict(V=3, pad=0, eos=-1), E), (dict(V=1 << 30, ld=1 << 30), E),
      (dict(R=1 << 22), U), (dict(dt=4), E), (dict(logits=None), E), (dict(logits=FAKE + 1), E),
      (dict(logits=FAKE + 2, dt=uc.UC_F32), E), (dict(ld=999), E), (dict(pad=-1), E), (dict(pad=1000), E),
      (dict(eos=-2), E), (dict(eos=1000), E), (dict(ws=None), W), (dict(ws=FAKE + 8), W), (dict(ws_bytes=16), W)]),
    ("uc_beam_reorder", REORDER, PAGING + ints("parent", "token", "table", "len", "table_out", "copies",
                                               "history_out") +
     [(dict(R=0), E), (dict(W=0), E), (dict(W=33), E), (dict(R=1 << 22), U), (dict(ld=0), E),
      (dict(ld=(1 << 22) + 1), E), (dict(n_history=-1), E), (dict(n_history=20), E),
      (dict(n_history=(1 << 22) + 1, history_ld=1 << 23), E), (dict(history=FAKE + 2), E)]),
]


@pytest.mark.parametrize("name,args,bad", CASES, ids=[c[0] for c in CASES])
def test_refusals(name, args, bad):
    f = getattr(L, name)
    for kw, status in bad:
        assert call(f, args, **kw) == status, (kw, uc.uc_last_error())
        assert uc.uc_last_error(), kw


@pytest.mark.parametrize("name,args", [("uc_page_append", APPEND), ("uc_page_read", READ), ("uc_page_attend", ATTEND)])
def test_refusals_of_caches(name, args):
    f = getattr(L, name)
    wrong = [dict(page_rows=p) for p in (8, 48, 2048)] + [dict(n_pages=n) for n in (0, -1, 1 << 25)]
    wrong += [dict(D=96), dict(D=256), dict(Hkv=0), dict(Hkv=4097), dict(group=16), dict(group=256),
              dict(D=64, group=128), dict(group=0)]
    wrong += [{k: v} for k in ("codes_k", "codes_v", "scale_k", "scale_v") for v in (None, FAKE + 8)]
    for kw in wrong:
        assert call(f, args, cache=cache(**kw)) == E, (kw, uc.uc_last_error())
    assert call(f, args, cache=None) == E


def test_calls_without_work():
    """Nothing to do is no error, and launches nothing."""
    assert call(L.uc_page_append, APPEND, T=0, n_copies=0, k=None, v=None, slots=None, copies=None) == uc.UC_OK
    assert call(L.uc_page_read, READ, T=0, k=None, v=None, slots=None) == uc.UC_OK
    assert call(L.uc_page_attend, ATTEND, T=0, q=None, o=None, lse=None, ws=None, ws_bytes=0) == uc.UC_OK


def test_workspace_sizes():
    free, attend, beam = (L.uc_page_free_workspace_size, L.uc_page_attend_workspace_size,
                          L.uc_beam_select_workspace_size)
    assert free(0) == free(-3) == 0 and 100000 <= free(100000) < 110000
    c = cache()
    one, prompt = attend(ctypes.byref(c), 28, 3, 3, 1), attend(ctypes.byref(c), 28, 300, 3, 200)
    assert 0 < one < prompt
    for bad in ((30, 3, 3, 1), (0, 3, 3, 1), (28, -1, 3, 1), (28, 3, 0, 1), (28, 3, 3, 0)):
        assert attend(ctypes.byref(c), *bad) == 0
    assert attend(ctypes.byref(cache(D=96)), 28, 3, 3, 1) == 0
    assert beam(2, 4, 1000) > 0
    for bad in ((0, 4, 1000), (2, 0, 1000), (2, 33, 1000), (2, 4, 3), (2, 4, 1 << 30), (1 << 22, 4, 1000)):
        assert beam(*bad) == 0


def ints_on_host(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def test_wrappers_refuse_what_does_not_fit():
    """Tensors off the GPU, of another type, shape or layout, before the library
    is called."""
    c = uc.page_cache(4, 16, 2, 64, 32, device="cpu")
    t, n = ints_on_host(3, 2), ints_on_host(3)
    x = torch.zeros(3, 2, 64)
    bad = [
        lambda: uc.uc_page_free(t, n, 16, ints_on_host(4), ints_on_host(2)),
        lambda: uc.uc_page_step(n, n, t, 16, ints_on_host(4), ints_on_host(2), n, ints_on_host(4), n,
                                ints_on_host(2), torch.zeros(3, dtype=torch.uint8)),
        lambda: uc.uc_page_append(c, x, x, n),
        lambda: uc.uc_page_read(c, n, x, x),
        lambda: uc.uc_page_attend(c, x, ints_on_host(4), n, t, 1, 0.1, x),
        lambda: uc.uc_beam_select(torch.zeros(1, 2, 9), torch.zeros(1, 2), None, -1, 0, torch.zeros(1, 2),
                                  ints_on_host(1, 2), ints_on_host(1, 2)),
        lambda: uc.uc_beam_reorder(ints_on_host(1, 3), None, t, n, 16, t, ints_on_host(3, 3)),
        lambda: uc.page_cache(4, 16, 2, 64, 128, device="cpu"),
        lambda: uc.PageCache(*(y.long() for y in c.t.values())),
        lambda: uc.PageCache(c.t["codes_k"], c.t["codes_v"][:2], c.t["scale_k"], c.t["scale_v"]),
        lambda: uc.PageCache(c.t["codes_k"].transpose(1, 2), c.t["codes_v"], c.t["scale_k"], c.t["scale_v"]),
    ]
    for f in bad:
        with pytest.raises(AssertionError):
            f()


def test_struct_layout():
    assert ctypes.sizeof(uc.uc_page_cache) == 56 and uc.uc_page_cache.codes_k.offset == 24
