"""Edges of the paged attention and of the beam selection, against the plain
reference in 64 bits.  Bounds are those of test_gpu_paged.py, or derived beside
the test."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paged_ref as ref  # noqa: E402
import paper_2609_32831_amd as uc  # noqa: E402
from test_gpu_paged import DT, _case, check_beams, check_sized, f64, half, i32, make_cache, put_rows, select  # noqa: E402


# ---------------------------------------------------------------- queries

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("size", [200.0, 600.0, -1000.0, 2100.0, 30000.0])
@pytest.mark.parametrize("tokens", [3, 70])
def test_queries_of_one_sign(tokens, size, D, group, dtype):
    """Queries whose elements are alike, so that the sums over a group are as
    many times larger, over keys that leave the logits ordinary.  Rows of
    ordinary queries lie between them."""
    _case(test="one_sign", tokens=tokens, size=size, D=D, group=group, dtype=dtype)
    lens, Hkv, G = [150], 2, 2
    cache, table = make_cache(lens, 16, Hkv, D, group, 101)
    r = np.random.default_rng(102)
    put_rows(cache, table, 0, range(150), r.standard_normal((150, Hkv, D)) / abs(size), r.standard_normal((150, Hkv, D)))
    q = size * (1 + 0.01 * r.standard_normal((tokens, Hkv * G, D)))
    q[1::3] = r.standard_normal(q[1::3].shape)
    q = torch.tensor(q, device="cuda").to(DT[dtype])
    o, lse = torch.empty_like(q), torch.empty(tokens, Hkv * G, device="cuda")
    uc.uc_page_attend(cache.device(uc), q, i32([0, tokens]), i32(lens), i32(table), tokens, 0.1, o, lse)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    check_sized(cache, q, [0, tokens], lens, table, float(np.float32(0.1)), o, lse, dtype)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("tokens", [3, 70])
def test_queries_as_large_as_they_may_be(tokens, group):
    """Elements up to 2^100, of one sign and of both, over keys as small."""
    _case(test="largest", tokens=tokens, group=group)
    lens, Hkv, G, D = [150], 2, 2, 128
    cache, table = make_cache(lens, 16, Hkv, D, group, 105)
    r = np.random.default_rng(106)
    put_rows(cache, table, 0, range(150), r.standard_normal((150, Hkv, D)) * 2.0 ** -99, r.standard_normal((150, Hkv, D)))
    q = r.random((tokens, Hkv * G, D)) + 1
    q[::2] *= r.choice([-1, 1], q[::2].shape)
    q = torch.tensor(q * 2.0 ** 99, device="cuda").bfloat16()
    o, lse = torch.empty_like(q), torch.empty(tokens, Hkv * G, device="cuda")
    uc.uc_page_attend(cache.device(uc), q, i32([0, tokens]), i32(lens), i32(table), tokens, 0.1, o, lse)
    check_sized(cache, q, [0, tokens], lens, table, float(np.float32(0.1)), o, lse, "bf16")


@pytest.mark.parametrize("peak", [100, 61000])
@pytest.mark.parametrize("tokens,G", [(3, 1), (4096, 16)])
def test_a_long_tail_under_a_peak(tokens, G, peak):
    """One key takes nearly all, and some 65500 others, each of weight 2^-25.5
    of it, take 2^-9.5 together.  Every value is 1 but the peak's, which is
    zero, so the output is the tail's share.  (65536 query rows of a KV head:
    as many blocks as there are pieces, so a piece holds most of a block's
    rows.)

    A prompt's weights are rounded to fp16: by 2^-12 of themselves, or by 2^-25
    where they are subnormal, with the largest at 2^7 at least: n 2^-32 of the
    values.  Single tokens: 2^-18 of the weights."""
    _case(test="tail", tokens=tokens, G=G, peak=peak)
    n, D, P = 65600, 64, 64
    r = np.random.default_rng(peak)
    one = 0x3F80 << 16  # a minimum of 1, steps of 0
    pages = n // P
    shape = (pages, 1, P, D // 2)
    k, v = (torch.full((pages, 1, P, 1), w, dtype=torch.int32, device="cuda") for w in (0, one))
    table = r.permutation(pages)
    page = int(table[peak // P])
    k[page, 0, peak % P], v[page, 0, peak % P] = one, 0
    codes = torch.zeros(shape, dtype=torch.uint8, device="cuda")
    q = torch.ones(tokens, G, D, device="cuda", dtype=torch.float16)
    scale = np.float32(25.5 * np.log(2) / D)
    o, lse = torch.empty_like(q), torch.empty(tokens, G, device="cuda")
    uc.uc_page_attend(uc.PageCache(codes, codes, k, v), q, i32([0, tokens]), i32([n]), i32(table[None]), tokens,
                      float(scale), o, lse)
    logit = D * float(scale)
    tail = (n - tokens + np.arange(tokens))[:, None] * np.exp(-logit)  # of the peak's weight
    want, want_lse = (tail / (1 + tail))[..., None], logit + np.log1p(tail)
    err = np.abs(f64(o) - want)
    print(f"want {want.max():.3e} off {err.max():.3e}", flush=True)
    # the logit of 17.7: sums of D terms of up to 22 times its size, by 2^-24 each
    bound = (half("f16") + 2.0 ** -12 + logit * D * 22 * 2.0 ** -24) * want + n * 2.0 ** -32
    assert np.all(err <= bound)
    assert np.all(np.abs(f64(lse) - want_lse) <= 1e-5 * want_lse + 2.0 ** -12)


# ---------------------------------------------------------------- starts and lengths

@pytest.mark.parametrize("path", ["auto", "valu"])
@pytest.mark.parametrize("G", [2, 32])
@pytest.mark.parametrize("start,lens,rows", [
    ([-5, 3, 900], [64, 40], [64, 40]),
    ([0, 5, 2], [10 ** 9, -4], [64, 0]),
    ([1, 3, 6], [64, -7], [64, 0]),
    ([6, 6, 6], [64, 64], [64, 64]),
    ([900, -3, 4], [64, 64], [64, 64]),
    ([2, 5, 3], [64, 64], [64, 64]),
])
def test_starts_and_lengths_are_held_to_the_arrays(start, lens, rows, G, path):
    """A sequence's tokens and rows count as far as the arrays go; tokens of no
    sequence keep what they have.  (32 heads a KV head: the prompt kernel.)"""
    _case(test="held", start=start, lens=lens, G=G, path=path)
    cache, table = make_cache([64, 64], 16, 1, 64, 32, 41)
    q = torch.randn(6, G, 64, device="cuda", dtype=torch.bfloat16)
    o, lse = torch.full_like(q, 5.0), torch.full((6, G), 5.0, device="cuda")
    prev = uc.uc_set_path(uc.UC_PATH_VALU if path == "valu" else uc.UC_PATH_AUTO)
    try:
        uc.uc_page_attend(cache.device(uc), q, i32(start), i32(lens), i32(table), 6, 0.1, o, lse)
        torch.cuda.synchronize()
    finally:
        uc.uc_set_path(prev)
    want, want_lse = ref.attend(cache, f64(q), np.clip(start, 0, 6), rows, table, float(np.float32(0.1)))
    none = np.isnan(want).all((1, 2))
    assert torch.all(o[torch.from_numpy(none)] == 5.0) and torch.all(lse[torch.from_numpy(none)] == 5.0)
    some = torch.from_numpy(~none)
    got, got_lse, want, want_lse = f64(o[some]), f64(lse[some]), want[~none], want_lse[~none]
    empty = np.isneginf(want_lse)
    assert np.array_equal(empty, np.isneginf(got_lse)) and np.all(got[empty] == 0)
    assert np.all(np.abs(got - want) <= 2e-3 + half("bf16") * np.abs(want))
    assert np.allclose(got_lse[~empty], want_lse[~empty], rtol=1e-5, atol=1e-4)


def test_tokens_that_many_sequences_claim():
    """800 sequences of the same 62500 tokens over 128000 rows hold more work
    than a call's indexes count: no prompt is taken, and what was there stays.
    The next call is an ordinary one."""
    T, G, D, P, m = 62500, 16, 64, 1024, 800
    cache = uc.page_cache(125, P, 1, D, 64)
    for x in cache.t.values():
        x.zero_()
    start = i32([0, T] * m + [0])
    lens, table = i32([128000] * (2 * m)), torch.arange(125, device="cuda", dtype=torch.int32).repeat(2 * m, 1)
    q = torch.zeros(T, G, D, device="cuda", dtype=torch.bfloat16)
    o = torch.full_like(q, 5.0)
    uc.uc_page_attend(cache, q, start, lens, table, T, 0.1, o)
    assert torch.all(o == 5.0)
    uc.uc_page_attend(cache, q[:300], i32([0, 300]), lens[:1], table[:1], 300, 0.1, o[:300])
    assert torch.all(o[:300] == 0) and torch.all(o[300:] == 5.0)


# ---------------------------------------------------------------- equal beams

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,W,V", [(2, 4, 1), (3, 4, 37), (2, 3, 1501), (2, 5, 32003), (40, 8, 4099), (1, 4, 131071)])
def test_equal_beams_go_by_the_lower_index(R, W, V, dtype):
    """Beams of the same logits and the same score have the same totals,
    wherever in memory their rows begin, so the lower beam comes first."""
    if W > V:
        V = W
    _case(test="equal_beams", R=R, W=W, V=V, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(R, 1, V, generator=g, device="cuda") * 3
    for pad in (0, 1, 3):  # rows further apart than they are long
        y = torch.zeros(R, W, V + pad, device="cuda").to(DT[dtype])
        y = y[:, :, pad:]
        y.copy_(x.expand(R, W, V))
        score = torch.full((R, W), -7.25, device="cuda")
        done = torch.zeros(R, W, dtype=torch.uint8, device="cuda")
        check_beams(select(y, score, done, -1, 0), ref.beam_select(f64(y), f64(score), done.cpu().numpy(), -1, 0))
