"""Layouts that the paged calls' binding takes, and calls that launch nothing (so
this runs without a GPU)."""
import threading

import pytest
import torch

import paper_2609_32831_amd as uc
from test_abi_paged import ATTEND, FREE, SELECT, STEP, E, L, U, call


def test_a_single_token_has_no_distance():
    """Keys and values of one token: a slice of a fused projection beside a
    tensor of its own."""
    fused, own = torch.zeros(1, 9, 64), torch.zeros(1, 2, 64)
    assert uc._token_rows(own, fused[:, 2:4], 1, 2, 64) == 128
    assert uc._token_rows(fused[:, 2:4], own, 1, 2, 64) == 128
    # and a single head none either
    x, y = torch.zeros(5, 3, 64)[:, 1:2], torch.zeros(5 * 192).as_strided((5, 1, 64), (192, 7, 1))
    assert y.stride(1) != x.stride(1)
    assert uc._token_rows(x, y, 5, 1, 64) == 192
    for k, v, T in ((fused.expand(3, 9, 64)[:, :2], torch.zeros(3, 2, 64), 3),  # tokens at different distances
                    (torch.zeros(1, 64, 2).transpose(1, 2), own, 1), (own, own.half(), 1),
                    (own, torch.zeros(1, 4, 64)[:, ::2], 1)):
        with pytest.raises(AssertionError):
            uc._token_rows(k, v, T, 2, 64)


def test_rows_of_logits_at_one_distance():
    x = torch.zeros(3, 4, 10)
    assert uc._logit_rows(x) == 10
    assert uc._logit_rows(x[:, :1]) == 40  # one beam of four: every fourth row
    assert uc._logit_rows(x[:1, 1:3, 2:]) == 10
    assert uc._logit_rows(x[1:2, 1:2, :7]) == 7
    assert uc._logit_rows(torch.zeros(10, 3, 1).transpose(0, 1)[:, :1]) == 1
    for bad in (x[:, :2], x[..., ::2], x.transpose(1, 2)):
        with pytest.raises(AssertionError):
            uc._logit_rows(bad)


@pytest.mark.skipif(torch.cuda.is_available(), reason="a launch has to fail, as it does without a GPU")
def test_a_failed_launch_leaves_the_last_kernel():
    got = []

    def run():
        for path in (uc.UC_PATH_AUTO, uc.UC_PATH_VALU):
            prev = uc.uc_set_path(path)
            got.append((call(L.uc_page_attend, ATTEND), uc.uc_last_kernel()))
            uc.uc_set_path(prev)

    t = threading.Thread(target=run)  # the name is the calling thread's: none yet
    t.start()
    t.join()
    assert got == [(uc.UC_E_DEVICE, ""), (uc.UC_E_DEVICE, "")]


def test_limits_of_the_kernels_indexes():
    """Sizes whose next stride passes 31 bits are refused, not launched."""
    most = (1 << 31) - 1
    for kw in (dict(S=most), dict(ld=most), dict(ld=(1 << 30) + 1)):
        assert call(L.uc_page_free, FREE, **kw) == U and uc.uc_last_error(), kw
    for kw in (dict(S=most), dict(ld=most), dict(n_slots=most), dict(n_slots=(1 << 30) + 1)):
        assert call(L.uc_page_step, STEP, **kw) == U and uc.uc_last_error(), kw
    for W, V in ((1, most), (1, (1 << 30) + 1), (2, (1 << 29) + 1)):
        assert call(L.uc_beam_select, SELECT, W=W, V=V, ld=V) == E and uc.uc_last_error(), (W, V)
        assert L.uc_beam_select_workspace_size(1, W, V) == 0
    assert L.uc_beam_select_workspace_size(1, 2, 1 << 29) > 0
