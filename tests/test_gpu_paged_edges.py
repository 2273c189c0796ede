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
from test_gpu_paged import DT, _case, check_sized, i32, make_cache, put_rows  # noqa: E402


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
