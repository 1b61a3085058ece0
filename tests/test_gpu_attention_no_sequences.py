"""attention_paged over packed rows without a sequence, through the C entry: every row is one of none, so it
is zeroed as zero_rest asks or left."""
import math

import pytest
import torch

from paper_2609_04910_amd import attention as at

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rest", [0, at.REST_OUT, at.REST_OUT | at.REST_LSE])
@pytest.mark.parametrize("T,width", [(2, 3), (300, 3), (3, 400)])
def test_rows_of_no_sequence(T, width, rest):
    q = torch.ones((T, 4, 64), dtype=torch.float16, device="cuda")
    pages = torch.ones((2, 4, 16, 2, 64), dtype=torch.float16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((4, T), 7.0, device="cuda")
    offs = torch.zeros(1, dtype=torch.int32, device="cuda")
    p = at.Problem(0, T, 0, 4, 2, 64, 64, 0, at.gs.GS_F16, 1, 1, rest, 0.125)
    rows = [at.Array(t.data_ptr(), 0, 4 * 64, 64) for t in (q, out)]
    kv = [at.Array(t.data_ptr(), *t.stride()[:3]) for t in pages]
    cache = at.Cache(kv[0], kv[1], 4, 16, width, None, None)
    lib = at.load()
    need = lib.gs_attention_paged_workspace_size(at._ref(p), at._ref(cache))
    workspace = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    assert lib.gs_attention_paged(at._ref(p), at._ref(rows[0]), at._ref(cache), offs.data_ptr(), at._ref(rows[1]), lse.data_ptr(),
                                  workspace.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    assert (out == (0 if rest else 7)).all()
    assert (lse == (-math.inf if rest & at.REST_LSE else 7)).all()
