"""mars_kv_commit where the root's own row has no page: its position is the first behind the committed tokens, whatever was accepted."""
import numpy as np
import pytest
import torch

from paper_2601_15498_amd import cache as C
from tests.cache_util import Filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("D,P,layers", [(64, 8, 2), (128, 16, 1)])
def test_a_root_without_a_page_is_not_committed(D, P, layers, alias):
    print("commit root", D, P, layers, alias, flush=True)
    # every token of requests 0 .. 2 fills its pages; request 0 fills the table too, request 3 has room for the root alone, request 4 for all
    lens = (3 * P, P, 0, 2 * P - 1, 5)
    f = Filled(np.random.default_rng(P), lens, 0, 2, D, P, layers=layers, sequences=6, rows=False, stale=3, width=3)
    assert [int(f.held[s]) for s in f.seqs] == [3, 1, 0, 2, 1]
    d = f.to()
    before = d["pool"].clone()
    N = 4
    accept = torch.zeros(5, dtype=torch.int32, device="cuda")
    path = torch.full((5, N), -1, dtype=torch.int32, device="cuda")
    status = torch.full((5,), 77, dtype=torch.int32, device="cuda")
    new = d["lens"] if alias else torch.full_like(d["lens"], -5)
    C.mars_kv_commit(d["pool"], d["table"], d["lens"], accept, path, page_size=P, seqs=d["seqs"], new_lens=None if alias else new, status=status)
    want = f.lens.copy() if alias else np.full(6, -5, np.int32)
    for b, s in enumerate(f.seqs):
        want[s] = lens[b] + (b >= 3)
    assert status.tolist() == [C.MARS_KV_NO_PAGES] * 3 + [C.MARS_KV_OK] * 2
    assert np.array_equal(new.cpu().numpy(), want)
    assert torch.equal(d["pool"], before)
    # what is no path stays that, with or without a page for the root
    accept.fill_(N)
    C.mars_kv_commit(d["pool"], d["table"], d["lens"].clone(), accept, path, page_size=P, seqs=d["seqs"], new_lens=new, status=status)
    assert status.tolist() == [C.MARS_KV_BAD_PATH] * 5 and np.array_equal(new.cpu().numpy()[f.seqs], want[f.seqs] if alias else np.array(lens))
