"""mars_kv_reserve where a call wants more pages than 32 bits count."""
import pytest
import torch

from paper_2601_15498_amd import cache as C

pytestmark = pytest.mark.gpu


def test_wants_beyond_what_32_bits_count():
    """1 024 requests of 2^24 tokens in pages of 8 want 2^31 pages.  The first can have its own, the others go without."""
    print("2^31 pages", flush=True)
    P, B, each = 8, 1024, 1 << 21
    pages = each + 5
    table = torch.full((B, each), -1, dtype=torch.int32, device="cuda")
    lens, held = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[7] = 1                                      # (nobody's of this call)
    pool = torch.zeros((1, pages, 1, P * 68), dtype=torch.uint8, device="cuda")
    status = C.mars_kv_reserve(pool, table, lens, held, refs, 1 << 24, page_size=P)
    assert status.tolist() == [0] + [C.MARS_KV_NO_PAGES] * (B - 1)
    assert held.tolist() == [each] + [0] * (B - 1) and (table[1:] == -1).all()
    got = torch.arange(each, dtype=torch.int32, device="cuda")
    assert torch.equal(table[0], torch.where(got < 7, got, got + 1))
    assert int(refs.sum()) == each + 1 and (refs[: each + 1] == 1).all()
