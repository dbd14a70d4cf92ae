"""Page bounds under promises of many more tokens than the sequences bring, up to the largest number: the bounds of a tight promise, and
no more work than the table has entries."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_kv,bits", [(256, 2), (3, 4), (1, 3)])
def test_any_larger_promise_gives_the_same_bounds(n_kv, bits):
    import torch
    from paper_2609_38121_b200 import binding as B
    T = np.tile(np.eye(128, dtype=np.float32), (n_kv, 1, 1))
    c = B.PagedCache(n_kv, n_kv, bits, 2, 300, 4, 64, 1, 0.96, 0.92, T, T, page_bounds=True)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    slot, seq_len, cu = ints([0, 1]), ints([0, 0]), ints([0, 290, 430])
    gen = torch.Generator(device="cuda").manual_seed(bits)
    K, V = (torch.randn((430, n_kv, 128), generator=gen, device="cuda").to(torch.bfloat16).view(torch.int16) for _ in range(2))
    B.append(c.desc, 2, slot, seq_len, cu, 430, 290, K, V)
    want = None
    for max_new in (290, 300, 330, 1000, 1 << 30, (1 << 31) - 1):
        c.bounds.fill_(77)
        c.exponents.fill_(99)
        B.update_page_bounds(c.desc, 2, slot, seq_len, cu, max_new, c.bounds, c.exponents)
        got = c.bounds.clone(), c.exponents.clone()
        want = want or got
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), max_new
    assert c.status() == 0 and not bool((want[1][:5] == 99).any())
    B.update_page_bounds(c.desc, 2, slot, ints([321, 140]), cu, (1 << 31) - 1, c.bounds, c.exponents)      # a length behind the table's end
    assert c.status() == B.DEV_PAGE_TABLE_FULL
