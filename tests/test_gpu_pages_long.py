"""Pages of sequences at the end of the tokens that 31 bits count."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_own_at_the_last_token():
    """Of a sequence of 2^31 - 1 tokens, the page behind them (kept from a rollback) holds none: it is replaced without a copy."""
    from paper_2606_03113_amd import lede
    say("own, 2^31 - 1 tokens")
    width, i32 = (1 << 25) + 2, dict(dtype=torch.int32, device="cuda")
    tables = torch.full((2, width), -1, **i32)
    last = (1 << 25) - 1      # the last tokens' place
    tables[0, last:last + 2] = torch.tensor([3, 4], **i32)
    tables[1, :2] = torch.tensor([3, 4], **i32)
    shares = torch.tensor([0, 0, 0, 1, 1, 0, 0], **i32)
    m = lede.op_cache_own(torch.tensor([(1 << 31) - 1, 128], **i32), torch.tensor([100, 0], **i32), torch.tensor([last + 2, 2], **i32),
                          torch.tensor([6, 5, 2], **i32), torch.tensor([0], **i32), tables, shares, 1)
    assert m.status.tolist() == [0, 1, 2, -1] and m.pairs.tolist() == [[3, 6]]
    assert tables[0, last:].tolist() == [6, 5, -1] and tables[1, :3].tolist() == [3, 4, -1]
    assert shares.tolist() == [0] * 7
