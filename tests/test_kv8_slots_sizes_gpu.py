"""Places for more tokens or requests than splash_kv_slots has: refused before memory for the outputs (12 bytes a place) is asked for."""
import pytest
import torch

from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("places", [2 ** 31 - 1, 2 ** 33, 2 ** 40, 2 ** 62, 2 ** 63 - 1])
def test_more_places_than_there_can_be(places):
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    args = (table, ints(0, 5), ints(1, 1), ints(3, 4, 5), ints(0))
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.max_memory_allocated()
    with pytest.raises(B.SplashError, match="places"):
        B.splash_kv_slots(*args, places)
    assert torch.cuda.max_memory_allocated() == before
    assert (table == -1).all()


def test_more_requests_than_a_call_takes():
    n = 16385
    zeros = torch.zeros(n, dtype=torch.int32, device="cuda")
    with pytest.raises(B.SplashError, match="requests"):
        B.splash_kv_slots(torch.zeros((n, 1), dtype=torch.int32, device="cuda"), zeros, zeros, zeros, zeros[:1], 10)
