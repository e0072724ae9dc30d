"""One token of many rows, some or all of one slot: rows of a slot far apart, and a time that grows with the rows alone."""
import pytest
import torch

from paper_2609_34318_amd import hydra
from test_gpu_step import BF16, check, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [[0, 1023, 1024, 2047, 2049, 4999], [4998, 4999], [7, 4097], list(range(1020, 3080, 5))], ids=str)
def test_rows_of_a_slot_far_apart(rows):
    n = 5000
    x = draw(len(rows), n, 40, 1, 1, 64, 64)
    slots = [40 + i for i in range(n)]  # padding, but for the rows of slot 11, of 3 and of 5
    for r in rows:
        slots[r] = 11
    slots[1], slots[2], slots[3000], slots[4000] = 3, 5, 5, 3
    c = {t: y.cuda() for t, y in x.items()}
    o = torch.full((n, 1, 64), 7.0, dtype=BF16, device="cuda")
    before = c["state"].clone()
    hydra.linear_step(c["q"], c["k"], c["v"], c["decay"], c["state"], o, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"))
    check(x, slots, o, c["state"], before, 64)


def test_a_row_of_a_long_slot_costs_what_one_of_a_short_slot_does():
    """All rows of one slot are a walk of one after another, each with the same work: a row of 32K at most twice the time of
    one of 2K (the search for the next row, if it went on to the last one, would take 16 times as long)."""
    def per_row(n):
        q, k, v = (torch.randn((n, 1, 64), device="cuda").to(BF16) for _ in range(3))
        decay, state, o = torch.full((1,), -0.01, device="cuda"), torch.zeros((1, 1, 64, 64), device="cuda"), torch.empty_like(q)
        slots = torch.zeros(n, dtype=torch.int32, device="cuda")
        best = float("inf")
        for i in range(4):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            hydra.linear_step(q, k, v, decay, state, o, slots=slots)
            end.record()
            end.synchronize()
            if i:
                best = min(best, start.elapsed_time(end) / n)
        return best
    short, long = per_row(2048), per_row(32768)
    print(f"a row of 2048: {short * 1e3:.2f} us, of 32768: {long * 1e3:.2f} us")
    assert long <= 2 * short, (short, long)
