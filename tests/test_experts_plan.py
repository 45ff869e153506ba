"""The routing of the expert block (host logic, no GPU)."""
import pytest
import torch

from paper_2608_01653_gb300.experts import plan


@pytest.mark.parametrize("tokens,topk,experts", [(1, 1, 1), (1, 8, 64), (7, 3, 4), (50, 2, 5), (0, 2, 3)])
@pytest.mark.parametrize("dropped", [False, True])
def test_plan(tokens, topk, experts, dropped):
    g = torch.Generator().manual_seed(tokens + experts)
    ids = torch.randint(-1 if dropped else 0, experts + (2 if dropped else 0), (tokens, topk), generator=g)
    rows, offsets, slots = plan(ids, experts)
    assert rows.dtype == offsets.dtype == slots.dtype == torch.int32
    o = offsets.tolist()
    taken = int(((ids >= 0) & (ids < experts)).sum())
    assert o[0] == 0 and o[-1] == taken and all(a <= b for a, b in zip(o, o[1:]))
    seen = set()
    for t in range(tokens):
        for j in range(topk):
            e, r = int(ids[t, j]), int(slots[t, j])
            if 0 <= e < experts:
                assert o[e] <= r < o[e + 1] and int(rows[r]) == t and r not in seen
                seen.add(r)
            else:
                assert r == -1
    for e in range(experts):                       # stable: an expert's rows come in the tokens' order
        part = rows[o[e]:o[e + 1]].tolist()
        assert part == sorted(part)
