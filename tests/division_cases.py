"""Calls of attention over pages whose work is divided in each of its ways, at every head_dim: a step for a workgroup, two steps, and runs
of one line that go on from pair to pair."""
import numpy as np

# (way, head_dim, group, kv heads, query heads, sequences, capacity, most new rows)
CASES = [("step", 64, 64, 2, 12, 20, 256, 3), ("step", 128, 128, 1, 9, 30, 192, 2), ("step", 256, 64, 1, 9, 24, 192, 3),
         ("two", 64, 64, 2, 12, 75, 256, 3), ("two", 128, 64, 2, 2, 150, 256, 2), ("two", 128, 128, 1, 9, 140, 256, 2), ("two", 256, 256, 1, 9, 140, 128, 2),
         ("line", 64, 64, 1, 9, 300, 768, 2), ("line", 128, 64, 2, 12, 130, 768, 3), ("line", 128, 128, 2, 2, 240, 768, 2),
         ("line", 256, 64, 1, 10, 160, 768, 2), ("line", 256, 256, 2, 2, 130, 768, 2)]


def lengths_and_rows(case):
    """Lengths of the sequences and their numbers of new rows: `two` takes sequences that fill their last steps, the others any."""
    way, _, _, _, _, n, N, most = case
    rng = np.random.RandomState(N + n)
    lens = rng.randint(N * 5 // 8, N + 1, n) if way == "two" else rng.randint(0, N + 1, n)
    rows = rng.randint(0 if way != "two" else most, most + 1, n)
    lens[[3, 5]], rows[[4, 6]] = (0, 1), (0, 1)
    return lens.astype(np.int32), rows.astype(np.int32)
