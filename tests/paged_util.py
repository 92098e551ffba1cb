"""Plain numpy forms of the paged cache's integer work, and helpers shared by its tests."""
import numpy as np
import torch


def plan_oracle(cached, new, table, P, max_tokens, held=None, free=(), next_free=0):
    """What sdvg.h says of sdvg_page_plan, one request and one token after the other, in Python integers."""
    table = np.array(table, dtype=np.int64)
    R, W = table.shape
    q_start, kv_lens, positions, slots, held_out = [0], [], [], [], []
    cursor = next_free
    for r in range(R):
        c, n = max(0, int(cached[r])), max(0, int(new[r]))
        need = min(-(-(c + n) // P), W)
        if held is not None:
            h = max(0, int(held[r]))
            got = 0
            for j in range(h, need):
                ok = 0 <= cursor < len(free)
                table[r, j] = free[cursor] if ok else -1
                got += ok
                cursor += 1
            held_out.append(h + got)
        n = min(n, max_tokens - q_start[-1])
        q_start.append(q_start[-1] + n)
        kv_lens.append(c + n)
        for i in range(n):
            pos = c + i
            page = int(table[r, pos // P]) if pos // P < W else -1
            if held is not None and pos // P >= max(int(held[r]), need):
                page = -1
            positions.append(pos)
            slots.append(page * P + pos % P if page >= 0 else -1)
    pad = max_tokens - len(slots)
    return dict(table=table, q_start=np.array(q_start), kv_lens=np.array(kv_lens, dtype=np.int64),
                positions=np.array(positions + [0] * pad, dtype=np.int64), slots=np.array(slots + [-1] * pad, dtype=np.int64),
                held=np.array(held_out, dtype=np.int64), next_free=cursor)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
