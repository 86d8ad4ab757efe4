"""Block tables and slots, one sequence and one page after the other."""
import numpy as np


def block_tables(want, page_tokens, table, held, stack):
    """table [B, max_blocks], held [B], stack: list of free pages, its top last.  Returns (table, held, stack, refused) afterwards."""
    table, held, stack = np.array(table), list(held), list(stack)
    B, most = table.shape
    need = [-(-max(int(w), 0) // page_tokens) for w in want]
    refused = [2 if n > most else 0 for n in need]
    for s in range(B):
        if not refused[s] and need[s] < held[s]:
            stack += [int(p) for p in table[s, need[s]:held[s]]]
            held[s] = need[s]
    served = True
    for s in range(B):
        if refused[s] or need[s] <= held[s]:
            continue
        served = served and need[s] - held[s] <= len(stack)
        if not served:
            refused[s] = 1
            continue
        while held[s] < need[s]:
            table[s, held[s]] = stack.pop()
            held[s] += 1
    return table, held, stack, refused


def slot_map(node_offsets, NN, cache_lens, table, page_tokens, n_pages, held=None, accept_path=None, accept_len=None):
    """(slots [NN], new lengths)."""
    slots, new = np.full(NN, -1, np.int64), np.array(cache_lens, np.int64)
    for s in range(len(node_offsets) - 1):
        a, b = int(node_offsets[s]), int(node_offsets[s + 1])
        rows = list(range(a, b))
        if accept_path is not None and b > a:
            rows = [a] + [a + int(r) for r in accept_path[s][:max(0, int(accept_len[s]))]]
        pages = table.shape[1] if held is None else min(max(int(held[s]), 0), table.shape[1])
        for row in rows:
            t = int(new[s])
            if t >= pages * page_tokens:
                break
            page = int(table[s, t // page_tokens])
            if 0 <= page < n_pages and a <= row < b:
                slots[row] = page * page_tokens + t % page_tokens
            new[s] += 1
    return slots, new
