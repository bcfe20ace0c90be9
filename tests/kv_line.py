"""What each CTA of the attention's tile kernel has to do with a batch, from the sizes alone."""
ROWS, KEYS, OVERHEAD, FEW_ROWS, SEQS = 256, 64, 5, 32, 1024


def shares(sizes, kv_heads, group, window=0, n_ctas=148, limit=FEW_ROWS, whole=False):
    """[[(blocks, halves) of each unit or piece of one] for each CTA] of the first launch; sizes: (new rows, positions)."""
    line = []                                 # (blocks, halves) of every unit
    for n, length in sizes[:SEQS]:
        rows = n * group
        if rows <= limit:
            continue
        tiles = []
        for r0 in range(0, rows, ROWS):
            r1 = min(rows, r0 + ROWS) - 1
            hi, lo = max(0, length - n + r1 // group + 1), max(0, length - n + r0 // group + 1 - window) if window else 0
            tiles.append((max(1, -(-hi // KEYS) - lo // KEYS), 2 if r1 - r0 >= ROWS // 2 else 1))
        line += tiles * kv_heads
    total = sum(b + OVERHEAD for b, _ in line)
    n_ctas = min(n_ctas, total)
    out = [[] for _ in range(n_ctas)]
    at = 0
    for blocks, halves in line:
        for c in range(at * n_ctas // total, n_ctas):
            begin, end = c * total // n_ctas, (c + 1) * total // n_ctas
            if begin >= at + blocks:
                break
            if whole:
                if begin <= at < end:
                    out[c].append((blocks, halves))
            else:
                count = min(end, at + blocks) - max(begin, at)
                if count > 0:
                    out[c].append((count, halves))
        at += blocks + OVERHEAD
    return out


def most(sizes, kv_heads, group, **kw):
    """(units, blocks) of the CTA that has the most of them."""
    all_of = shares(sizes, kv_heads, group, **kw)
    return max(map(len, all_of)), max(sum(b for b, _ in s) for s in all_of)
