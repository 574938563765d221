"""How much work a call of pp_paged_attention has, counted as its kernels cut it."""


def _tiles(fresh, cached, group, kv_heads, window, rows_of_item):
    total = 0
    for f, c in zip(fresh, cached):
        n, rows = f + c, f * group
        for r0 in range(0, rows, rows_of_item):
            first, last = (n - f + r // group for r in (r0, min(r0 + rows_of_item, rows) - 1))
            lo = max(0, max(first, 0) - window + 1) if window else 0
            total += 1 if last < lo else last // 128 - lo // 128 + 1
    return total * kv_heads


def chunk_tiles(fresh, cached, group, kv_heads, window=0):
    """Tiles of 128 keys of the items (256 rows) of the chunk kernel."""
    return _tiles(fresh, cached, group, kv_heads, window, 256)


def token_tiles(fresh, cached, group, kv_heads, window=0):
    """The same of the kernel of single tokens (16 rows)."""
    return _tiles(fresh, cached, group, kv_heads, window, 16)
