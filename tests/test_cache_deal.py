"""The model of the dealing out, against the library's workspace sizes and by its own rule."""
import random

import torch

import cache_deal
import paper_2603_29494_amd as va


def test_workspace_sizes_and_chunk_limits():
    rng = random.Random(1)
    seconds = 0
    for _ in range(3000):
        H, D, bits = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128]), rng.choice([4, 8])
        Hq, n, B = H * rng.choice([1, 4, 7, 33]), rng.choice([1, 1, 2, 5, 40]), rng.randint(1, 300)
        page, cols = rng.choice([32, 64, 1024]), rng.randint(1, 200)
        window, sinks = rng.choice([1, 100, 5000, 1 << 30]), rng.choice([0, 5, 1000])
        d = cache_deal.deal(B, Hq, H, n, D, cols, page, window, sinks)
        q = torch.empty(B, Hq, n, D, dtype=torch.bfloat16, device="meta")
        size = va.cache_bytes(4, H, D, page, bits)
        c = va.Cache(torch.empty(size, dtype=torch.uint8, device="meta"), 4, H, D, page, bits)
        assert va.cache_attn_workspace_bytes(q, c, cols, window, sinks) == d.workspace
        if not d.merge:
            continue
        top = rng.randint(1, cols * page)
        lens = [rng.randint(0, top) for _ in range(B)]
        seen = cache_deal.blocks_seen(d, lens, n, Hq // H, cols, page, window, sinks)
        _, second, counts = cache_deal.chunks(d, H, seen)
        assert len(seen) == d.units and sum(counts) * H <= d.items
        seconds += second
    assert seconds > 20
