"""A resumed request, from its checkpoint to the next tokens, over one layer.

1. The suffix's reusable blocks are restored from their checkpoint into 16-bit pages.
2. The rows that are not in it (the prefix and the repaired blocks) are
   written into the pages as a model's projections deliver them, and the repaired
   rows, scattered over the context, attend over the pages.
3. The whole context moves into a cache that stays in 4 bits: read back, appended.
4. Tokens are decoded over both caches, each step a row appended and attended,
   the 4-bit step also replayed from a HIP graph with a sliding window and sinks.

Keys, values and queries are drawn, since there is no model: what it prints is how
far the 4-bit cache's attention is from the 16-bit one's.

    python examples/resume_and_decode.py [tiny|llama8b_1l] [decode steps]
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_26219_amd import serving  # noqa: E402
from paper_2609_26219_amd import workloads as wl  # noqa: E402
from paper_2609_26219_amd.device import DeviceRestore  # noqa: E402


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def run(name: str = "llama8b_1l", steps: int = 16, group: int = 4, window: int = 256, sinks: int = 4) -> dict:
    case = wl.make_case(name)
    shape, request = case.shape, case.requests[0]
    H, D, P, B = shape.num_kv_heads, shape.head_dim, shape.page_size, shape.block_tokens
    dtype = torch.bfloat16 if shape.out_dtype == wl.OUT_BF16 else torch.float16
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda n, heads: torch.randn((n, heads, D), generator=gen, device="cuda").to(dtype)  # noqa: E731

    # 1. Restore.
    restored = DeviceRestore(case, workers=1)
    restored.run()
    pages = serving.PagedCache(H, D, P, dtype, wl.TAG_FP16, k_cache=restored.k_cache, v_cache=restored.v_cache)
    context = request.dst_row0 + request.suffix_tokens
    width = -(-(context + steps) // P)
    table = np.full(width, -1, np.int32)
    table[:min(width, len(request.page_table))] = request.page_table[:width]
    # pages of the context's other rows: any that the request does not use
    free = iter(np.setdiff1d(np.arange(shape.pool_pages), request.page_table))
    table = np.array([p if p >= 0 else next(free) for p in table], np.int32)
    table = torch.from_numpy(table).cuda()[None]

    # 2. The rows outside the checkpoint, and attention of the repaired ones.
    suffix = torch.arange(request.dst_row0, context, dtype=torch.int32, device="cuda")
    repaired = suffix[torch.from_numpy(np.repeat(request.repair != 0, B)[:request.suffix_tokens]).cuda()]
    missing = torch.cat([torch.arange(request.dst_row0, dtype=torch.int32, device="cuda"), repaired])
    n = missing.numel()
    serving.append(pages, serving.Batch(_ints([0, n]), _ints([context]), table, n, positions=missing), draw(n, H), draw(n, H))
    n = repaired.numel()
    rows = serving.Batch(_ints([0, n]), _ints([context]), table, n, positions=repaired, max_kv_len=context)
    hidden, lse = serving.attention(pages, rows, draw(n, H * group), return_lse=True)

    # 3. Into 4 bits, on pages of its own.
    small = serving.PagedCache(H, D, P, dtype, wl.TAG_K4V4, pool_pages=width)
    own = torch.arange(width, dtype=torch.int32, device="cuda").flip(0).contiguous()[None]
    kv_len = _ints([context])
    whole = lambda t: serving.Batch(_ints([0, context]), kv_len, t, context)  # noqa: E731
    serving.append(small, whole(own), *serving.read(pages, whole(table)))

    # 4. Decode: the same buffers every step, their contents changed in place.
    step = {c: serving.Batch(_ints([0, 1]), kv_len, t, 1, max_tokens=1, max_kv_len=context + steps)
            for c, t in ((pages, table), (small, own))}
    q, k, v = draw(1, H * group), draw(1, H), draw(1, H)

    def decode(cache, out, **mask):
        serving.append(cache, step[cache], k, v)
        return serving.attention(cache, step[cache], q, out=out, **mask)

    out = {c: torch.empty_like(q) for c in step}
    windowed = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (a first call outside the capture, which loads the kernels)
        serving.attention(small, step[small], q, out=windowed, window=window, sinks=sinks)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode(small, windowed, window=window, sinks=sinks)
    worst, replays_agree = 0.0, True
    for _ in range(steps):
        kv_len += 1
        for t, heads in ((q, H * group), (k, H), (v, H)):
            t.copy_(draw(1, heads))
        exact, coarse = decode(pages, out[pages]), decode(small, out[small])
        worst = max(worst, float((exact.float() - coarse.float()).abs().max()))
        graph.replay()
        eager = serving.attention(small, step[small], q, window=window, sinks=sinks)
        replays_agree &= torch.equal(windowed, eager)
    return {"context": context, "repaired_rows": n, "repaired_finite": bool(torch.isfinite(hidden).all() and
                                                                             torch.isfinite(lse).all()),
            "bytes_16bit": (context + steps) * 4 * H * D, "bytes_4bit": (context + steps) * H * (D + 8),
            "decoded": steps, "replays_agree": replays_agree, "worst_difference": worst}


if __name__ == "__main__":
    print(run(*sys.argv[1:2], *(int(a) for a in sys.argv[2:3])))
