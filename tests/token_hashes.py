"""Run the calls on drafted tokens and on single tokens on small fixed inputs and print one JSON object of output hashes.

Helper of test_gpu_token_programs.py, run as a script of its own so that the library named by RA_LIBRARY is the one loaded."""
import hashlib
import json
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import paper_2502_15294_amd as ra  # noqa: E402
from token_reference import TORCH, Cache, context, selection  # noqa: E402

LENS = [[300, 17, 0, 640, 33], [5], [64, 64, 900]]
# (type, KV heads, group, channels, nodes, paged): every kernel a tree can go to
TREES = [("bf16", 2, 4, 128, 3, False), ("bf16", 2, 4, 128, 7, True), ("bf16", 2, 4, 128, 40, False), ("bf16", 2, 8, 128, 40, True),
         ("bf16", 2, 4, 64, 20, False), ("f32", 2, 4, 64, 9, True), ("f32", 1, 4, 128, 33, False)]


def digest(*tensors):
    torch.cuda.synchronize()
    h = hashlib.sha1()
    for t in tensors:
        h.update(np.ascontiguousarray(t.float().cpu().numpy()).tobytes())
    return h.hexdigest()[:16]


def main():
    res = {}

    def record(tag, fn):
        torch.randn(1 << 22, device="cuda").sum().item()
        first = digest(*fn())
        second = digest(*fn())
        res[tag] = first if first == second else [first, second]

    for many in (False, True):
        for dtype, Hkv, G, d, n, paged in TREES:
            lens = LENS + [[7, 3] for _ in range(66)] if many else LENS
            rng = np.random.default_rng(n)
            cache = Cache(lens, Hkv, d, dtype, paged)
            B, Hq = cache.B, Hkv * G
            up = lambda x: torch.from_numpy(x).to(TORCH[dtype]).cuda()  # noqa: E731
            q, k, v = up(cache.draw(rng, (B, n, Hq, d))), up(cache.draw(rng, (B, n + 50, Hkv, d))), up(cache.draw(rng, (B, n + 50, Hkv, d)))
            mask = ra.make_tree_mask([[max(-1, i - 1 - i % 3) for i in range(n)]] * B).cuda()
            cur_len = torch.arange(B, dtype=torch.int32, device="cuda") % 50
            si, ns = selection(cache, [list(range(0, m, 2)) for m in cache.n])
            ctx, ws = context(cache, Hq, n, n + 50)
            tag = f"{dtype}_{Hkv}_{G}_{d}_{n}_{paged}_{many}"
            record("tree_" + tag, lambda: ra.ra_round_sparse_attn_tree(ctx, q, cache.view, mask, k, v, cur_len, sel_idx=si, n_sel=ns))
            _, lse = ra.ra_round_sparse_attn_tree(ctx, q, cache.view, mask, k, v, cur_len, sel_idx=si, n_sel=ns)
            record("weights_" + tag, lambda: [ra.ra_token_weights(ctx, q, cache.view, lse, sel_idx=si, n_sel=ns)])
            w = ra.ra_token_weights(ctx, q, cache.view, lse, sel_idx=si, n_sel=ns)
            record("select_" + tag, lambda: ra.ra_select_tokens(ctx, w, cache.seg_len, cache.n_rounds, 200, 4, 30))
            ra.ra_destroy(ctx)
    ctx = ra.ra_create(0)
    w = torch.randn((3, 200000), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    lens = torch.full((3, 500), 390, dtype=torch.int32, device="cuda")
    n = torch.full((3,), 500, dtype=torch.int32, device="cuda")
    record("select_long", lambda: ra.ra_select_tokens(ctx, w, lens, n, 50000, 4, 30))
    print("HASHES " + json.dumps(res))


if __name__ == "__main__":
    main()
