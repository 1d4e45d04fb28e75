"""Attention of a tree of drafted tokens against a plain 64-bit form, and the accepted path's move, exactly."""
import numpy as np
import pytest
import torch

import paper_2502_15294_amd as ra
from token_reference import TORCH, Cache, context, logit_error, scale_of, selection, softmax_rows, unit_roundoff_sum

pytestmark = pytest.mark.gpu

LENS = {
    "one_round": [[40]],
    "edges": [[1, 15, 16, 17, 31, 32, 33, 0, 64], [0, 0], [5], [], [300, 2, 129]],
    "longer": [[900, 3, 700], [1025, 640, 33, 16, 1], [48]],
    "many_sequences": [[(7 * b) % 50, 3] for b in range(70)],
    "many_rounds": [[(5 * r) % 9 for r in range(330)], [4] * 500],
}


def tree_mask(rng, B, n, kind):
    if kind == "tree":
        parents = [[int(rng.integers(max(-1, i - 6), i)) if i else -1 for i in range(n)] for _ in range(B)]
        return ra.make_tree_mask(parents).numpy()
    m = rng.random((B, n, (n + 31) // 32 * 32)) < 0.3
    m[:, :, n:] = True  # bits of nodes that are not there
    m[:, n // 2, :n] = False
    return np.packbits(m, axis=2, bitorder="little").view(np.uint32).view(np.int32).copy()


def run_tree(lens, Hkv, G, d, dtype, n, cap, paged, kind="tree", seed=0, select=True, with_len=True, empty_cur=False):
    rng = np.random.default_rng(seed)
    cache = Cache(lens, Hkv, d, dtype, paged, seed=seed)
    B, Hq = cache.B, Hkv * G
    sel = None
    if select:
        sel = [sorted(rng.choice(m, size=(m + 1) // 2, replace=False).tolist()) if m else [] for m in cache.n]
        sel[0] = sel[0] + [cache.n[0], -1] if len(sel[0]) + 2 <= cache.R else sel[0]  # entries that are no rounds
    q = cache.draw(rng, (B, n, Hq, d))
    ck, cv = cache.draw(rng, (B, cap, Hkv, d)), cache.draw(rng, (B, cap, Hkv, d))
    cur_len = np.zeros(B, dtype=np.int32) if empty_cur else rng.integers(0, cap - n + 1, size=B).astype(np.int32)
    tree_len = rng.integers(0, n + 1, size=B).astype(np.int32) if with_len else np.full(B, n, dtype=np.int32)
    if with_len:
        tree_len[-1] = n
    for b in range(B):  # nothing there is used
        ck[b, cur_len[b] + tree_len[b]:] = cv[b, cur_len[b] + tree_len[b]:] = np.nan
        q[b, tree_len[b]:] = np.nan
    mask = tree_mask(rng, B, n, kind)
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[dtype]).cuda()  # noqa: E731
    ints = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    ctx, ws = context(cache, Hq, n, cap)
    si, ns = selection(cache, sel) if select else (None, None)
    call = lambda: ra.ra_round_sparse_attn_tree(ctx, up(q), cache.view, ints(mask), up(ck), up(cv), ints(cur_len),  # noqa: E731
                                                tree_len=ints(tree_len) if with_len else None, sel_idx=si, n_sel=ns)
    out, lse = call()
    again, lse_again = call()
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(lse, lse_again)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    bits = np.unpackbits(mask.view(np.uint8).reshape(B, n, -1), axis=2, bitorder="little")[:, :, :n].astype(bool)
    for b in range(B):
        c, m = int(cur_len[b]), int(tree_len[b])
        assert np.all(out[b, m:] == 0) and np.all(lse[b, m:] == -np.inf)
        if m == 0:
            continue
        hk, hv = cache.history(b, sel)
        k = np.concatenate([hk, ck[b, :c + m].transpose(1, 0, 2)], 1)
        v = np.concatenate([hv, cv[b, :c + m].transpose(1, 0, 2)], 1)
        T = k.shape[1]
        sees = np.ones((m, T), dtype=bool)
        sees[:, T - m:] = bits[b, :m, :m]
        # bf16: a weight goes to the matrix cores as three bf16 numbers, which hold all of its bits: 3 T products are added up in
        # fp32, T weights, and what is merged
        rounding = 4 * unit_roundoff_sum(T + 64)
        for h in range(Hq):
            g = h // G
            s = np.where(sees, q[b, :m, h] @ k[g].T * scale_of(d), -np.inf)
            p, ref_lse = softmax_rows(s)
            off = logit_error(q[b, :m, h], k[g], scale_of(d)) + 2.0 ** -22 * (1 + np.abs(np.where(sees, s, 0)).max(initial=0))
            bound = (rounding + 2 * off) * (p @ np.abs(v[g])) + 1e-30
            assert np.all(np.abs(out[b, :m, h] - p @ v[g]) <= bound), (b, h, np.abs(out[b, :m, h] - p @ v[g]).max())
            seen = np.isfinite(ref_lse)
            assert np.all(lse[b, :m, h][~seen] == -np.inf) and np.all(out[b, :m, h][~seen] == 0)
            tol = off + unit_roundoff_sum(T + 64) + 2.0 ** -22 * np.abs(ref_lse[seen])
            assert np.all(np.abs(lse[b, :m, h][seen] - ref_lse[seen]) <= tol), (b, h)
    ra.ra_destroy(ctx)


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("dtype,Hkv,G,d", [("bf16", 2, 4, 128), ("bf16", 2, 2, 64), ("f32", 2, 4, 64), ("f32", 1, 2, 128), ("bf16", 8, 1, 128)])
@pytest.mark.parametrize("n,cap", [(1, 1), (7, 40), (33, 100)])
def test_tree(dtype, Hkv, G, d, n, cap, paged):
    run_tree(LENS["edges"], Hkv, G, d, dtype, n, cap, paged, seed=n + d)


@pytest.mark.parametrize("n,cap", [(2, 300), (31, 64), (32, 33), (64, 200), (65, 70), (100, 129)])
@pytest.mark.parametrize("dtype,Hkv,G,d", [("bf16", 2, 8, 128), ("bf16", 1, 3, 128), ("bf16", 2, 4, 64), ("f32", 2, 1, 64)])
def test_sizes(dtype, Hkv, G, d, n, cap):
    run_tree(LENS["longer"], Hkv, G, d, dtype, n, cap, paged=n % 2 == 1, seed=n, select=n != 64)


@pytest.mark.parametrize("lens", ["many_sequences", "many_rounds", "one_round"])
@pytest.mark.parametrize("dtype,G,d,n", [("bf16", 4, 128, 3), ("bf16", 4, 128, 5), ("bf16", 4, 128, 40), ("bf16", 2, 64, 20), ("f32", 2, 64, 9)])
def test_batches(lens, dtype, G, d, n):
    run_tree(LENS[lens], 2, G, d, dtype, n, n + 30, paged=G == 4, seed=3, select=lens != "one_round")


@pytest.mark.parametrize("dtype,G,d,n", [("bf16", 4, 128, 6), ("bf16", 4, 128, 50), ("bf16", 4, 64, 50), ("f32", 4, 128, 50)])
@pytest.mark.parametrize("empty_cur", [False, True])
def test_any_relation_and_nodes_that_see_nothing(dtype, G, d, n, empty_cur):
    run_tree([[0, 0], [3, 40], [], [100]], 2, G, d, dtype, n, n + 45, paged=False, kind="random", seed=5, empty_cur=empty_cur, with_len=empty_cur)


@pytest.mark.parametrize("n", [8, 48])
def test_a_chain_is_a_question(n):
    """A tree that is a chain: bit for bit the causal attention of the question call where both have the same cut, and within the
    tests' bound anyway."""
    rng = np.random.default_rng(1)
    cache = Cache([[200, 33, 500]], 2, 128, "bf16", False)
    q, ck, cv = (torch.from_numpy(cache.draw(rng, s)).bfloat16().cuda() for s in ((1, n, 8, 128), (1, n + 20, 2, 128), (1, n + 20, 2, 128)))
    ctx, ws = context(cache, 8, n, n + 20)
    mask = ra.make_tree_mask([list(range(-1, n - 1))]).cuda()
    out, lse = ra.ra_round_sparse_attn_tree(ctx, q, cache.view, mask, ck, cv, torch.tensor([20], dtype=torch.int32, device="cuda"))
    ref, ref_lse = ra.ra_round_sparse_attn_prefill(ctx, q, cache.view, cur_k=ck, cur_v=cv)
    assert (out - ref).abs().max().item() <= 2.0 ** -13 * cv.float().abs().max().item() and (lse - ref_lse).abs().max().item() <= 1e-5
    ra.ra_destroy(ctx)


def test_no_history_at_all():
    """R_max = 0: the current round and the tree alone."""
    n, cap = 5, 20
    empty = torch.zeros((1, 0), dtype=torch.int32, device="cuda")
    view = ra.KVView(torch.zeros(8, device="cuda", dtype=torch.bfloat16), torch.zeros(8, device="cuda", dtype=torch.bfloat16),
                     empty.long(), empty, torch.zeros(1, dtype=torch.int32, device="cuda"), 1, 128, 0)
    gen = torch.Generator("cuda").manual_seed(0)
    q, k, v = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((1, n, 2, 128), (1, cap, 1, 128), (1, cap, 1, 128)))
    ctx = ra.ra_create(0)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    ra.ra_set_workspace(ctx, ws)
    mask = ra.make_tree_mask([[-1, 0, 0, 1, 2]])
    out, lse = ra.ra_round_sparse_attn_tree(ctx, q, view, mask.cuda(), k, v, torch.tensor([9], dtype=torch.int32, device="cuda"))
    sees = torch.ones((n, 14), dtype=torch.bool)
    sees[:, 9:] = (mask[0, :, :1] >> torch.arange(n) & 1).bool()
    s = q[0].double().cpu().transpose(0, 1) @ k[0, :14, 0].double().cpu().T * scale_of(128)
    p = s.masked_fill(~sees, -np.inf).softmax(-1)
    ref = (p @ v[0, :14, 0].double().cpu()).transpose(0, 1)
    assert (out[0].double().cpu() - ref).abs().max().item() < 2.0 ** -13 * 4
    ra.ra_destroy(ctx)


def test_lengths_out_of_range_are_clamped():
    """cur_len and tree_len beyond the buffers: what does not fit is not there."""
    rng = np.random.default_rng(2)
    for dtype, d, n in (("bf16", 128, 4), ("bf16", 128, 40), ("f32", 64, 4)):
        cache = Cache([[20], [20], [20]], 1, d, dtype, False)
        cap = n + 6
        q, ck, cv = (torch.from_numpy(cache.draw(rng, s)).to(TORCH[dtype]).cuda() for s in ((3, n, 4, d), (3, cap, 1, d), (3, cap, 1, d)))
        ctx, ws = context(cache, 4, n, cap)
        mask = ra.make_tree_mask([list(range(-1, n - 1))] * 3).cuda()
        ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        out, _ = ra.ra_round_sparse_attn_tree(ctx, q, cache.view, mask, ck, cv, ints(-5, 8, cap + 9), tree_len=ints(n + 7, n, -3))
        ref, _ = ra.ra_round_sparse_attn_tree(ctx, q, cache.view, mask, ck, cv, ints(0, 8, cap), tree_len=ints(n, cap - 8, 0))
        assert torch.equal(out, ref) and out[2].abs().max().item() == 0
        ra.ra_destroy(ctx)


def test_tokens_far_into_a_long_round():
    """One round of 70 000 tokens, more units than a workgroup looks up at a time."""
    run_tree([[70000], [9]], 1, 4, 128, "bf16", 5, 20, paged=True, seed=8, select=False)
    run_tree([[40000, 3] + [1] * 700] * 2, 1, 8, 128, "bf16", 9, 20, paged=False, seed=9, select=False)


# ---- the accepted path -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layers,B,cap,Hkv,d,max_path", [(1, 1, 1, 1, 64, 1), (3, 5, 40, 2, 128, 12), (33, 3, 150, 8, 128, 100), (2, 2, 30, 40, 128, 9)])
def test_commit(dtype, layers, B, cap, Hkv, d, max_path):
    rng = np.random.default_rng(layers)
    ks, vs = ([torch.randn((B, cap, Hkv, d), device="cuda").to(TORCH[dtype]) for _ in range(layers)] for _ in range(2))
    cur_len = rng.integers(0, max(1, cap // 3), size=B).astype(np.int32)
    path = np.full((B, max_path), -1, dtype=np.int32)
    n_path = np.zeros(B, dtype=np.int32)
    for b in range(B):
        room = min(cap - cur_len[b], max_path)
        m = int(rng.integers(0, room + 1)) if b else min(room, max_path)
        path[b, :m] = np.sort(rng.choice(cap - cur_len[b], size=m, replace=False))
        n_path[b] = m
    old = [t.clone() for t in (*ks, *vs)]
    ctx = ra.ra_create(0)
    ints = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    new_len = ra.ra_tree_commit(ctx, ks, vs, ints(cur_len), ints(path), ints(n_path))
    assert new_len.cpu().tolist() == (cur_len + n_path).tolist()
    for new, was in zip((*ks, *vs), old):
        want = was.clone()
        for b in range(B):
            c, m = int(cur_len[b]), int(n_path[b])
            want[b, c:c + m] = was[b, c + torch.from_numpy(path[b, :m]).long().cuda()]
        assert torch.equal(new, want)
    ra.ra_destroy(ctx)


def test_a_path_ends_at_an_entry_that_is_none():
    k, v = torch.randn((4, 12, 1, 64), device="cuda"), torch.randn((4, 12, 1, 64), device="cuda")
    was = k.clone()
    ctx = ra.ra_create(0)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    # smaller than its place; outside the buffer; the same node twice (taken twice); n_path beyond the list, cur_len at the end
    new_len = ra.ra_tree_commit(ctx, [k], [v], ints([2, 4, 0, 12]), ints([[1, 3, 1, 5], [0, 8, 3, 3], [2, 2, 5, 5], [0, 1, 2, 3]]),
                                ints([4, 4, 9, 4]))
    assert new_len.tolist() == [4, 5, 4, 12]
    want = was.clone()
    want[0, 2:4] = was[0, [3, 5]]
    want[2, :4] = was[2, [2, 2, 5, 5]]
    assert torch.equal(k, want)
    ra.ra_destroy(ctx)
