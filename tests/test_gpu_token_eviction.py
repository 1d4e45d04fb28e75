"""Token weights against a plain 64-bit form; the tokens to keep and the smaller cache exactly; and all of it as one
program."""
import numpy as np
import pytest
import torch

import paper_2502_15294_amd as ra
from token_reference import TORCH, Cache, context, logit_error, scale_of, selection, softmax_rows, unit_roundoff_sum

pytestmark = pytest.mark.gpu

EDGES = [[1, 15, 16, 17, 31, 32, 33, 0, 64], [0, 0], [5], [], [300, 2, 129]]


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


# ---- weights -----------------------------------------------------------------------------------------------------------
def run_weights(lens, Hkv, G, d, dtype, q_len, paged, select, with_prev, seed=0, n_pos=None, in_place=False, twice=False):
    rng = np.random.default_rng(seed)
    cache = Cache(lens, Hkv, d, dtype, paged, seed=seed, values=False)
    B, Hq = cache.B, Hkv * G
    sel = None
    if select:
        sel = [sorted(rng.choice(m, size=(m + 1) // 2, replace=False).tolist()) if m else [] for m in cache.n]
        if twice:
            sel = [s[:-1] + s[:1] if len(s) > 1 else s for s in sel]
    q = cache.draw(rng, (B, q_len, Hq, d))
    total = int(cache.lens.sum(1).max())
    n_pos = n_pos or total + 5
    lse = np.empty((B, q_len, Hq))
    for b in range(B):
        k, _ = cache.history(b, sel)
        for h in range(Hq):
            lse[b, :, h] = softmax_rows(q[b, :, h] @ k[h // G].T * scale_of(d))[1]
    lse = np.where(np.isfinite(lse), lse + rng.random(lse.shape), lse)  # (some of the weight went to the current round)
    if q_len > 2:  # rows that add nothing, whatever they hold
        lse[:, 1, 0], lse[:, 2, Hq - 1], lse[:, 0, Hq // 2] = np.inf, np.nan, -np.inf
        q[:, 1, 0] = q[:, 2, Hq - 1] = np.nan
        q[:, 0, Hq // 2] = np.inf
    lse = lse.astype(np.float32).astype(np.float64)
    prev = rng.random((B, n_pos)).astype(np.float32) if with_prev else np.zeros((B, n_pos), dtype=np.float32)
    ctx = ra.ra_create(0)
    si, ns = selection(cache, sel) if select else (None, None)
    dq, dl = torch.from_numpy(q).to(TORCH[dtype]).cuda(), torch.from_numpy(lse).float().cuda()
    dp = torch.from_numpy(prev).cuda() if with_prev else None
    got = ra.ra_token_weights(ctx, dq, cache.view, dl, prev=dp, n_pos=n_pos, sel_idx=si, n_sel=ns)
    again = ra.ra_token_weights(ctx, dq, cache.view, dl, prev=dp, n_pos=n_pos, sel_idx=si, n_sel=ns,
                                weights=dp if in_place else None)
    assert torch.equal(got, again) and (not in_place or again is dp)
    got = got.double().cpu().numpy()
    for b in range(B):
        want, off = prev[b].astype(np.float64), 0.0
        first = np.cumsum(cache.lens[b]) - cache.lens[b]
        add = np.zeros(max(n_pos, total) + 1)
        for r in range(cache.n[b]) if sel is None else sel[b]:
            k = cache.k[b][r]
            for h in range(Hq):
                rows = np.isfinite(lse[b, :, h])
                s = q[b, rows, h] @ k[h // G].T * scale_of(d)
                add[first[r]:first[r] + k.shape[1]] += np.exp(s - lse[b, rows, h, None]).sum(0)
                off = max(off, logit_error(q[b, rows, h], k[h // G], scale_of(d)) + 2.0 ** -22 * (1 + np.abs(s).max(initial=0) + np.abs(lse[b, rows, h]).max(initial=0)))
        bound = add[:n_pos] * (2 * off + unit_roundoff_sum(q_len * Hq + 8)) + 2.0 ** -23 * (want + add[:n_pos])
        assert np.all(np.abs(got[b] - want - add[:n_pos]) <= bound), (b, np.abs(got[b] - want - add[:n_pos]).max())
        assert np.array_equal(got[b][add[:n_pos] == 0], want[add[:n_pos] == 0])
    ra.ra_destroy(ctx)


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("dtype,Hkv,G,d", [("bf16", 2, 4, 128), ("bf16", 8, 1, 64), ("f32", 3, 2, 64), ("f32", 1, 16, 128), ("bf16", 5, 3, 128)])
@pytest.mark.parametrize("q_len", [1, 5, 40])
def test_weights(dtype, Hkv, G, d, q_len, paged):
    run_weights(EDGES, Hkv, G, d, dtype, q_len, paged, select=q_len != 5, with_prev=q_len != 1, seed=q_len)


@pytest.mark.parametrize("dtype,Hkv,G,d,q_len", [("bf16", 2, 8, 128, 129), ("bf16", 2, 4, 128, 128), ("f32", 2, 1, 128, 600), ("bf16", 8, 8, 128, 1)])
def test_weights_of_long_rounds(dtype, Hkv, G, d, q_len):
    run_weights([[1000, 257, 256, 255], [2100], [31, 33] * 6], Hkv, G, d, dtype, q_len, paged=q_len == 128, select=q_len == 1, with_prev=True)


def test_weights_of_many_sequences_and_rounds():
    run_weights([[(3 * b) % 40, 7, (5 * b) % 70] for b in range(90)], 2, 4, 128, "bf16", 2, True, True, True)
    run_weights([[(5 * r) % 9 for r in range(700)], [4] * 1000], 1, 4, 64, "bf16", 3, False, True, True)


def test_weights_cut_off_in_place_and_named_twice():
    run_weights(EDGES, 2, 2, 64, "f32", 4, False, False, True, n_pos=100)
    run_weights(EDGES, 2, 2, 128, "bf16", 4, True, True, True, in_place=True)
    run_weights(EDGES, 2, 2, 128, "bf16", 1, False, True, False, twice=True)


def test_weights_of_the_decode_call_add_up_to_its_heads():
    """Every head's weights over the history and the current round add up to one."""
    cache = Cache([[200, 33, 500], [64]], 2, 128, "bf16", True)
    gen = torch.Generator("cuda").manual_seed(0)
    q = torch.randn((2, 8, 128), generator=gen, device="cuda").bfloat16()
    ctx, ws = context(cache, 8, 1)
    _, lse = ra.ra_round_sparse_attn_decode(ctx, q, cache.view)
    w = ra.ra_token_weights(ctx, q, cache.view, lse)
    assert w.shape == (2, 733) and (w.double().sum(1) - 8).abs().max().item() < 1e-3
    ra.ra_destroy(ctx)


# ---- the tokens to keep --------------------------------------------------------------------------------------------------
def keep(w, lens, budget, first, last, unit, base):
    n = min(int(lens.sum()), len(w))
    f = min(first, n)
    l = min(last, n - f)
    forced = list(range(f)) + list(range(n - l, n))
    w = w + 0.0  # (one zero)
    rest = sorted(range(f, n - l), key=lambda p: (-w[p], p))
    kept = np.sort(np.array(forced + rest[:max(0, min(budget, n) - len(forced))], dtype=np.int64))
    ends = np.minimum(np.cumsum(lens), len(w))
    starts = np.minimum(np.cumsum(lens) - lens, len(w))
    kept_len = np.searchsorted(kept, ends) - np.searchsorted(kept, starts)
    blocks = (kept_len + 15) // 16
    return kept, kept_len, base + (np.cumsum(blocks) - blocks) * unit


def check_selection(w, lens, n_rounds, budget, first=0, last=0, block_size=0, stride=0):
    ctx = ra.ra_create(0)
    idx, n, kept_len, off, left = (x.cpu().numpy() for x in ra.ra_select_tokens(
        ctx, torch.from_numpy(w).cuda(), ints(lens), ints(n_rounds), budget, first, last, block_size, stride))
    for b in range(len(w)):
        l = lens[b] * (np.arange(lens.shape[1]) < n_rounds[b])
        kept, kl, ko = keep(w[b], l, budget, first, last, 1 if block_size else 16, b * stride)
        assert n[b] == len(kept) and idx[b, :n[b]].tolist() == kept.tolist() and np.all(idx[b, n[b]:] == -1)
        assert kept_len[b].tolist() == kl.tolist() and off[b].tolist() == ko.tolist()
        assert np.array_equal(left[b, :n[b]], w[b, kept]) and np.all(left[b, n[b]:] == 0)
    ra.ra_destroy(ctx)


WEIGHTS = {
    "spread": lambda rng, s: rng.lognormal(0, 3, s),
    "ties": lambda rng, s: rng.integers(0, 4, s) * 0.25,
    "equal": lambda rng, s: np.full(s, 0.5),
    "close": lambda rng, s: (np.float32(1.0).view(np.int32) + rng.integers(0, 3000, s).astype(np.int32)).view(np.float32),
    "signs": lambda rng, s: rng.standard_normal(s) * (rng.random(s) < 0.7),
    "extremes": lambda rng, s: rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, 3.4e38, 1e-45, -1e-45]), size=s),
}


@pytest.mark.parametrize("kind", list(WEIGHTS))
@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (40, 0, 0), (100, 7, 13), (333, 0, 64), (64, 64, 0), (2000, 4, 4)])
def test_selection(kind, budget, first, last):
    rng = np.random.default_rng(budget)
    lens = np.array([[100, 0, 200, 33], [1, 0, 0, 0], [0, 0, 0, 0], [64, 64, 64, 64], [500, 17, 90, 100], [5, 6, 7, 999999]], dtype=np.int32)
    n_rounds = np.array([4, 1, 0, 4, 4, 3])
    w = WEIGHTS[kind](rng, (6, 720)).astype(np.float32)
    check_selection(w, lens, n_rounds, budget, first, last, block_size=16 if first else 0, stride=100000)


@pytest.mark.parametrize("n,R,budget", [(1, 1, 1), (64, 2, 63), (1025, 3, 512), (5000, 1000, 1234), (70001, 200, 17500), (131072, 128, 32768)])
def test_selection_sizes(n, R, budget):
    rng = np.random.default_rng(n)
    lens = rng.multinomial(n, np.ones(R) / R, size=3).astype(np.int32)
    w = rng.lognormal(0, 2, (3, n + 3)).astype(np.float32)
    w[1] = np.float32(0.25)
    check_selection(w, lens, np.full(3, R), budget, first=min(16, budget // 4), last=budget // 8)


@pytest.mark.parametrize("kind", list(WEIGHTS) + ["mostly_zero"])
@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (20000, 100, 300), (400, 100, 300), (69999, 0, 0), (90000, 5, 5)])
def test_selection_by_several_workgroups(kind, budget, first, last):
    """From 65536 positions on a sequence is several workgroups': every kind of weights, short and empty sequences among them."""
    rng = np.random.default_rng(budget)
    n_pos = 80000
    lens = np.zeros((4, 150), dtype=np.int32)
    lens[0] = rng.multinomial(70001, np.ones(150) / 150)
    lens[1, :3] = [16384, 1, 16383]  # ends where a workgroup's part does
    lens[2, 140:] = 9999  # more than there are positions
    n_rounds = np.array([150, 3, 150, 0])
    if kind == "mostly_zero":
        w = np.where(rng.random((4, n_pos)) < 0.97, 0.0, rng.random((4, n_pos))).astype(np.float32)
    else:
        w = WEIGHTS[kind](rng, (4, n_pos)).astype(np.float32)
    check_selection(w, lens, n_rounds, budget, first, last, block_size=16 if first else 0, stride=200000)


@pytest.mark.parametrize("B,n_pos", [(32, 70000), (33, 66000), (1, 2_700_000)])
def test_selection_of_large_batches_and_very_long_sequences(B, n_pos):
    """The most sequences of several workgroups each, one more, and parts of which a wave does not hold all weights at once."""
    rng = np.random.default_rng(B)
    lens = rng.multinomial(n_pos - 1000, np.ones(900) / 900, size=B).astype(np.int32)
    w = rng.lognormal(0, 2, (B, n_pos)).astype(np.float32)
    check_selection(w, lens, np.full(B, 900), n_pos // 4, 16, 1000, stride=n_pos)


@pytest.mark.parametrize("n_pos,most", [(9000, 8191), (80000, 70001), (80000, 65536)])
def test_selection_of_many_rounds_that_begin_together(n_pos, most):
    """Hundreds of empty rounds at one position: before, between and behind the others; weights behind the last token are NaN."""
    rng = np.random.default_rng(most)
    lens = np.zeros((3, 1000), dtype=np.int32)
    lens[0, 70:140] = rng.multinomial(most, np.ones(70) / 70)
    lens[1, [0, 1, 500, 999]] = [256, 3, 300, 40]
    lens[2, :500] = 1
    w = rng.lognormal(0, 2, (3, n_pos)).astype(np.float32)
    for b in range(3):
        w[b, lens[b].sum():] = np.nan
    check_selection(w, lens, np.array([1000, 1000, 700]), 4000, 5, 70, stride=100000)


def test_positions_behind_the_weights_are_not_there():
    w = np.linspace(0, 1, 50, dtype=np.float32)[None].repeat(2, 0)
    check_selection(w, np.array([[30, 40, 5], [10, 10, 10]], dtype=np.int32), np.array([3, 3]), 20, 3, 5)


# ---- the smaller cache -----------------------------------------------------------------------------------------------------
def smaller_cache(cache, kept_len, paged, values=True):
    """Storage full of 3s and a view of it for rounds of kept_len tokens."""
    like = Cache.__new__(Cache)
    like.__dict__.update(B=cache.B, R=cache.R, Hkv=cache.Hkv, d=cache.d, dtype=cache.dtype, paged=paged, n=cache.n)
    like.lens = kept_len
    like.place(np.random.default_rng(9))
    nk, nv = like.pool
    like.dk = torch.full((nk * cache.Hkv + 1, cache.d), 3.0, dtype=TORCH[cache.dtype], device="cuda")
    like.dv = torch.full((nv * cache.Hkv * cache.d + 16,), 3.0, dtype=TORCH[cache.dtype], device="cuda") if values else None
    t = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    like.view = ra.KVView(like.dk, like.dv, t(like.off), t(kept_len), cache.n_rounds, cache.Hkv, cache.d, int(kept_len.sum(1).max()),
                          block_table=t(like.table) if paged else None, block_size=16 if paged else 0,
                          seg_off_v=None if paged else t(like.off_v))
    return like


def check_compaction(lens, Hkv, d, dtype, paged, to_paged, share, seed=0, values=True):
    rng = np.random.default_rng(seed)
    cache = Cache(lens, Hkv, d, dtype, paged, seed=seed, values=values)
    most = max(1, int(cache.lens.sum(1).max()))
    idx = np.full((cache.B, most), -1, dtype=np.int32)
    n_kept, kept_len = np.zeros(cache.B, dtype=np.int32), np.zeros_like(cache.lens)
    for b in range(cache.B):
        total = int(cache.lens[b].sum())
        kept = np.flatnonzero(rng.random(total) < share)
        idx[b, :len(kept)], n_kept[b] = kept, len(kept)
        ends = np.cumsum(cache.lens[b])
        kept_len[b] = np.searchsorted(kept, ends) - np.searchsorted(kept, ends - cache.lens[b])
    small = smaller_cache(cache, kept_len, to_paged, values)
    ctx = ra.ra_create(0)
    ra.ra_compact_rounds(ctx, cache.view, ints(idx), ints(n_kept), small.view)
    k = np.full(small.dk.shape, 3.0)
    v = np.full(small.dv.shape, 3.0) if values else None
    for b in range(cache.B):
        ends = np.cumsum(cache.lens[b])
        for r in range(cache.n[b]):
            mine = idx[b, :n_kept[b]]
            t = mine[(mine >= ends[r] - cache.lens[b, r]) & (mine < ends[r])] - (ends[r] - cache.lens[b, r])
            rows, elems, pad = small.where(b, r)
            k[rows] = cache.k[b][r][:, t]
            if values:
                v[elems], v[pad] = cache.v[b][r][:, t], 0.0
    assert np.array_equal(small.dk.double().cpu().numpy(), k)
    assert not values or np.array_equal(small.dv.double().cpu().numpy(), v)
    ra.ra_destroy(ctx)


@pytest.mark.parametrize("dtype,Hkv,d", [("bf16", 2, 128), ("bf16", 5, 64), ("f32", 3, 64), ("f32", 8, 128)])
@pytest.mark.parametrize("paged,to_paged", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("share", [1.0, 0.5, 0.05])
def test_compaction(dtype, Hkv, d, paged, to_paged, share):
    check_compaction(EDGES + [[700, 45]], Hkv, d, dtype, paged, to_paged, share)


def test_compaction_of_keys_alone_and_of_many_rounds():
    check_compaction(EDGES, 2, 128, "bf16", True, False, 0.4, values=False)
    check_compaction([[(5 * r) % 9 for r in range(700)], [40] * 30], 2, 64, "bf16", False, True, 0.3)
    check_compaction([[(7 * b) % 90, 50] for b in range(80)], 1, 128, "bf16", False, False, 0.3)


@pytest.mark.parametrize("tokens", [350, 700, 1400])
@pytest.mark.parametrize("dtype,paged,share", [("bf16", False, 0.9), ("f32", True, 0.2)])
def test_compaction_in_pieces_of_every_length(tokens, dtype, paged, share):
    """Six dialogues of 8 heads: pieces of 16, 32 and 64 tokens; rounds that end inside a piece, at its end and behind it."""
    check_compaction([[tokens]] + [[tokens - 64 - 17 * b, 64, 17 * b] for b in range(5)], 8, 64, dtype, paged, not paged, share)


def test_positions_that_are_none_give_zeros():
    cache = Cache([[10, 20]], 2, 64, "f32", False)
    small = smaller_cache(cache, np.array([[3, 2]], dtype=np.int32), False)
    ctx = ra.ra_create(0)
    # the third is no position of round 0, the fourth none at all; n_kept ends before the fifth
    ra.ra_compact_rounds(ctx, cache.view, ints([[1, 4, 25, -7, 12]]), ints([4]), small.view)
    rows0, _, _ = small.where(0, 0)
    rows1, _, _ = small.where(0, 1)
    k = small.dk.double().cpu().numpy()
    assert np.array_equal(k[rows0[:, :2]], cache.k[0][0][:, [1, 4]]) and np.all(k[rows0[:, 2]] == 0) and np.all(k[rows1] == 0)
    ra.ra_destroy(ctx)


# ---- together ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,paged", [("bf16", 128, False), ("bf16", 128, True), ("f32", 64, True)])
def test_a_drafted_step_and_an_eviction(dtype, d, paged):
    """Attend with a tree, commit the accepted path, weigh the tokens by the accepted nodes, evict, and attend again over what
    stayed: the last attention is that of the kept tokens, in 64 bits."""
    rng = np.random.default_rng(4)
    Hkv, G, n, cap, budget = 2, 4, 12, 60, 150
    Hq = Hkv * G
    cache = Cache([[120, 40, 0, 77], [200], [30, 31]], Hkv, d, dtype, paged)
    B = cache.B
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[dtype]).cuda()  # noqa: E731
    q, ck, cv = cache.draw(rng, (B, n, Hq, d)), cache.draw(rng, (B, cap, Hkv, d)), cache.draw(rng, (B, cap, Hkv, d))
    parents = [[-1, -1, 0, 0, 1, 2, 2, 3, 5, 5, 6, 8]] * B
    path = [[0, 2, 5, 8], [1, 4, -1, -1], [-1] * 4]
    cur_len, n_path = ints([20, 3, 0]), ints([4, 2, 0])
    ctx, ws = context(cache, Hq, n, cap)
    dk, dv, dq = up(ck), up(cv), up(q)
    out, lse = ra.ra_round_sparse_attn_tree(ctx, dq, cache.view, ra.make_tree_mask(parents).cuda(), dk, dv, cur_len)
    accepted = torch.zeros((B, n), dtype=torch.bool, device="cuda")
    for b, p in enumerate(path):
        accepted[b, [x for x in p if x >= 0]] = True
    new_len = ra.ra_tree_commit(ctx, [dk], [dv], cur_len, ints(path), n_path)
    w = ra.ra_token_weights(ctx, dq, cache.view, lse.masked_fill(~accepted[..., None], float("inf")))
    w = ra.ra_token_weights(ctx, dq, cache.view, torch.full_like(lse, float("inf")), prev=w, weights=w)  # nothing more
    stride = budget + 15 * cache.R
    idx, n_kept, kept_len, kept_off, left = ra.ra_select_tokens(ctx, w, cache.seg_len, cache.n_rounds, budget, 4, 16, 0, (stride + 15) // 16 * 16)
    assert n_kept.tolist() == [150, 150, 61]
    room = B * ((stride + 15) // 16 * 16)
    k2 = torch.zeros((room * Hkv, d), dtype=dk.dtype, device="cuda")
    v2 = torch.zeros((room * Hkv * d,), dtype=dk.dtype, device="cuda")
    small = ra.KVView(k2, v2, kept_off, kept_len, cache.n_rounds, Hkv, d, budget)
    ra.ra_compact_rounds(ctx, cache.view, idx, n_kept, small)
    q1 = cache.draw(rng, (B, Hq, d))
    got, got_lse = ra.ra_round_sparse_attn_decode(ctx, up(q1), small, cur_k=dk, cur_v=dv, cur_len=new_len)
    w2 = ra.ra_token_weights(ctx, up(q1), small, got_lse, prev=left[:, :budget].contiguous(), n_pos=budget)
    assert torch.all(w2 >= left[:, :budget])
    assert new_len.tolist() == [24, 5, 0]
    got, dk, dv, idx = got.double().cpu().numpy(), dk.double().cpu().numpy(), dv.double().cpu().numpy(), idx.cpu().numpy()
    for b in range(B):
        hk, hv = cache.history(b, None)
        mine, c = idx[b, :int(n_kept[b])], int(new_len[b])
        moved = ck[b].copy()
        for j, p in enumerate(path[b][:int(n_path[b])]):
            moved[int(cur_len[b]) + j] = ck[b, int(cur_len[b]) + p]
        assert np.array_equal(dk[b], moved)
        k = np.concatenate([hk[:, mine], dk[b, :c].transpose(1, 0, 2)], 1)
        v = np.concatenate([hv[:, mine], dv[b, :c].transpose(1, 0, 2)], 1)
        for h in range(Hq):
            s = q1[b, h:h + 1] @ k[h // G].T * scale_of(d)
            p, _ = softmax_rows(s)
            off = logit_error(q1[b, h], k[h // G], scale_of(d)) + 2.0 ** -22 * (1 + np.abs(s).max())
            bound = (2.0 ** -14 + 2 * unit_roundoff_sum(k.shape[1] + 64) + 2 * off) * (p @ np.abs(v[h // G]))
            assert np.all(np.abs(got[b, h] - p @ v[h // G]) <= bound)
    ra.ra_destroy(ctx)
