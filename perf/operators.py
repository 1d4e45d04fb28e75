"""Timed cases of the calls around drafted tokens and token eviction, each beside its plain form.

Operators:
  tree      attention of a tree of drafted tokens over the selected rounds, the answer so far and the drafted tokens
            themselves (`ra_round_sparse_attn_tree`)
  commit    the accepted path of the tree moved to the rows behind the answer, for every layer (`ra_tree_commit`)
  weights   attention weight of every history token added to its running total, from the log-sum-exp that the attention
            returned (`ra_token_weights`)
  evict     the tokens that stay: the heaviest ones beside the first and the last few (`ra_select_tokens`)
  compact   a layer's keys and values of the tokens that stay, as a cache of its own (`ra_compact_rounds`)

Every case is a dialogue batch in the library's layout (include/round_attention.h): `B` sequences of history rounds whose
keys and values are N(0, 1); queries lean towards a common direction and some keys lie in it, so that some tokens are heavy.
With `own` false the operators are computed by elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # True: the library's calls; False: the plain forms

HEAVY = 0.03  # share of the keys that lie in the queries' direction


def listed():
    return [
        # one short fp32 dialogue with two KV heads: a draft of seven tokens, launches and round trips only
        dict(name="tree_tiny", op="tree", dtype="f32", B=1, Hq=4, Hkv=2, d=64, R=8, lo=64, hi=64, paged=False, keep=0.5, cur=24, nodes=7),
        # a small serving batch of an 8B-shaped model, 25 drafted tokens a sequence, the answer well under way
        dict(name="tree_small_batch", op="tree", dtype="bf16", B=8, Hq=32, Hkv=8, d=128, R=20, lo=200, hi=1000, paged=False, keep=0.25, cur=350, nodes=25),
        # a large batch of a 70B-shaped layer slice over paged blocks, 60 drafted tokens: the largest tree
        dict(name="tree_paged_batch", op="tree", dtype="bf16", B=32, Hq=64, Hkv=8, d=128, R=50, lo=300, hi=1000, paged=True, keep=0.14, cur=260, nodes=60),
        # a single sequence's accepted path: launches only
        dict(name="commit_single", op="commit", dtype="bf16", B=1, Hkv=8, d=128, layers=4, cur=120, nodes=25, path=5),
        # 24 layers of a batch
        dict(name="commit_batch", op="commit", dtype="bf16", B=32, Hkv=8, d=128, layers=24, cur=150, nodes=60, path=6),
        # one decode token of one fp32 dialogue
        dict(name="weights_tiny", op="weights", dtype="f32", B=1, Hq=4, Hkv=2, d=64, R=8, lo=64, hi=64, paged=False, keep=1.0, q_len=1),
        # one decode token a sequence of a large paged batch, selected rounds only
        dict(name="weights_paged_decode", op="weights", dtype="bf16", B=64, Hq=64, Hkv=8, d=128, R=50, lo=300, hi=1000, paged=True, keep=0.3, q_len=1),
        # a question of 128 tokens over 32K-token dialogues, every round: the most arithmetic
        dict(name="weights_question", op="weights", dtype="bf16", B=4, Hq=32, Hkv=8, d=128, R=60, lo=80, hi=1012, paged=False, keep=1.0, q_len=128),
        # a small cache of one sequence
        dict(name="evict_single", op="evict", B=1, R=12, lo=200, hi=1000, budget=2048, first=4, last=256, paged=False),
        # long dialogues: 128K tokens down to a quarter
        dict(name="evict_long", op="evict", B=16, R=200, lo=130, hi=1180, budget=32768, first=16, last=1024, paged=True),
        # one layer of one sequence down to 2048 tokens
        dict(name="compact_single", op="compact", dtype="bf16", B=1, Hkv=8, d=128, R=12, lo=200, hi=1000, budget=2048, first=4, last=256, paged=False),
        # one layer of a paged batch, half of the tokens kept
        dict(name="compact_paged_batch", op="compact", dtype="bf16", B=16, Hkv=8, d=128, R=50, lo=300, hi=1000, budget=16000, first=16, last=1024, paged=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("tree", "tree", "weights", "weights", "commit", "evict", "compact"))
    Hkv = rng.choice((2, 4, 8, 8))
    G = rng.choice((1, 2, 4, 4, 8))
    dtype, d = rng.choice((("bf16", 128), ("bf16", 128), ("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)))
    R = log(1, 60)
    lo = log(1, 300)
    hi = lo + log(1, 600)
    mean = (lo + hi) / 2
    paged = rng.random() < 0.5
    if op == "tree":
        nodes, cur, keep = log(1, 96), log(1, 500), rng.choice((1.0, 0.5, 0.25, 0.14))
        tokens = keep * R * mean + cur + nodes
        # the largest listed tree: 32 sequences x 60 nodes x 64 heads x 5000 tokens, in fp32 a twentieth of that
        most = 6e8 if dtype == "bf16" and d == 128 else 3e7
        B = max(1, min(log(1, 64), int(most / (nodes * G * Hkv * tokens))))
        return dict(op=op, dtype=dtype, B=B, Hq=G * Hkv, Hkv=Hkv, d=d, R=R, lo=lo, hi=hi, paged=paged, keep=keep, cur=cur, nodes=nodes)
    if op == "commit":
        nodes = log(2, 96)
        return dict(op=op, dtype=dtype, B=log(1, 32), Hkv=Hkv, d=d, layers=log(1, 24), cur=log(1, 150), nodes=nodes,
                    path=rng.randint(1, max(1, min(8, nodes // 2))))
    if op == "weights":
        q_len, keep = rng.choice((1, 1, log(2, 128))), rng.choice((1.0, 0.5, 0.3))
        tokens = keep * R * mean
        most = 5e8 if dtype == "bf16" and d == 128 else 2e7
        B = max(1, min(log(1, 64), int(most / (q_len * G * Hkv * tokens))))
        return dict(op=op, dtype=dtype, B=B, Hq=G * Hkv, Hkv=Hkv, d=d, R=R, lo=lo, hi=hi, paged=paged, keep=keep, q_len=q_len)
    first, last = rng.choice((0, 4, 16)), rng.choice((0, 1, 100))
    budget = max(first + last, 1, int(rng.choice((0.1, 0.25, 0.5, 0.9, 1.1)) * R * mean))
    if op == "evict":
        return dict(op=op, B=log(1, 64), R=R, lo=lo, hi=hi, budget=budget, first=first, last=last, paged=paged)
    B = max(1, min(log(1, 16), int(16 * 33000 * 8 * 256 / (R * mean * Hkv * d * (2 if dtype == "bf16" else 4)))))
    return dict(op=op, dtype=dtype, B=B, Hkv=Hkv, d=d, R=R, lo=lo, hi=hi, budget=budget, first=first, last=last, paged=paged)


# ---- inputs --------------------------------------------------------------------------------------------------------------
def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


class State:
    pass


def _rounds(case, rng, st):
    """Lengths of the rounds: R in most sequences, fewer in some."""
    B, R = case["B"], case["R"]
    n = np.where(rng.random(B) < 0.7, R, rng.integers(max(1, R - R // 4), R + 1, size=B)).astype(np.int32)
    lens = rng.integers(case["lo"], case["hi"] + 1, size=(B, R)).astype(np.int32)
    lens[np.arange(R)[None] >= n[:, None]] = 0
    st.lens, st.n = lens, n
    st.tokens = R * case["hi"]  # what the sequences have room for
    st.seg_len, st.n_rounds = torch.from_numpy(lens).cuda(), torch.from_numpy(n).cuda()


def _places(lens, paged, rng):
    """Starts of round blocks of these lengths packed one after the other: (seg_off, seg_off_v, block table, pool tokens of
    keys and values)."""
    B, R = lens.shape
    l16 = (lens.astype(np.int64) + 15) // 16 * 16
    if not paged:
        l = lens.astype(np.int64).ravel()
        off = (np.cumsum(l) - l).reshape(B, R)
        off_v = (np.cumsum(l16.ravel()) - l16.ravel()).reshape(B, R)
        return off, off_v, None, int(l.sum()), int(l16.sum())
    slots = l16 // 16
    off = np.cumsum(slots, 1) - slots
    most = max(int(slots.sum(1).max()), 1)
    total = int(slots.sum())
    table = np.full((B, most), 0, dtype=np.int32)
    ids = rng.permutation(total).astype(np.int32)
    at = 0
    for b in range(B):
        k = int(slots[b].sum())
        table[b, :k] = ids[at:at + k]
        at += k
    return off, None, table, total * 16, total * 16


def _cache(case, rng, gen, st, values=True):
    Hkv, d, dt = case["Hkv"], case["d"], _torch_dtype(case)
    off, off_v, table, nk, nv = _places(st.lens, case["paged"], rng)
    st.seg_off = torch.from_numpy(off).cuda()
    st.seg_off_v = None if off_v is None else torch.from_numpy(off_v).cuda()
    st.table = None if table is None else torch.from_numpy(table).cuda()
    st.k = torch.randn((nk * Hkv, d), generator=gen, device="cuda", dtype=dt)
    heavy = torch.randint(0, nk * Hkv, (int(HEAVY * nk * Hkv),), generator=gen, device="cuda")
    st.direction = torch.randn((d,), generator=gen, device="cuda")
    st.direction *= 4 / st.direction.norm()
    st.k[heavy] += (3 * st.direction).to(dt)
    st.v = torch.randn((nv * Hkv * d,), generator=gen, device="cuda", dtype=dt) if values else None
    st.units = int(((st.lens + 15) // 16).sum(1).max())


def _selection(case, rng, st):
    """A share of every sequence's rounds, ascending; none: every round."""
    st.sel = st.n_sel = None
    if case["keep"] < 1.0:
        B, R = case["B"], case["R"]
        sel = np.full((B, R), -1, dtype=np.int32)
        n = np.zeros(B, dtype=np.int32)
        units = 0
        for b in range(B):
            n[b] = max(1, round(case["keep"] * st.n[b]))
            sel[b, :n[b]] = np.sort(rng.choice(st.n[b], size=n[b], replace=False))
            units = max(units, int(((st.lens[b, sel[b, :n[b]]] + 15) // 16).sum()))
        st.sel, st.n_sel = torch.from_numpy(sel).cuda(), torch.from_numpy(n).cuda()
        st.units = units


def _queries(case, n, gen, st):
    q = torch.randn((case["B"], n, case["Hq"], case["d"]), generator=gen, device="cuda") + st.direction
    st.q = q.to(_torch_dtype(case))


def _view(case, st, k, v, off, off_v, seg_len, table, max_tokens):
    import paper_2502_15294_amd as ra
    return ra.KVView(k, v, off, seg_len, st.n_rounds, case["Hkv"], case["d"], max_tokens, block_table=table,
                     block_size=16 if case["paged"] else 0, seg_off_v=off_v)


def _context(case, st, q_len=1, extra=0):
    import paper_2502_15294_amd as ra
    st.ctx = ra.ra_create(0)
    if "Hq" in case:
        n = ra.ra_workspace_bytes(case["B"], case["R"], case["Hq"], case["Hkv"], case["d"], q_len,
                                  ra.RA_BF16 if case["dtype"] == "bf16" else ra.RA_F32, st.tokens + extra)
        st.workspace = torch.empty(n, dtype=torch.uint8, device="cuda")
        ra.ra_set_workspace(st.ctx, st.workspace)


def prepare(case, seed):
    rng = np.random.default_rng([seed, 1])
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = State()
    st.case = case
    B, op = case["B"], case["op"]
    if op == "commit":
        _prepare_commit(case, rng, gen, st)
        if own:
            _context(case, st)
        return st
    _rounds(case, rng, st)
    if op == "evict":
        st.weights = torch.randn((B, st.tokens), generator=gen, device="cuda").mul_(2).exp_().mul_(1e-3)
        # weights that a token never attended has: exact ties at zero
        st.weights[torch.rand((B, st.tokens), generator=gen, device="cuda") < 0.05] = 0
        if own:
            _context(case, st)
        return st
    _cache(case, rng, gen, st, values=op != "weights")
    if op == "compact":
        _prepare_compact(case, rng, gen, st)
    else:
        _selection(case, rng, st)
    if op == "tree":
        n = case["nodes"]
        _queries(case, n, gen, st)
        cur_len = rng.integers(case["cur"] // 2, case["cur"] + 1, size=B).astype(np.int32)
        tree_len = np.where(rng.random(B) < 0.5, n, rng.integers((n + 1) // 2, n + 1, size=B)).astype(np.int32)
        st.cap = case["cur"] + n
        shape = (B, st.cap, case["Hkv"], case["d"])
        st.cur_k = torch.randn(shape, generator=gen, device="cuda").to(st.k.dtype)
        st.cur_v = torch.randn(shape, generator=gen, device="cuda").to(st.k.dtype)
        sees = np.zeros((B, n, n), dtype=bool)  # a node sees its ancestors and itself
        for b in range(B):
            for i in range(n):
                parent = int(rng.integers(max(-1, i - 9), i)) if i else -1
                if parent >= 0:
                    sees[b, i] = sees[b, parent]
                sees[b, i, i] = True
        words = (n + 31) // 32
        bits = np.zeros((B, n, words * 32), dtype=np.uint8)
        bits[:, :, :n] = sees
        mask = np.packbits(bits, axis=2, bitorder="little").view(np.uint32).view(np.int32)
        st.cur_len, st.tree_len = torch.from_numpy(cur_len).cuda(), torch.from_numpy(tree_len).cuda()
        st.mask = torch.from_numpy(np.ascontiguousarray(mask)).cuda()
    if op == "weights":
        _queries(case, case["q_len"], gen, st)
        st.prev = torch.rand((B, st.tokens), generator=gen, device="cuda")
        # what the attention of these queries over these tokens (and a few of their own) returned
        logits, _, valid, _ = _logits(st)
        logits = logits.masked_fill_(~valid[:, None, None, :], -math.inf)
        lse = torch.logaddexp(logits.logsumexp(3), torch.randn(logits.shape[:3], generator=gen, device="cuda"))
        st.lse = _by_token(lse.unsqueeze(3), case).squeeze(3).contiguous()
        del logits, lse
    if own:
        st.view = _view(case, st, st.k, st.v, st.seg_off, st.seg_off_v, st.seg_len, st.table, st.tokens)
        _context(case, st, case.get("nodes") or case.get("q_len") or 1, case.get("cur", 0) + case.get("nodes", 0))
    return st


def _prepare_commit(case, rng, gen, st):
    B, n, p = case["B"], case["nodes"], case["path"]
    st.cap = case["cur"] + n
    shape = (B, st.cap, case["Hkv"], case["d"])
    dt = _torch_dtype(case)
    st.ks = [torch.randn(shape, generator=gen, device="cuda", dtype=dt) for _ in range(case["layers"])]
    st.vs = [torch.randn(shape, generator=gen, device="cuda", dtype=dt) for _ in range(case["layers"])]
    st.cur_len = torch.from_numpy(rng.integers(case["cur"] // 2, case["cur"] + 1, size=B).astype(np.int32)).cuda()
    # nodes are numbered level by level: the first one stays or all of them come from behind the path's end, so that a
    # second pass over the same rows moves the same values
    path = np.full((B, p), -1, dtype=np.int32)
    count = rng.integers(0, p + 1, size=B).astype(np.int32)
    for b in range(B):
        path[b, :count[b]] = np.sort(p + rng.choice(n - p, size=count[b], replace=False)) if n - p >= count[b] else np.arange(count[b])
        if count[b] and rng.random() < 0.5:
            path[b, 0] = 0
    st.path, st.n_path = torch.from_numpy(path).cuda(), torch.from_numpy(count).cuda()


def _prepare_compact(case, rng, gen, st):
    """Which tokens stay (as the eviction leaves them), and room for them."""
    B, R = st.lens.shape
    weights = rng.lognormal(0.0, 2.0, size=(B, st.tokens))
    idx = np.full((B, case["budget"]), -1, dtype=np.int32)
    n_kept = np.zeros(B, dtype=np.int32)
    kept_len = np.zeros((B, R), dtype=np.int32)
    for b in range(B):
        total = int(st.lens[b].sum())
        w = weights[b, :total]
        w[:case["first"]] = w[max(0, total - case["last"]):] = np.inf
        keep = np.sort(np.argsort(-w, kind="stable")[:case["budget"]])
        idx[b, :len(keep)] = keep
        n_kept[b] = len(keep)
        ends = np.cumsum(st.lens[b])
        kept_len[b] = np.bincount(np.searchsorted(ends, keep, side="right"), minlength=R)[:R]
    off, off_v, table, nk, nv = _places(kept_len, case["paged"], rng)
    Hkv, d = case["Hkv"], case["d"]
    st.kept_lens, st.kept_off, st.kept_off_v, st.kept_table = kept_len, off, off_v, table
    st.idx, st.n_kept, st.kept_len = torch.from_numpy(idx).cuda(), torch.from_numpy(n_kept).cuda(), torch.from_numpy(kept_len).cuda()
    st.new_off = torch.from_numpy(off).cuda()
    st.new_off_v = None if off_v is None else torch.from_numpy(off_v).cuda()
    st.new_table = None if table is None else torch.from_numpy(table).cuda()
    room = B * (min(case["budget"], st.tokens) + 16 * R)
    assert max(nk, nv) <= room - 1
    st.new_k = torch.zeros((room * Hkv, d), device="cuda", dtype=st.k.dtype)
    st.new_v = torch.zeros((room * Hkv * d,), device="cuda", dtype=st.k.dtype)
    if own:
        st.new_view = _view(case, st, st.new_k, st.new_v, st.new_off, st.new_off_v, st.kept_len, st.new_table, case["budget"])


# ---- plain forms ---------------------------------------------------------------------------------------------------------
def _units(st):
    """The selected rounds of every sequence as units of 16 tokens: (round, first token inside the round, tokens in it from
    there), [B, units]; a unit past the end has no tokens."""
    lens = st.seg_len.long()
    if st.sel is None:
        rounds = torch.arange(lens.shape[1], device="cuda").expand_as(lens)
    else:
        listed_ = torch.arange(lens.shape[1], device="cuda")[None] < st.n_sel[:, None]
        rounds = st.sel.long().clamp(min=0)
        lens = lens.gather(1, rounds) * listed_
    ends = ((lens + 15) // 16).cumsum(1)
    u = torch.arange(st.units, device="cuda").expand(lens.shape[0], -1).contiguous()
    slot = torch.searchsorted(ends, u, right=True).clamp(max=lens.shape[1] - 1)
    start = (ends - (lens + 15) // 16).gather(1, slot)
    tok0 = (u - start) * 16
    left = (lens.gather(1, slot) - tok0) * (u < ends[:, -1:])
    return rounds.gather(1, slot), tok0.clamp(min=0), left.clamp(min=0)


def _gather(st, values):
    """Keys (and values) of the selected rounds as [B, Hkv, 16 * units, d] in 32 bits, which of them are tokens, and their
    positions in the sequence."""
    case = st.case
    Hkv, d = case["Hkv"], case["d"]
    rnd, tok0, left = _units(st)
    B, U = rnd.shape
    g = torch.arange(Hkv, device="cuda")[None, :, None]
    t = torch.arange(16, device="cuda")
    inside = torch.minimum(t.expand(B, U, 16), (left - 1).clamp(min=0)[:, :, None])
    off = st.seg_off.gather(1, rnd)
    if st.table is None:
        lens = st.seg_len.long().gather(1, rnd)
        rows = ((off * Hkv + tok0)[:, None] + g * lens[:, None])[..., None] + inside[:, None]
        tiles = ((st.seg_off_v.gather(1, rnd) * Hkv + tok0)[:, None] + g * ((lens + 15) // 16 * 16)[:, None]) // 16
    else:
        block = st.table.long().gather(1, (off + tok0 // 16).clamp(max=st.table.shape[1] - 1))
        tiles = block[:, None] * Hkv + g
        rows = tiles[..., None] * 16 + inside[:, None]
    rows = rows.clamp(max=st.k.shape[0] - 1)
    keys = st.k[rows].float().view(B, Hkv, U * 16, d)
    vals = None
    if values:
        vals = st.v.view(-1, d, 16)[tiles.clamp(max=st.v.numel() // (16 * d) - 1)].float()
        vals = vals.transpose(3, 4).reshape(B, Hkv, U * 16, d)
    first = st.seg_len.long().cumsum(1) - st.seg_len
    pos = (first.gather(1, rnd) + tok0)[..., None] + t
    return keys, vals, (t < left[..., None]).view(B, U * 16), pos.view(B, U * 16)


def _by_group(q, case):
    """[B, n, Hq, d] -> [B, Hkv, n * G, d]"""
    B, n, Hq, d = q.shape
    G = Hq // case["Hkv"]
    return q.view(B, n, case["Hkv"], G, d).transpose(1, 2).reshape(B, case["Hkv"], n * G, d)


def _by_token(x, case):
    """[B, Hkv, n * G, d] -> [B, n, Hq, d]"""
    B, Hkv, rows, d = x.shape
    G = case["Hq"] // Hkv
    return x.view(B, Hkv, rows // G, G, d).transpose(1, 2).reshape(B, rows // G, case["Hq"], d)


def _logits(st, values=False):
    keys, vals, valid, pos = _gather(st, values)
    q = _by_group(st.q.float(), st.case)
    return torch.matmul(q, keys.transpose(2, 3)) * st.case["d"] ** -0.5, vals, valid, pos


def _tree_plain(st):
    case = st.case
    n, G = case["nodes"], case["Hq"] // case["Hkv"]
    history, vals, valid, _ = _logits(st, values=True)
    history.masked_fill_(~valid[:, None, None, :], -math.inf)
    ck, cv = st.cur_k.float().transpose(1, 2).contiguous(), st.cur_v.float().transpose(1, 2).contiguous()
    q = _by_group(st.q.float(), case)
    current = torch.matmul(q, ck.transpose(2, 3)) * case["d"] ** -0.5
    node = torch.arange(st.cap, device="cuda")[None] - st.cur_len[:, None]  # [B, cap]: which drafted token a row holds
    j = node.clamp(0, n - 1).long()
    words = st.mask.gather(2, (j // 32)[:, None].expand(-1, n, -1))
    sees = ((words >> (j % 32)[:, None]) & 1).bool() & ((node >= 0) & (node < st.tree_len[:, None]))[:, None]
    sees |= (node < 0)[:, None]
    current.masked_fill_(~sees.repeat_interleave(G, 1)[:, None], -math.inf)
    top = torch.maximum(history.amax(3, keepdim=True), current.amax(3, keepdim=True)).clamp(min=-1e30)
    history = (history - top).exp_()
    current = (current - top).exp_()
    total = history.sum(3, keepdim=True) + current.sum(3, keepdim=True)
    out = (torch.matmul(history, vals) + torch.matmul(current, cv)) / total
    lse = total.log() + top
    drafted = torch.arange(n, device="cuda")[None] < st.tree_len[:, None]
    out, lse = _by_token(out, case), _by_token(lse, case).squeeze(3)
    return out * drafted[:, :, None, None], lse.masked_fill(~drafted[:, :, None], -math.inf)


def _commit_plain(st):
    p = st.path.shape[1]
    b = torch.arange(st.path.shape[0], device="cuda")[:, None]
    j = torch.arange(p, device="cuda")[None]
    used = j < st.n_path[:, None]
    dst = st.cur_len[:, None].long() + j
    src = torch.where(used, st.cur_len[:, None] + st.path, dst)
    for layer in (*st.ks, *st.vs):
        layer[b, dst] = layer[b, src]
    return [*st.ks, *st.vs], st.cur_len + st.n_path


def _weights_plain(st):
    logits, _, valid, pos = _logits(st)
    lse = _by_group(st.lse.unsqueeze(3), st.case)
    w = (logits - lse).exp_().masked_fill_(~valid[:, None, None, :], 0).sum((1, 2))
    return st.prev.scatter_add(1, pos.clamp(max=st.tokens - 1), w)


def _evict_plain(st):
    case = st.case
    B, n = st.weights.shape
    pos = torch.arange(n, device="cuda")[None]
    total = st.seg_len.sum(1, keepdim=True)
    w = st.weights.masked_fill((pos < case["first"]) | (pos >= total - case["last"]), math.inf)
    w = w.masked_fill(pos >= total, -math.inf)
    take = min(case["budget"], n)
    order = w.sort(dim=1, descending=True, stable=True).indices[:, :take]
    kept = torch.zeros((B, n), dtype=torch.bool, device="cuda").scatter_(1, order, True) & (pos < total)
    n_kept = kept.sum(1, dtype=torch.int32)
    place = (kept.cumsum(1) - 1).masked_fill(~kept, case["budget"])
    idx = torch.full((B, case["budget"] + 1), -1, dtype=torch.int32, device="cuda")
    idx.scatter_(1, place, pos.int().expand(B, -1))
    left = torch.zeros((B, n + 1), device="cuda").scatter_(1, place.masked_fill(~kept, n), st.weights)[:, :n]
    left = left * (pos < n_kept[:, None])
    before = torch.cat([torch.zeros((B, 1), dtype=torch.int64, device="cuda"), kept.cumsum(1)], 1)
    ends = st.seg_len.cumsum(1)
    kept_len = (before.gather(1, ends) - before.gather(1, ends - st.seg_len)).int()
    unit = (kept_len.long() + 15) // 16 * (1 if case["paged"] else 16)
    off = unit.cumsum(1) - unit + (0 if case["paged"] else _stride(case)) * torch.arange(B, device="cuda")[:, None]
    return idx[:, :-1].contiguous(), n_kept, kept_len, off, left


def _stride(case):
    """Tokens of a sequence's part of the smaller cache: the budget, and what its rounds' last tiles waste."""
    return (case["budget"] + 15 * case["R"] + 15) // 16 * 16


def _compact_plain(st):
    case = st.case
    Hkv, d = case["Hkv"], case["d"]
    B, K = st.idx.shape
    used = torch.arange(K, device="cuda")[None] < st.n_kept[:, None]
    pos = st.idx.long().clamp(min=0)
    ends, new_ends = st.seg_len.long().cumsum(1), st.kept_len.long().cumsum(1)
    R = ends.shape[1]
    rnd = torch.searchsorted(ends, pos, right=True).clamp(max=R - 1)
    t = pos - (ends - st.seg_len).gather(1, rnd)
    new_t = torch.arange(K, device="cuda")[None] - (new_ends - st.kept_len).gather(1, rnd)
    g = torch.arange(Hkv, device="cuda")[None, :, None]
    c = torch.arange(d, device="cuda") * 16

    def places(off, off_v, lens, table, t, spare_k, spare_v):
        t = t.clamp(min=0)
        o = off.gather(1, rnd)
        if table is None:
            n = lens.long().gather(1, rnd)
            rows = (o * Hkv + t)[:, None] + g * n[:, None]
            cols = ((off_v.gather(1, rnd) * Hkv + t // 16 * 16)[:, None] + g * ((n + 15) // 16 * 16)[:, None]) * d + (t % 16)[:, None]
        else:
            block = table.long().gather(1, (o + t // 16).clamp(max=table.shape[1] - 1))
            rows = (block[:, None] * Hkv + g) * 16 + (t % 16)[:, None]
            cols = (block[:, None] * Hkv + g) * d * 16 + (t % 16)[:, None]
        return rows.masked_fill(~used[:, None], spare_k), cols.masked_fill(~used[:, None], spare_v)[..., None] + c

    rows, cols = places(st.seg_off, st.seg_off_v, st.seg_len, st.table, t, 0, 0)
    new_rows, new_cols = places(st.new_off, st.new_off_v, st.kept_len, st.new_table, new_t, st.new_k.shape[0] - 1,
                                st.new_v.numel() - 16 * d)
    st.new_k[new_rows] = st.k[rows] * used[:, None, :, None]
    st.new_v[new_cols] = st.v[cols] * used[:, None, :, None]
    return st.new_k, st.new_v


_PLAIN = {"tree": _tree_plain, "commit": _commit_plain, "weights": _weights_plain, "evict": _evict_plain, "compact": _compact_plain}


# ---- the library's calls -------------------------------------------------------------------------------------------------
def _run_own(st):
    import paper_2502_15294_amd as ra
    case, op = st.case, st.case["op"]
    if op == "tree":
        return ra.ra_round_sparse_attn_tree(st.ctx, st.q, st.view, st.mask, st.cur_k, st.cur_v, st.cur_len, tree_len=st.tree_len,
                                            sel_idx=st.sel, n_sel=st.n_sel)
    if op == "commit":
        new_len = ra.ra_tree_commit(st.ctx, st.ks, st.vs, st.cur_len, st.path, st.n_path)
        return [*st.ks, *st.vs], new_len
    if op == "weights":
        return ra.ra_token_weights(st.ctx, st.q, st.view, st.lse, prev=st.prev, n_pos=st.tokens, sel_idx=st.sel, n_sel=st.n_sel)
    if op == "evict":
        return ra.ra_select_tokens(st.ctx, st.weights, st.seg_len, st.n_rounds, case["budget"], keep_first=case["first"],
                                   keep_last=case["last"], block_size=16 if case["paged"] else 0,
                                   stride=0 if case["paged"] else _stride(case))
    ra.ra_compact_rounds(st.ctx, st.view, st.idx, st.n_kept, st.new_view)
    return st.new_k, st.new_v


def run(st):
    return _run_own(st) if own else _PLAIN[st.case["op"]](st)


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------------
def _round_block(st, b, r, off, off_v, lens, table, k, v):
    """Keys [Hkv, len, d] and values [Hkv, len, d] of one round, as views or gathers of its block; which rows of `k` and which
    elements of `v` they are."""
    Hkv, d = st.case["Hkv"], st.case["d"]
    n = int(lens[b, r])
    o = int(off[b, r])
    t = torch.arange(n, device="cuda")
    head = torch.arange(Hkv, device="cuda")[:, None]
    if table is None:
        rows = o * Hkv + head * n + t
        ov = int(off_v[b, r]) if off_v is not None else o
        n16 = -(-n // 16) * 16
        elems = (ov * Hkv + head * n16 + t // 16 * 16) * d + t % 16
    else:
        blocks = torch.as_tensor(table[b, o:o + -(-n // 16)], device="cuda").long()
        rows = (blocks[t // 16] * Hkv + head) * 16 + t % 16
        elems = (blocks[t // 16] * Hkv + head) * d * 16 + t % 16
    elems = elems[..., None] + 16 * torch.arange(d, device="cuda")
    return rows, elems


def _history(st, b, rounds, values):
    host = _host(st)
    ks, vs = [], []
    for r in rounds:
        rows, elems = _round_block(st, b, r, host[0], host[1], st.lens, host[2], st.k, st.v)
        ks.append(st.k[rows].double())
        if values:
            vs.append(st.v[elems].double())
    Hkv, d = st.case["Hkv"], st.case["d"]
    empty = torch.zeros((Hkv, 0, d), dtype=torch.float64, device="cuda")
    return torch.cat([empty, *ks], 1), torch.cat([empty, *vs], 1) if values else None


def _host(st):
    if not hasattr(st, "host"):
        st.host = (st.seg_off.cpu().numpy(), None if st.seg_off_v is None else st.seg_off_v.cpu().numpy(),
                   None if st.table is None else st.table.cpu().numpy())
    return st.host


def _chosen(st, b):
    return range(int(st.n[b])) if st.sel is None else st.sel[b, :int(st.n_sel[b])].tolist()


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "tree":
        return _tree_exact(st)
    if op == "commit":
        path, count, start = st.path.cpu().numpy(), st.n_path.cpu().numpy(), st.cur_len.cpu().numpy()
        moved = []
        for layer in (*st.ks, *st.vs):
            new = layer.double()
            for b in range(case["B"]):
                for j in range(int(count[b])):
                    new[b, start[b] + j] = layer[b, start[b] + path[b, j]].double()
            moved.append(new)
        return moved, torch.from_numpy(start + count).cuda()
    if op == "weights":
        total = st.prev.double()
        for b in range(case["B"]):
            first = np.cumsum(st.lens[b]) - st.lens[b]
            for r in _chosen(st, b):
                if st.lens[b, r] == 0:
                    continue
                keys, _ = _history(st, b, [r], False)
                for g in range(case["Hkv"]):
                    G = case["Hq"] // case["Hkv"]
                    q = st.q[b, :, g * G:(g + 1) * G].double().reshape(-1, case["d"])
                    lse = st.lse[b, :, g * G:(g + 1) * G].double().reshape(-1, 1)
                    total[b, first[r]:first[r] + st.lens[b, r]] += torch.exp(q @ keys[g].T / math.sqrt(case["d"]) - lse).sum(0)
        return total
    if op == "evict":
        return _evict_exact(st)
    new_k, new_v = torch.zeros_like(st.new_k, dtype=torch.float64), torch.zeros_like(st.new_v, dtype=torch.float64)
    host, idx = _host(st), st.idx.cpu().numpy()
    for b in range(case["B"]):
        ends = np.cumsum(st.lens[b])
        at = 0
        for r in range(int(st.n[b])):
            m = int(st.kept_lens[b, r])
            t = torch.as_tensor(idx[b, at:at + m] - (ends[r] - st.lens[b, r]), device="cuda").long()
            rows, elems = _round_block(st, b, r, host[0], host[1], st.lens, host[2], st.k, st.v)
            new_rows, new_elems = _round_block(st, b, r, st.kept_off, st.kept_off_v, st.kept_lens, st.kept_table, st.new_k, st.new_v)
            new_k[new_rows] = st.k[rows[:, t]].double()
            new_v[new_elems] = st.v[elems[:, t]].double()
            at += m
    return new_k, new_v


def _tree_exact(st):
    case = st.case
    B, n, Hq, Hkv, d = case["B"], case["nodes"], case["Hq"], case["Hkv"], case["d"]
    G = Hq // Hkv
    out = torch.zeros((B, n, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, n, Hq), -math.inf, dtype=torch.float64, device="cuda")
    words = st.mask.cpu().numpy().view(np.uint32)
    for b in range(B):
        c, m = int(st.cur_len[b]), int(st.tree_len[b])
        keys, vals = _history(st, b, _chosen(st, b), True)
        keys = torch.cat([keys, st.cur_k[b, :c + m].double().transpose(0, 1)], 1)
        vals = torch.cat([vals, st.cur_v[b, :c + m].double().transpose(0, 1)], 1)
        blind = np.zeros((m, keys.shape[1]), dtype=bool)
        for i in range(m):
            for j in range(m):
                blind[i, keys.shape[1] - m + j] = not (int(words[b, i, j // 32]) >> (j % 32)) & 1
        blind = torch.from_numpy(blind).cuda()
        for h in range(Hq):
            s = st.q[b, :m, h].double() @ keys[h // G].T / math.sqrt(d)
            s[blind] = -math.inf
            lse[b, :m, h] = torch.logsumexp(s, 1)
            out[b, :m, h] = torch.exp(s - lse[b, :m, h, None]) @ vals[h // G]
    return out, lse


def _evict_exact(st):
    case = st.case
    B, R, budget = case["B"], case["R"], case["budget"]
    w = st.weights.cpu().double().numpy()
    idx = np.full((B, budget), -1, dtype=np.int32)
    n_kept, kept_len = np.zeros(B, dtype=np.int32), np.zeros((B, R), dtype=np.int32)
    off, left = np.zeros((B, R), dtype=np.int64), np.zeros_like(w)
    for b in range(B):
        total = int(st.lens[b].sum())
        forced = set(range(min(case["first"], total))) | set(range(max(0, total - case["last"]), total))
        others = sorted((p for p in range(total) if p not in forced), key=lambda p: (-w[b, p], p))
        keep = np.sort(np.array([*sorted(forced), *others][:budget], dtype=np.int64))
        idx[b, :len(keep)], n_kept[b] = keep, len(keep)
        left[b, :len(keep)] = w[b, keep]
        at = 0 if case["paged"] else b * _stride(case)
        end = 0
        for r in range(R):
            begin, end = end, end + int(st.lens[b, r])
            kept_len[b, r] = np.searchsorted(keep, end) - np.searchsorted(keep, begin)
            off[b, r] = at
            at += -(-int(kept_len[b, r]) // 16) * (1 if case["paged"] else 16)
    return tuple(torch.from_numpy(x).cuda() for x in (idx, n_kept, kept_len, off, left))


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    op, B = case["op"], case["B"]
    e = 2 if case.get("dtype") == "bf16" else 4
    if op == "commit":
        rows = B * case["path"] / 2
        return {"bytes": 2 * 2 * rows * case["layers"] * case["Hkv"] * case["d"] * e + 4 * B * (case["path"] + 3), "flops": 0}
    tokens = case["R"] * (case["lo"] + case["hi"]) / 2
    if op == "evict":
        kept = min(case["budget"], tokens)
        return {"bytes": 4 * B * (2 * tokens + case["budget"]) + 16 * B * case["R"], "flops": 0 * kept}
    kv = case["Hkv"] * case["d"] * e
    if op == "compact":
        return {"bytes": 2 * 2 * B * min(case["budget"], tokens) * kv, "flops": 0}
    seen = case["keep"] * tokens
    if op == "weights":
        rows = case["q_len"] * case["Hq"]
        return {"bytes": B * (seen * kv + rows * (case["d"] * e + 4) + 8 * tokens), "flops": 2.0 * B * seen * rows * case["d"]}
    seen += 0.75 * case["cur"] + 0.9 * case["nodes"]
    rows = case["nodes"] * case["Hq"]
    return {"bytes": B * (2 * seen * kv + rows * (case["d"] * (e + 4) + 4)), "flops": 4.0 * B * seen * rows * case["d"]}
