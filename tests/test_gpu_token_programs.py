"""The calls on drafted tokens and on single tokens as programs use them: on streams of their own, recorded into graphs, two
at a time, with less workspace, and built under other instruction schedules."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2502_15294_amd as ra
from paper_2502_15294_amd import build as rabuild
from token_reference import TORCH, Cache, context

pytestmark = pytest.mark.gpu
HELPER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "token_hashes.py")
LENS = [[300, 17, 0, 640, 33], [5], [64, 64, 900]]


class Program:
    """A drafted step and an eviction over static buffers."""

    def __init__(self, dtype="bf16", d=128, n=40, paged=True, seed=0, budget=300):
        self.cache = c = Cache(LENS, 2, d, dtype, paged, seed=seed)
        self.n, self.budget, self.dtype = n, budget, dtype
        self.ctx, self.ws = context(c, 8, n, n + 50)
        self.mask = ra.make_tree_mask([[max(-1, i - 1 - i % 3) for i in range(n)]] * c.B).cuda()
        self.q = torch.empty((c.B, n, 8, d), dtype=TORCH[dtype], device="cuda")
        self.k, self.v = (torch.empty((c.B, n + 50, 2, d), dtype=TORCH[dtype], device="cuda") for _ in range(2))
        self.cur_len = torch.tensor([20, 0, 50], dtype=torch.int32, device="cuda")
        self.path = torch.tensor([[0, 2, 5], [1, -1, -1], [-1, -1, -1]], dtype=torch.int32, device="cuda")
        self.n_path = torch.tensor([3, 1, 0], dtype=torch.int32, device="cuda")
        stride = (budget + 15 * c.R + 15) // 16 * 16
        self.stride = stride
        self.k2 = torch.zeros((c.B * stride * 2, d), dtype=TORCH[dtype], device="cuda")
        self.v2 = torch.zeros((c.B * stride * 2 * d,), dtype=TORCH[dtype], device="cuda")

    def fill(self, seed):
        gen = torch.Generator("cuda").manual_seed(seed)
        for t in (self.q, self.k, self.v):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))

    def run(self, stream=None):
        c = self.cache
        out, lse = ra.ra_round_sparse_attn_tree(self.ctx, self.q, c.view, self.mask, self.k, self.v, self.cur_len, stream=stream)
        new_len = ra.ra_tree_commit(self.ctx, [self.k], [self.v], self.cur_len, self.path, self.n_path, stream=stream)
        w = ra.ra_token_weights(self.ctx, self.q, c.view, lse, stream=stream)
        idx, n, kept_len, kept_off, left = ra.ra_select_tokens(self.ctx, w, c.seg_len, c.n_rounds, self.budget, 4, 20, 0, self.stride, stream=stream)
        small = ra.KVView(self.k2, self.v2, kept_off, kept_len, c.n_rounds, 2, c.d, self.budget)
        ra.ra_compact_rounds(self.ctx, c.view, idx, n, small, stream=stream)
        return [out, lse, new_len, w, idx, n, kept_len, kept_off, left, self.k, self.v, self.k2, self.v2]


def same(a, b):
    torch.cuda.synchronize()
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,d,n", [("bf16", 128, 40), ("bf16", 128, 3), ("bf16", 64, 9), ("f32", 64, 9)])
def test_on_a_stream_of_its_own(dtype, d, n):
    p = Program(dtype, d, n)
    p.fill(1)
    want = [t.clone() for t in p.run()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(10 ** 7)  # what another stream ran ahead with would see the old inputs
        p.fill(1)
        got = p.run()
    s.synchronize()
    assert same(got, want)
    p.fill(1)
    torch.cuda.synchronize()
    got = p.run(stream=s)  # named instead of current
    s.synchronize()
    assert same(got, want)
    ra.ra_destroy(p.ctx)


@pytest.mark.parametrize("dtype,d,n", [("bf16", 128, 40), ("bf16", 128, 7), ("bf16", 128, 2), ("f32", 128, 9)])
def test_recorded_into_a_graph(dtype, d, n):
    p = Program(dtype, d, n)
    p.fill(1)
    p.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = p.run()
    for seed in (2, 3, 4):
        p.fill(seed)
        g.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in got]
        p.fill(seed)
        assert same(p.run(), replayed), seed
    ra.ra_destroy(p.ctx)


def test_long_selection_recorded_into_a_graph():
    w = torch.empty((2, 150000), device="cuda")
    lens = torch.full((2, 300), 490, dtype=torch.int32, device="cuda")
    n = torch.tensor([300, 200], dtype=torch.int32, device="cuda")
    ctx = ra.ra_create(0)
    call = lambda: ra.ra_select_tokens(ctx, w, lens, n, 40000, 4, 30)  # noqa: E731
    w.normal_()
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call()
    for seed in (1, 2, 3):
        w.normal_(generator=torch.Generator("cuda").manual_seed(seed))
        g.replay()
        assert same(got, call()), seed
    ra.ra_destroy(ctx)


def test_two_at_once():
    """Two contexts, each with a workspace of its own, on two streams."""
    a, b = Program("bf16", 128, 40, seed=1), Program("bf16", 128, 9, paged=False, seed=2)
    want = []
    for p in (a, b):
        p.fill(7)
        want.append([t.clone() for t in p.run()])
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for p in (a, b):
            p.fill(7)
        torch.cuda.synchronize()
        x, y = a.run(stream=s), b.run(stream=t)
        torch.cuda.synchronize()
        assert same(x, want[0]) and same(y, want[1])
    for p in (a, b):
        ra.ra_destroy(p.ctx)


@pytest.mark.parametrize("dtype,d,n", [("bf16", 128, 40), ("bf16", 128, 7), ("bf16", 128, 2), ("bf16", 64, 60), ("f32", 64, 20)])
def test_with_less_workspace(dtype, d, n):
    """Fewer pieces, or a refusal; never another result."""
    p = Program(dtype, d, n)
    p.fill(3)
    call = lambda: ra.ra_round_sparse_attn_tree(p.ctx, p.q, p.cache.view, p.mask, p.k, p.v, p.cur_len)  # noqa: E731
    want, want_lse = call()
    bytes_, refused, served = p.ws.numel(), 0, 0
    while bytes_ >= 32768:
        ws = torch.full((bytes_,), 0xff, dtype=torch.uint8, device="cuda")
        ra.ra_set_workspace(p.ctx, ws)
        try:
            out, lse = call()
        except ra.RaError as e:
            assert e.code == ra.RA_ERR_WORKSPACE
            refused += 1
        else:
            # weights in fp32 whatever the cut: 2^-23 of each, and the sums' order
            assert (out - want).abs().max().item() <= 2.0 ** -17 and (lse - want_lse).abs().max().item() <= 1e-5
            assert refused == 0
            served += 1
        torch.cuda.synchronize()
        bytes_ = bytes_ * 2 // 3 // 256 * 256
    assert refused and served
    ra.ra_destroy(p.ctx)


def test_outputs_of_the_caller():
    p = Program("f32", 64, 9)
    p.fill(1)
    want = p.run()
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    got = ra.ra_round_sparse_attn_tree(p.ctx, p.q, p.cache.view, p.mask, p.k.clone(), p.v.clone(), p.cur_len, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    new_len = torch.empty_like(p.cur_len)
    assert ra.ra_tree_commit(p.ctx, (p.k,), (p.v,), p.cur_len, p.path, p.n_path, new_len=new_len) is new_len
    outs = [torch.empty_like(t) for t in want[4:9]]
    got = ra.ra_select_tokens(p.ctx, want[3], p.cache.seg_len, p.cache.n_rounds, p.budget, 4, 20, 0, p.stride, *outs)
    assert all(x is y for x, y in zip(got, outs)) and same(outs, want[4:9])
    ra.ra_destroy(p.ctx)


def _hashes(library):
    env = dict(os.environ)
    env.pop("RA_LIBRARY", None)
    if library:
        env["RA_LIBRARY"] = library
    r = subprocess.run([sys.executable, "-u", HELPER], env=env, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads([l for l in r.stdout.splitlines() if l.startswith("HASHES ")][-1][len("HASHES "):])


def test_outputs_do_not_depend_on_the_instruction_schedule():
    have = []
    for strategy in rabuild.ALT_STRATEGIES:
        lib = rabuild.alt_library(strategy)
        if os.path.exists(lib) and os.path.exists(lib + ".stamp") and open(lib + ".stamp").read() == rabuild.sources_digest():
            have.append((strategy, lib))
    if not have:
        pytest.skip("no up-to-date alternative builds (python -m paper_2502_15294_amd.build --alt-schedules)")
    ref = _hashes(None)
    unstable = {k: v for k, v in ref.items() if isinstance(v, list)}
    assert not unstable, unstable
    for strategy, lib in have:
        got = _hashes(lib)
        assert got == ref, (strategy, [k for k in ref if got.get(k) != ref[k]])
