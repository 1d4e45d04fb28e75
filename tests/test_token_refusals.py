"""What the calls on drafted tokens and on single tokens refuse, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2502_15294_amd as ra

BLANK = C.create_string_buffer(4096)  # a context that holds nothing: no workspace, no compute units
CTX = C.c_void_p(C.addressof(BLANK))
BAD, NOT_MADE = ra.RA_ERR_INVALID_ARG, ra.RA_ERR_UNSUPPORTED


def view(B=2, R=3, Hkv=2, d=64, dtype=torch.float32, values=True, **more):
    k = torch.zeros(B * R * 16 * Hkv * d, dtype=dtype)
    lens = torch.full((B, R), 16, dtype=torch.int32)
    off = (torch.arange(R) * 16).repeat(B, 1)
    v = ra.KVView(k, k.clone() if values else None, off, lens, torch.full((B,), R, dtype=torch.int32), Hkv, d, R * 16)
    for name, value in more.items():
        setattr(v.c, name, value)
    return v


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def refused(code, call, *args, **kw):
    with pytest.raises(ra.RaError) as e:
        call(*args, stream=0, **kw)
    assert e.value.code == code, e.value
    return str(e.value)


# ---- tree ------------------------------------------------------------------------------------------------------------------
def tree(ctx=CTX, v=None, n=3, Hq=4, cap=8, dtype=torch.float32, d=64, Hkv=2, B=2, **kw):
    v = v or view(dtype=dtype, d=d, Hkv=Hkv, B=B)
    args = dict(q=torch.zeros(B, n, Hq, d, dtype=dtype), mask=i32(B, n, (n + 31) // 32), ck=torch.zeros(B, cap, Hkv, d, dtype=dtype),
                cv=torch.zeros(B, cap, Hkv, d, dtype=dtype), cl=i32(B))
    args.update({k: kw.pop(k) for k in list(kw) if k in args})
    return ra.ra_round_sparse_attn_tree, (ctx, args["q"], v, args["mask"], args["ck"], args["cv"], args["cl"]), kw


def misaligned(t):
    return torch.zeros(t.numel() + 1, dtype=t.dtype)[1:].view(t.shape)


TREE = {
    "no context": (BAD, dict(ctx=None), "NULL"),
    "no room": (BAD, dict(n=9, cap=8), "no room"),
    "no nodes": (BAD, dict(n=0), "positive"),
    "heads": (BAD, dict(Hq=3), "multiple"),
    "group": (NOT_MADE, dict(Hq=34), "exceeds 16"),
    "channels": (NOT_MADE, dict(d=32), "head_dim"),
    "scale": (BAD, dict(scale=0.0), "scale"),
    "scale NaN": (BAD, dict(scale=float("nan")), "scale"),
    "half a selection": (BAD, dict(sel_idx=i32(2, 3)), "both"),
    "no mask": (BAD, dict(mask=None), "tree_mask"),
    "no current round": (BAD, dict(ck=None, cv=torch.zeros(2, 0, 2, 64)), "cur_k"),
    "no lengths": (BAD, dict(cl=None), "cur_len"),
    "alignment": (BAD, dict(q=misaligned(torch.zeros(2, 3, 4, 64))), "aligned"),
    "no workspace": (ra.RA_ERR_WORKSPACE, dict(), "workspace"),
    "no workspace, bf16": (ra.RA_ERR_WORKSPACE, dict(dtype=torch.bfloat16, d=128), "workspace"),
    "no workspace, 64 channels": (ra.RA_ERR_WORKSPACE, dict(dtype=torch.bfloat16, d=64, n=40, cap=50), "workspace"),
}


@pytest.mark.parametrize("name", list(TREE))
def test_tree_refuses(name):
    code, change, text = TREE[name]
    call, args, kw = tree(**change)
    assert text in refused(code, call, *args, **kw)


def test_tree_checks_its_tensors():
    for change in (dict(mask=i32(2, 3, 2)), dict(mask=torch.zeros(2, 3, 1)), dict(q=torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)),
                   dict(q=torch.zeros(1, 3, 4, 64)), dict(cv=torch.zeros(2, 7, 2, 64)), dict(cl=torch.zeros(2, dtype=torch.int64)),
                   dict(tree_len=i32(3)), dict(sel_idx=i32(2, 4), n_sel=i32(2)), dict(out=torch.zeros(2, 3, 4, 32)), dict(lse=torch.zeros(2, 3))):
        call, args, kw = tree(**change)
        with pytest.raises(ValueError):
            call(*args, stream=0, **kw)
    call, args, kw = tree(q=torch.zeros(2, 4, 3, 64).transpose(1, 2))
    with pytest.raises(AssertionError, match="contiguous"):
        call(*args, stream=0, **kw)


def test_tree_masks():
    m = ra.make_tree_mask([[-1, 0, 0, 2], [-1, -1]])
    assert m[:, :, 0].tolist() == [[1, 3, 5, 13], [1, 2, 0, 0]]
    m = ra.make_tree_mask([list(range(-1, 69))])
    assert m.shape == (1, 70, 3) and m[0, 69].tolist() == [-1, -1, 63] and m[0, 31].tolist() == [-1, 0, 0] and m[0, 30, 0] == 0x7fffffff
    for parents in ([0], [-1, 1], [-1, -2]):
        with pytest.raises(ValueError):
            ra.make_tree_mask([parents])


# ---- commit ------------------------------------------------------------------------------------------------------------------
def test_commit_refuses():
    k, v = ([torch.zeros(2, 8, 2, 64) for _ in range(2)] for _ in range(2))
    ok = dict(cur_k_layers=k, cur_v_layers=v, cur_len=i32(2), path=i32(2, 3), n_path=i32(2))
    call = ra.ra_tree_commit
    assert "NULL" in refused(BAD, call, None, **ok)
    same = i32(2)
    for name in ("cur_len", "n_path"):
        assert "another buffer" in refused(BAD, call, CTX, **{**ok, name: same, "new_len": same})
    assert "another buffer" in refused(BAD, call, CTX, **{**ok, "new_len": ok["path"].flatten()[2:4]})
    assert "positive" in refused(BAD, call, CTX, **{**ok, "path": i32(2, 0)})
    refused(BAD, call, CTX, **{**ok, "path": None})
    assert "aligned" in refused(BAD, call, CTX, **{**ok, "cur_v_layers": [v[0], misaligned(v[1])]})
    odd = [torch.zeros(2, 8, 1, 6)]
    assert "multiple of 16" in refused(NOT_MADE, call, CTX, **{**ok, "cur_k_layers": odd, "cur_v_layers": [odd[0].clone()]})
    for change in (dict(cur_k_layers=[]), dict(cur_v_layers=v[:1]), dict(cur_k_layers=[k[0], torch.zeros(2, 9, 2, 64)]), dict(path=i32(3, 3)),
                   dict(n_path=torch.zeros(2))):
        with pytest.raises(ValueError):
            call(CTX, **{**ok, **change}, stream=0)
    with pytest.raises(TypeError):
        call(CTX, **{**ok, "cur_k_layers": [t.double() for t in k], "cur_v_layers": [t.double() for t in v]}, stream=0)
    with pytest.raises(TypeError):
        call(CTX, **{**ok, "cur_k_layers": 3}, stream=0)


# ---- weights -----------------------------------------------------------------------------------------------------------------
def test_weights_refuse():
    ok = dict(q=torch.zeros(2, 3, 4, 64), view=view(), lse=torch.zeros(2, 3, 4))
    call = ra.ra_token_weights
    assert "NULL" in refused(BAD, call, None, **ok)
    assert "multiple" in refused(BAD, call, CTX, **{**ok, "q": torch.zeros(2, 3, 3, 64), "lse": torch.zeros(2, 3, 3)})
    assert "q_len" in refused(BAD, call, CTX, **{**ok, "q": torch.zeros(2, 0, 4, 64), "lse": torch.zeros(2, 0, 4)})
    assert "n_pos" in refused(BAD, call, CTX, **{**ok, "n_pos": 0})
    assert "scale" in refused(BAD, call, CTX, **{**ok, "scale": -1.0})
    assert "both" in refused(BAD, call, CTX, **{**ok, "n_sel": i32(2)})
    assert "exceeds 16" in refused(NOT_MADE, call, CTX, **{**ok, "q": torch.zeros(2, 3, 34, 64), "lse": torch.zeros(2, 3, 34)})
    assert "head_dim" in refused(NOT_MADE, call, CTX, **{**ok, "q": torch.zeros(2, 3, 4, 32), "view": view(d=32)})
    assert "lse" in refused(BAD, call, CTX, **{**ok, "lse": None})
    assert "aligned" in refused(BAD, call, CTX, **{**ok, "q": misaligned(ok["q"])})
    assert "too large" in refused(NOT_MADE, call, CTX, **{**ok, "n_pos": 8, "view": view(max_tokens=1 << 40)})
    for change in (dict(lse=torch.zeros(2, 4, 3)), dict(lse=torch.zeros(2, 3, 4).double()), dict(q=torch.zeros(2, 3, 4, 64).bfloat16()),
                   dict(prev=torch.zeros(2, 9), weights=torch.zeros(2, 8)), dict(prev=torch.zeros(1, 9)), dict(q=torch.zeros(6, 4, 64)),
                   dict(n_pos=1 << 40), dict(q=torch.zeros(2, 3))):
        with pytest.raises(ValueError):
            call(CTX, **{**ok, **change}, stream=0)


# ---- selection ---------------------------------------------------------------------------------------------------------------
def test_selection_refuses():
    ok = dict(weights=torch.zeros(2, 40), seg_len=i32(2, 3), n_rounds=i32(2), budget=10)
    call = ra.ra_select_tokens
    assert "NULL" in refused(BAD, call, None, **ok)
    for change in (dict(budget=0), dict(budget=-3), dict(keep_first=-1), dict(keep_last=-1), dict(keep_first=6, keep_last=5)):
        assert "budget" in refused(BAD, call, CTX, **{**ok, **change})
    assert "block_size" in refused(NOT_MADE, call, CTX, **{**ok, "block_size": 32})
    assert "stride" in refused(BAD, call, CTX, **{**ok, "stride": -1})
    assert "R_max" in refused(NOT_MADE, call, CTX, **{**ok, "seg_len": i32(2, 1025)})
    assert "positive" in refused(BAD, call, CTX, **{**ok, "seg_len": i32(2, 0)})
    assert "another buffer" in refused(BAD, call, CTX, **{**ok, "kept_weights": ok["weights"]})
    both = torch.zeros(3, 40)
    assert "another buffer" in refused(BAD, call, CTX, **{**ok, "weights": both[:2], "kept_weights": both[1:]})
    assert "other buffers" in refused(BAD, call, CTX, **{**ok, "kept_len": ok["seg_len"]})
    assert "other buffers" in refused(BAD, call, CTX, **{**ok, "n_kept": ok["n_rounds"]})
    assert "2^24" in refused(NOT_MADE, call, CTX, torch.zeros(1, (1 << 24) + 1), i32(1, 3), i32(1), 10)
    for change in (dict(seg_len=torch.zeros(2, 3)), dict(n_rounds=i32(3)), dict(weights=torch.zeros(40)), dict(weights=torch.zeros(2, 40).half()),
                   dict(kept_idx=i32(2, 9)), dict(kept_off=i32(2, 3))):
        with pytest.raises(ValueError):
            call(CTX, **{**ok, **change}, stream=0)
    with pytest.raises(OverflowError):
        call(CTX, **{**ok, "budget": 1 << 40}, stream=0)
    with pytest.raises(TypeError):
        call(CTX, **{**ok, "budget": 1.5}, stream=0)


# ---- compaction --------------------------------------------------------------------------------------------------------------
def test_compaction_refuses():
    call, src, dst, idx, n = ra.ra_compact_rounds, view(), view(), i32(2, 9), i32(2)
    assert "NULL" in refused(BAD, call, None, src, idx, n, dst)
    for other in (view(R=4), view(Hkv=1), view(d=128), view(dtype=torch.bfloat16)):
        assert "differ" in refused(BAD, call, CTX, src, idx, n, other)
    assert "neither" in refused(BAD, call, CTX, src, idx, n, view(values=False))
    assert "of its own" in refused(BAD, call, CTX, src, idx, n, src)
    assert "head_dim" in refused(NOT_MADE, call, CTX, view(d=32), idx, n, view(d=32))
    assert "positive" in refused(BAD, call, CTX, src, i32(2, 0), n, dst)
    assert "aligned" in refused(BAD, call, CTX, src, idx, n, view(k=dst.c.k + 4))
    assert "dst" in refused(BAD, call, CTX, src, idx, n, view(block_size=16))
    for a, b in ((i32(3, 9), n), (idx, i32(3)), (idx.long(), n)):
        with pytest.raises(ValueError):
            call(CTX, src, a, b, dst, stream=0)
    with pytest.raises(AttributeError):
        call(CTX, src, None, n, dst, stream=0)
