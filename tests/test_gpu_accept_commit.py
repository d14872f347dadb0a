"""Acceptance of drafts and the commit of their rows, against the definitions; whole numbers and moved bits: no tolerance."""
import numpy as np
import pytest

import round_oracle as ro

pytestmark = pytest.mark.gpu


def ints(x):
    import torch
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def accept(draft, root, sampled, lens, nq, parents, alias=False):
    import torch
    from paper_2605_19893_amd import binding as Bd
    B, T = draft.shape
    d = [ints(draft), ints(root), ints(sampled), ints(lens), None if nq is None else ints(nq), None if parents is None else ints(parents)]
    path, n, nxt, com = (torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B, T), (B,), (B,), (B,)))
    if alias:
        nxt, com = d[1], d[3]
    Bd.ssv_accept(*d, B, T, path, n, nxt, com, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (path, n, nxt, com)]


def check(draft, root, sampled, lens, nq, parents, **kw):
    B, T = draft.shape
    path, n, nxt, com = accept(draft, root, sampled, lens, nq, parents, **kw)
    for b in range(B):
        tq = T if nq is None else min(max(nq[b], 0), T)
        want, token, length = ro.accept(draft[b], root[b], sampled[b], lens[b], tq, list(range(-1, T - 1)) if parents is None else list(parents[b]))
        assert path[b].tolist() == want + [-1] * (T - len(want)), b
        assert (n[b], nxt[b], com[b]) == (len(want), token, length), b


@pytest.mark.parametrize("T", [1, 2, 5, 40, 63, 64, 65, 127, 128])
@pytest.mark.parametrize("vocab", [2, 3, 50])
def test_random_trees_and_chains(T, vocab):
    """A vocabulary of two or three tokens: long paths, siblings with the same token, samples that nothing matches."""
    rng = np.random.default_rng(T * 100 + vocab)
    B = 37
    draft, sampled = rng.integers(0, vocab, (B, T)), rng.integers(0, vocab, (B, T))
    root, lens = rng.integers(0, vocab, B), rng.integers(0, 1 << 20, B)
    par = np.stack([[int(rng.integers(max(-1, i - 4), i)) for i in range(T)] for _ in range(B)])
    check(draft, root, sampled, lens, None, None)
    check(draft, root, sampled, lens, None, par)
    check(draft, root, sampled, lens, rng.integers(-1, T + 2, B), par, alias=True)


@pytest.mark.parametrize("T", [64, 65, 128])
def test_whole_chain_accepted(T):
    draft = np.arange(T)[None] + 7
    check(draft, [7], draft + 1, [123456], None, None)
    check(draft, [7], draft + 1, [0], [T - 1], None)


def test_malformed_parents_and_negative_tokens():
    draft = np.array([[4, 5, 6, 4, -1, 5]] * 3)
    par = np.array([[3, -9, 1, 0, 2, 77]] * 3)
    check(draft, [4, 5, -1], np.array([[5, 6, -1, 4, 4, 4]] * 3), [10, 20, 30], [6, 6, 6], par)


def commit_case(seed, dt, *, L, B, T, Hk, dk, dv, cap, paths, counts, lens, layout="dense"):
    import torch
    from paper_2605_19893_amd import binding as Bd
    tdt = torch.bfloat16 if dt == "bf16" else torch.float32
    g = torch.Generator().manual_seed(seed)
    k, v = torch.randn((L, B, Hk, cap, dk), generator=g).to(tdt), torch.randn((L, B, Hk, cap, dv), generator=g).to(tdt)
    if layout == "dense":
        kd, vd = k.cuda(), v.cuda()
    else:                 # [B, cap, L, Hk, d + 8] storage
        kd = torch.full((B, cap, L, Hk, dk + 8), 5.0, dtype=tdt, device="cuda")[..., :dk].permute(2, 0, 3, 1, 4)
        vd = torch.full((B, cap, L, Hk, dv + 8), 5.0, dtype=tdt, device="cuda")[..., :dv].permute(2, 0, 3, 1, 4)
        kd.copy_(k)
        vd.copy_(v)
    p = Bd.make_commit_params(layers=L, B=B, T=T, H_kv=Hk, d_k=dk, d_v=dv, dtype=Bd.SSV_BF16 if dt == "bf16" else Bd.SSV_F32, kv_capacity=cap,
                              k_stride=kd.stride()[:4], v_stride=vd.stride()[:4])
    path = np.full((B, T), -1)
    for b, row in enumerate(paths):
        path[b, :len(row)] = row
    Bd.ssv_commit(kd, vd, ints(path), ints(counts), ints(lens), p, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for host, dev in ((k, kd), (v, vd)):
        want, got = host.float().numpy(), dev.float().cpu().numpy()
        for b in range(B):
            for layer in range(L):
                for h in range(Hk):
                    assert np.array_equal(got[layer, b, h], ro.commit(want[layer, b, h], path[b].tolist(), counts[b], lens[b], T, cap)), (b, layer, h)
    if layout != "dense":
        assert (kd._base[..., dk:] == 5.0).all() and (vd._base[..., dv:] == 5.0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["dense", "rows"])
def test_commit_moves_the_accepted_rows_of_every_layer(dt, layout):
    paths = [[0, 4, 16], [3, 13, 38], [], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 39], list(range(40)), list(range(0, 40, 2)), [39]]
    commit_case(1, dt, L=3, B=7, T=40, Hk=2, dk=192, dv=128, cap=90, paths=paths, counts=[len(p) for p in paths], lens=[0, 50, 20, 3, 50, 7, 50],
                layout=layout)


def test_commit_widths_and_long_paths():
    for dk, dv in ((8, 8), (64, 64), (128, 256), (1000, 24)):
        commit_case(2, "bf16", L=1, B=2, T=128, Hk=3, dk=dk, dv=dv, cap=160, paths=[sorted(np.random.default_rng(dk).permutation(128)[:70].tolist()), list(range(64, 128))],
                    counts=[70, 64], lens=[32, 0])


def test_commit_stops_at_an_entry_that_is_none():
    """Entries that do not ascend, lie outside the draft slots or beyond the capacity end the move; counts beyond T are cut."""
    paths = [[1, 3, 3, 5], [2, 1], [-1, 4], [1, 9], [0, 2, 4, 6], [1, 2, 3, 5, 6, 7], [1, 2], [1, 2]]
    commit_case(3, "f32", L=2, B=8, T=8, Hk=1, dk=64, dv=64, cap=40, paths=paths, counts=[4, 2, 2, 2, 4, 99, -3, 2], lens=[5, 5, 5, 5, 35, 32, 5, -1])
