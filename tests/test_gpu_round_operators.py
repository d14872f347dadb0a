"""The operators of a verification round together, as a serving loop uses them: attention over a shared prefix, logits,
sampling, acceptance, the commit of the accepted rows, the compressed cache, and the next round on what the last one left.
Every step is checked against its definition on the inputs that the steps before it really produced; the same rounds are
then replayed from one captured graph."""
import numpy as np
import pytest

import round_oracle as ro
import ssv_inputs as si

pytestmark = pytest.mark.gpu

B, H, HK, D, P, CAP, VOCAB, ROUNDS = 5, 8, 2, 64, 200, 96, 2, 3      # (two tokens: many drafts are accepted)


class Loop:
    """Buffers of a serving loop, everything on the device; step() enqueues one round on the current stream."""

    def __init__(self, parents, T):
        import torch
        from paper_2605_19893_amd import binding as Bd
        self.T, g = T, torch.Generator().manual_seed(77)
        rnd = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()
        ints = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()
        self.kp, self.vp = rnd(1, HK, P, D), rnd(1, HK, P, D)
        self.k, self.v = rnd(B, HK, CAP, D), rnd(B, HK, CAP, D)
        self.plen, self.lens, self.before = ints([P - 3]), ints([0, 7, 31, 40, 12]), ints([0] * B)
        self.nq = ints([T, T, T - 1, T, 1])
        self.par = None if parents is None else ints([parents] * B)
        self.q, self.w = rnd(B, T, H, D), torch.randn((H * D, VOCAB), generator=g).cuda()
        self.u, self.draft = torch.rand((B, T), generator=g).cuda(), ints(np.random.default_rng(1).integers(0, VOCAB, (B, T)))
        self.root = ints([0, 1, 0, 1, 1])
        self.temp, self.top_p = torch.full((B,), 0.9, device="cuda"), torch.full((B,), 0.95, device="cuda")
        self.out, self.logits = torch.zeros_like(self.q), torch.zeros((B, T, VOCAB), device="cuda")
        self.tokens, self.path = ints(np.full((B, T), -9)), ints(np.full((B, T), -9))
        self.n, self.new_lens = ints([0] * B), ints([0] * B)
        self.kc, self.vc, self.n_cmp = torch.zeros((B, HK, 8, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, HK, 8, D), dtype=torch.bfloat16, device="cuda"), ints([0] * B)
        kw = dict(H_kv=HK, d_k=D, d_v=D)
        self.pp = Bd.make_prefix_params(B=B, T=T, H=H, max_prefix_len=P, max_seq_len=CAP - T, kp_stride=self.kp.stride()[:3], vp_stride=self.vp.stride()[:3],
                                        k_stride=self.k.stride()[:3], v_stride=self.v.stride()[:3], **kw)
        self.sp = Bd.make_sample_params(B=B, T=T, V=VOCAB, dtype=Bd.SSV_F32)
        self.cp = Bd.make_commit_params(B=B, T=T, dtype=Bd.SSV_BF16, kv_capacity=CAP, k_stride=(0, *self.k.stride()[:3]), v_stride=(0, *self.v.stride()[:3]), **kw)
        self.zp = Bd.make_cmp_params(B=B, l=32, d=16, dtype=Bd.SSV_BF16, max_new_rows=8, kv_capacity=CAP, cmp_capacity=8, k_stride=self.k.stride()[:3],
                                     v_stride=self.v.stride()[:3], kc_stride=self.kc.stride()[:3], vc_stride=self.vc.stride()[:3], **kw)
        self.need = Bd.ssv_prefix_workspace_bytes(self.pp), Bd.ssv_sample_workspace_bytes(self.sp)
        self.ws = [torch.full((max(n, 1),), 0x55, dtype=torch.uint8, device="cuda") for n in self.need]

    def attend_and_sample(self):
        import torch
        from paper_2605_19893_amd import binding as Bd
        s = torch.cuda.current_stream().cuda_stream
        Bd.ssv_prefix_verify(self.q, self.kp, self.vp, self.k, self.v, self.plen, self.lens, self.nq, self.par, self.pp, self.out, self.ws[0], self.need[0], s)
        torch.matmul(self.out.reshape(B, self.T, H * D).float(), self.w, out=self.logits)
        Bd.ssv_sample(self.logits, self.temp, None, self.top_p, None, self.u, self.nq, self.sp, self.tokens, None, self.ws[1], self.need[1], s)

    def accept_and_commit(self):
        import torch
        from paper_2605_19893_amd import binding as Bd
        s = torch.cuda.current_stream().cuda_stream
        Bd.ssv_accept(self.draft, self.root, self.tokens, self.lens, self.nq, self.par, B, self.T, self.path, self.n, self.root, self.new_lens, s)
        Bd.ssv_commit(self.k, self.v, self.path, self.n, self.lens, self.cp, s)
        Bd.ssv_nsa_compress(self.k, self.v, self.kc, self.vc, self.before, self.new_lens, self.n_cmp, self.zp, s)
        self.before.copy_(self.new_lens)
        self.lens.copy_(self.new_lens)

    def state(self):
        return [x.clone() for x in (self.k, self.v, self.lens, self.before, self.root, self.kc, self.vc, self.n_cmp)]

    def restore(self, state):
        for x, y in zip((self.k, self.v, self.lens, self.before, self.root, self.kc, self.vc, self.n_cmp), state):
            x.copy_(y)


@pytest.mark.parametrize("fanout", [None, (2, 2), (3, 2, 1)])
def test_rounds(fanout):
    import torch
    parents = None if fanout is None else [int(x) for x in si.tree_parents(fanout, "bfs")]
    T = 6 if parents is None else len(parents)
    lp = Loop(parents, T)
    start, f = lp.state(), lambda x: x.double().cpu().numpy()
    tree = list(range(-1, T - 1)) if parents is None else parents
    nq, after, moved = lp.nq.tolist(), [], 0
    for _ in range(ROUNDS):
        lens, root = lp.lens.tolist(), lp.root.tolist()
        lp.attend_and_sample()
        torch.cuda.synchronize()
        want, mass, size = ro.prefix_attention(f(lp.q), f(lp.kp), f(lp.vp), f(lp.k), f(lp.v), [P - 3], lens, nq, [tree] * B, D ** -0.5)
        # (the terms of the shared-prefix tests: scores and sums in fp32, probabilities and result rounded to bf16)
        tol = 2 * ((D + 4) * 2.0 ** -24 * size + 2.0 ** -22 + (P + CAP) * 2.0 ** -24) * mass + 2.0 ** -8 * (mass + np.abs(want))
        assert (np.abs(f(lp.out) - want) <= tol).all()
        tokens, logits, u = lp.tokens.tolist(), f(lp.logits), lp.u.double().tolist()
        for b in range(B):
            for i in range(T):
                if i >= nq[b]:
                    assert tokens[b][i] == -1
                    continue
                token, _, margin = ro.sample(logits[b, i], float(np.float32(0.9)), 0, float(np.float32(0.95)), 0.0, u[b][i])
                assert margin < 2.0 ** -40 or tokens[b][i] == token
        k0, v0, draft = f(lp.k), f(lp.v), lp.draft.tolist()
        lp.accept_and_commit()
        torch.cuda.synchronize()
        for b in range(B):
            path, token, length = ro.accept(draft[b], root[b], tokens[b], lens[b], nq[b], tree)
            assert lp.path[b].tolist() == path + [-1] * (T - len(path)) and lp.n[b].item() == len(path)
            assert lp.root[b].item() == token and lp.lens[b].item() == length
            moved += sum(p != j for j, p in enumerate(path))
            for c in range(HK):
                for was, now in ((k0, lp.k), (v0, lp.v)):
                    assert np.array_equal(f(now[b, c]), ro.commit(was[b, c], path, len(path), lens[b], T, CAP))
            rows = (length - 32) // 16 + 1 if length >= 32 else 0
            assert lp.n_cmp[b].item() == rows
            for r in range(rows):
                mean = f(lp.k)[b, :, 16 * r:16 * r + 32].mean(1)
                assert (np.abs(f(lp.kc)[b, :, r] - mean) <= 2.0 ** -8 * np.abs(mean) + 1e-6 * 6).all()
        after.append([lp.out.clone(), lp.tokens.clone(), lp.path.clone(), *lp.state()])
    assert sum(x[6].sum().item() for x in after) > 0
    if parents is not None:
        assert moved > 0
    # the same rounds from one graph
    lp.restore(start)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        lp.attend_and_sample()
        lp.accept_and_commit()
    lp.restore(start)
    for want in after:
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, [lp.out, lp.tokens, lp.path, *lp.state()]):
            assert torch.equal(x, y)
        torch.randn(1000, device="cuda").sum().item()


@pytest.mark.parametrize("fanout", [None, (3, 2, 1)])
def test_rounds_of_sparse_attention(fanout, oracle):
    """The same loop around the library's own attention: ssv_nsa_verify on a compressed cache that every round extends by what it committed."""
    import dataclasses

    import torch
    from oracle import compress as oc
    from paper_2605_19893_amd import binding as Bd
    from paper_2605_19893_amd.device_case import DeviceCase
    from parity import check, compare
    start = [1400, 1023, 31]
    parents = None if fanout is None else si.tree_parents(fanout, "bfs")
    T = 8 if parents is None else len(parents)
    nq = [T, T - 2, T]
    nsa, n, Hk, d = si.NsaParams(n_sel=8, w=256), 3, 2, 64
    case = si.make_case("sparse_rounds", "bf16", n, T, 16, Hk, d, d, nsa, [x + T * ROUNDS for x in start], 147, rho=0.5, parents=parents, n_query=nq,
                        cmp_over_drafts=False)
    dev = DeviceCase(case)
    ints = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()
    g = torch.Generator().manual_seed(78)
    w, u = torch.randn((16 * d, VOCAB), generator=g).cuda(), torch.rand((n, T), generator=g).cuda()
    draft, root = ints(np.random.default_rng(2).integers(0, VOCAB, (n, T))), ints([0, 1, 1])
    logits, tokens, path, count = torch.zeros((n, T, VOCAB), device="cuda"), ints(np.full((n, T), -9)), ints(np.full((n, T), -9)), ints([0] * n)
    before, new_lens = ints([0] * n), ints(start)
    dev.seq_lens.copy_(new_lens)
    dev.k_cmp.zero_()
    dev.v_cmp.zero_()
    sp = Bd.make_sample_params(B=n, T=T, V=VOCAB, dtype=Bd.SSV_F32)
    need = Bd.ssv_sample_workspace_bytes(sp)
    ws = torch.full((need,), 0x55, dtype=torch.uint8, device="cuda")
    strides = dict(k_stride=dev.k.stride()[:3], v_stride=dev.v.stride()[:3])
    cp = Bd.make_commit_params(B=n, T=T, H_kv=Hk, d_k=d, d_v=d, dtype=Bd.SSV_BF16, kv_capacity=dev.k.shape[2],
                               k_stride=(0, *strides["k_stride"]), v_stride=(0, *strides["v_stride"]))
    zp = Bd.make_cmp_params(B=n, H_kv=Hk, d_k=d, d_v=d, l=nsa.l, d=nsa.d, dtype=Bd.SSV_BF16, max_new_rows=dev.k_cmp.shape[2], kv_capacity=dev.k.shape[2],
                            cmp_capacity=dev.k_cmp.shape[2], kc_stride=dev.k_cmp.stride()[:3], vc_stride=dev.v_cmp.stride()[:3], **strides)

    def compress(s):
        Bd.ssv_nsa_compress(dev.k, dev.v, dev.k_cmp, dev.v_cmp, before, new_lens, dev.n_cmp, zp, s)
        before.copy_(new_lens)
        dev.seq_lens.copy_(new_lens)

    def attend_and_sample():
        s = torch.cuda.current_stream().cuda_stream
        dev.run()
        torch.matmul(dev.out.reshape(n, T, 16 * d).float(), w, out=logits)
        Bd.ssv_sample(logits, None, None, None, None, u, dev.n_query, sp, tokens, None, ws, need, s)

    def accept_and_commit():
        s = torch.cuda.current_stream().cuda_stream
        Bd.ssv_accept(draft, root, tokens, dev.seq_lens, dev.n_query, dev.parents, n, T, path, count, root, new_lens, s)
        Bd.ssv_commit(dev.k, dev.v, path, count, dev.seq_lens, cp, s)
        compress(s)

    kept = [dev.k, dev.v, dev.k_cmp, dev.v_cmp, dev.n_cmp, dev.seq_lens, before, new_lens, root]
    compress(torch.cuda.current_stream().cuda_stream)
    begin, after, accepted = [x.clone() for x in kept], [], 0
    bits = lambda x: x.view(torch.int16).cpu().numpy().view(np.uint16)
    f = lambda x: x.double().cpu().numpy()
    tree = list(range(-1, T - 1)) if parents is None else [int(p) for p in parents]
    for r in range(ROUNDS):
        lens, first = dev.seq_lens.cpu().numpy(), root.tolist()
        assert dev.n_cmp.tolist() == [oc.n_cmp_rows(int(x), nsa.l, nsa.d) for x in lens]
        attend_and_sample()
        out, sel = dev.results()
        now = dataclasses.replace(case, name=f"sparse_rounds_{r}", seq_lens=lens, n_cmp=dev.n_cmp.cpu().numpy(), k=bits(dev.k), v=bits(dev.v),
                                  k_cmp=bits(dev.k_cmp), v_cmp=bits(dev.v_cmp))
        check(now, compare(now, oracle, oracle.nsa_verify(now), out, sel))
        said, x, given = tokens.tolist(), f(logits), u.double().tolist()
        for b in range(n):
            for i in range(T):
                token, _, margin = ro.sample(x[b, i], 1.0, 0, 1.0, 0.0, given[b][i]) if i < nq[b] else (-1, 0, 1.0)
                assert margin < 2.0 ** -40 or said[b][i] == token
        k0, v0 = f(dev.k), f(dev.v)
        accept_and_commit()
        torch.cuda.synchronize()
        for b in range(n):
            line, token, length = ro.accept(draft[b].tolist(), first[b], said[b], int(lens[b]), nq[b], tree)
            assert path[b].tolist() == line + [-1] * (T - len(line)) and root[b].item() == token and dev.seq_lens[b].item() == length
            accepted += len(line)
            rows = oc.n_cmp_rows(length, nsa.l, nsa.d)
            for c in range(Hk):
                for was, moved, pooled in ((k0, dev.k, dev.k_cmp), (v0, dev.v, dev.v_cmp)):
                    want = ro.commit(was[b, c], line, len(line), int(lens[b]), T, was.shape[2])
                    assert np.array_equal(f(moved[b, c]), want)
                    means = oc.compress(want, 0, length, nsa.l, nsa.d, "bf16")[2]
                    assert (np.abs(f(pooled[b, c, :rows]) - means) <= 2.0 ** -8 * np.abs(means) + 33 * 2.0 ** -24 * np.abs(want[:length]).max()).all()
        after.append([dev.out.clone(), dev.sel_idx.clone(), tokens.clone(), path.clone()] + [x.clone() for x in kept])
    assert accepted > 0
    # the same rounds from one graph
    for x, y in zip(kept, begin):
        x.copy_(y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        attend_and_sample()
        accept_and_commit()
    for x, y in zip(kept, begin):
        x.copy_(y)
    for want in after:
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, [dev.out, dev.sel_idx, tokens, path] + kept):
            assert torch.equal(x, y)
        torch.randn(1000, device="cuda").sum().item()
