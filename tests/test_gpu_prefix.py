"""Shared-prefix attention against its definition in 64 bits.

Tolerance, from the arithmetic, with P the sum of p |v| of the value (a relative error e of every probability moves the
value by at most 2 e P, numerator and denominator together):
  scores: d_k products added in fp32, each sum off by at most d_k 2^-24 times the sum of |q_i k_i|, and the scaling and the
  exponential's argument by 2 roundings of a value of that size: e = (d_k + 4) 2^-24 size, size = max scale sum |q_i k_i|;
  the exponential itself 2^-22; sums over n keys in fp32 n 2^-24 at worst; bf16: every probability rounded once (2^-8, in the
  numerator alone); the result rounded once (2^-8 or 2^-24 of its value)."""
import numpy as np
import pytest

import round_oracle as ro

pytestmark = pytest.mark.gpu

SHAPES = {"bf16_192": ("bf16", 192, 128), "bf16_128": ("bf16", 128, 128), "bf16_64": ("bf16", 64, 64), "f32_64": ("f32", 64, 64)}
TREES = {"chain": None, "tree6": [-1, -1, 0, 0, 1, 1], "messy": [-1, 5, 0, -7, 2, 2, 9, 1]}


def setup(seed, shape, *, B, T, H, Hk, G, plens, lens, nq=None, parents=None, P=None, S=None, strided=False, garbage=True, scale=0.0, sharp=1.0):
    import torch
    from paper_2605_19893_amd import binding as Bd
    dt, dk, dv = SHAPES[shape]
    tdt = torch.bfloat16 if dt == "bf16" else torch.float32
    g = torch.Generator().manual_seed(seed)
    P = max(plens) if P is None else P
    S = max(lens) if S is None else S
    nq = [T] * B if nq is None else nq

    def cache(n, rows, d, used):
        x = torch.randn((n, Hk, rows, d), generator=g).to(tdt)
        if garbage:
            for i, u in enumerate(used):
                x[i, :, u:] = float("nan")
        if strided:       # rows of a [n, rows, Hk, d + 8] buffer
            buf = torch.full((n, rows, Hk, d + 8), 3.0, dtype=tdt, device="cuda")
            buf[..., :d] = x.permute(0, 2, 1, 3)
            return x, buf.permute(0, 2, 1, 3)[..., :d]
        return x, x.cuda()

    has = P > 0
    kp, kp_d = cache(G, P, dk, plens) if has else (None, None)
    vp, vp_d = cache(G, P, dv, plens) if has else (None, None)
    k, k_d = cache(B, S + T, dk, [n + c for n, c in zip(lens, nq)])
    v, v_d = cache(B, S + T, dv, [n + c for n, c in zip(lens, nq)])
    q = (sharp * torch.randn((B, T, H, dk), generator=g)).to(tdt)
    q_d, out = q.cuda(), torch.full((B, T, H, dv), 7.0, dtype=tdt, device="cuda")
    st = {}
    if strided:
        q_d = torch.zeros((B, H, T, dk + 16), dtype=tdt, device="cuda").permute(0, 2, 1, 3)[..., :dk]
        q_d.copy_(q)
        out = torch.full((B, H, T, dv + 8), 7.0, dtype=tdt, device="cuda").permute(0, 2, 1, 3)[..., :dv]
        st = dict(q_stride=q_d.stride()[:3], out_stride=out.stride()[:3])
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    par = None if parents is None else [list(parents)] * B
    p = Bd.make_prefix_params(B=B, T=T, H=H, H_kv=Hk, d_k=dk, d_v=dv, n_prefix=G, dtype=Bd.SSV_BF16 if dt == "bf16" else Bd.SSV_F32,
                              max_prefix_len=P, max_seq_len=S, scale=scale, k_stride=k_d.stride()[:3], v_stride=v_d.stride()[:3],
                              **(dict(kp_stride=kp_d.stride()[:3], vp_stride=vp_d.stride()[:3]) if has else {}), **st)
    need = Bd.ssv_prefix_workspace_bytes(p)
    assert need > 0
    ws = torch.full((need,), 0x55, dtype=torch.uint8, device="cuda")
    args = [q_d, kp_d, vp_d, k_d, v_d, ints(plens) if has else None, ints(lens), ints(nq), None if par is None else ints(par), p, out, ws, need]
    f = lambda x: None if x is None else x.double().numpy()
    host = dict(q=f(q), kp=f(kp), vp=f(vp), k=f(k), v=f(v), plens=plens, lens=lens, nq=nq, parents=par, scale=scale or dk ** -0.5, dk=dk, dt=dt)
    return args, host


def call(args):
    import torch
    from paper_2605_19893_amd import binding as Bd
    Bd.ssv_prefix_verify(*args, torch.cuda.current_stream().cuda_stream)


def check(args, h):
    import torch
    torch.cuda.synchronize()
    got = args[10].double().cpu().numpy()
    want, mass, size = ro.prefix_attention(h["q"], h["kp"], h["vp"], h["k"], h["v"], h["plens"], h["lens"], h["nq"], h["parents"], h["scale"])
    n = max(h["plens"] or [0]) + max(h["lens"]) + got.shape[1]
    e = (h["dk"] + 4) * 2.0 ** -24 * size + 2.0 ** -22 + n * 2.0 ** -24
    rnd = 2.0 ** -8 if h["dt"] == "bf16" else 2.0 ** -24
    tol = 2 * e * mass + (rnd * mass if h["dt"] == "bf16" else 0) + rnd * np.abs(want) + 1e-30
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
    for b in range(got.shape[0]):
        assert (got[b, h["nq"][b]:] == 0).all()


CASES = [
    # lengths around the steps of 32 keys, one row to many rows
    dict(shape="bf16_192", B=1, T=1, H=1, Hk=1, G=1, plens=[1], lens=[0]),
    dict(shape="bf16_192", B=1, T=1, H=16, Hk=1, G=1, plens=[31], lens=[1]),
    dict(shape="bf16_192", B=4, T=1, H=64, Hk=4, G=1, plens=[257], lens=[0, 33, 64, 5]),
    dict(shape="bf16_192", B=2, T=3, H=8, Hk=4, G=1, plens=[64], lens=[31, 32]),
    dict(shape="bf16_192", B=6, T=8, H=32, Hk=2, G=2, plens=[700, 129], lens=[0, 40, 100, 7, 64, 65]),
    dict(shape="bf16_128", B=3, T=16, H=16, Hk=2, G=3, plens=[100, 0, 333], lens=[20, 21, 0]),
    dict(shape="bf16_128", B=1, T=128, H=4, Hk=2, G=1, plens=[96], lens=[70]),
    dict(shape="bf16_64", B=5, T=2, H=16, Hk=16, G=1, plens=[515], lens=[0, 1, 2, 3, 4]),
    dict(shape="bf16_64", B=2, T=70, H=2, Hk=1, G=1, plens=[65], lens=[90, 1]),
    dict(shape="f32_64", B=1, T=1, H=2, Hk=2, G=1, plens=[40], lens=[3]),
    dict(shape="f32_64", B=4, T=5, H=8, Hk=2, G=2, plens=[260, 77], lens=[10, 0, 31, 40]),
    dict(shape="f32_64", B=2, T=9, H=16, Hk=1, G=1, plens=[33], lens=[100, 64]),
    # nobody has a prefix; the cache of a prefix is there but empty
    dict(shape="bf16_192", B=2, T=4, H=16, Hk=1, G=1, plens=[], lens=[130, 0], P=0),
    dict(shape="bf16_64", B=2, T=4, H=4, Hk=2, G=1, plens=[0], lens=[130, 0], P=50),
    dict(shape="f32_64", B=3, T=2, H=2, Hk=2, G=1, plens=[], lens=[0, 0, 65], P=0),
]


@pytest.mark.parametrize("kw", CASES, ids=lambda c: f"{c['shape']}-B{c['B']}T{c['T']}H{c['H']}-{max(c['plens'] or [0])}")
def test_definition(kw):
    kw = dict(kw)
    args, h = setup(11, kw.pop("shape"), **kw)
    call(args)
    check(args, h)


@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("tree", ["tree6", "messy"])
def test_trees_ragged_counts_and_strides(shape, tree):
    T = len(TREES[tree])
    nq = [T, 0, 1, T - 1]
    args, h = setup(12, shape, B=4, T=T, H=8, Hk=2, G=2, plens=[150, 97], lens=[30, 17, 0, 64], nq=nq, parents=TREES[tree], strided=True)
    buf = args[10]
    call(args)
    check(args, h)
    assert (buf._base[..., h["v"].shape[3]:] == 7.0).all()          # the padding of the output is left alone


@pytest.mark.parametrize("shape", ["bf16_192", "f32_64"])
def test_many_rows_of_one_prefix(shape):
    """More stacked rows than any workgroup holds, and a count that ends inside one."""
    Hk = 2 if shape == "bf16_192" else 1
    args, h = setup(13, shape, B=9, T=7, H=8 * Hk, Hk=Hk, G=1, plens=[421], lens=[0, 5, 9, 33, 64, 2, 1, 40, 12], nq=[7, 7, 3, 0, 7, 7, 1, 7, 7])
    call(args)
    check(args, h)


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_scale_and_sharp_scores(shape):
    """Scores of a few hundred: the reference maximum moves often, most probabilities vanish."""
    args, h = setup(14, shape, B=2, T=4, H=4, Hk=2, G=1, plens=[300], lens=[50, 20], scale=0.9, sharp=4.0)
    call(args)
    check(args, h)


def test_lengths_beyond_the_bounds_are_clamped():
    args, h = setup(15, "bf16_64", B=2, T=3, H=4, Hk=2, G=1, plens=[60], lens=[40, 40], garbage=False)
    args[5].fill_(1 << 30)
    args[6].fill_(1 << 30)
    args[7].fill_(99)
    call(args)
    check(args, h)
    args[6][0] = -5
    h["lens"] = [0, 40]
    call(args)
    check(args, h)


def test_same_results_every_time_and_from_a_graph():
    """Bitwise the same eagerly, on another stream, and from every replay of a captured graph between eager work."""
    import torch
    from paper_2605_19893_amd import binding as Bd
    args, h = setup(16, "bf16_192", B=4, T=4, H=32, Hk=2, G=2, plens=[900, 333], lens=[100, 0, 77, 64], nq=[4, 2, 4, 4])
    call(args)
    check(args, h)
    want = args[10].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        Bd.ssv_prefix_verify(*args, s.cuda_stream)
    for _ in range(3):
        args[10].fill_(1.0)
        args[11].fill_(0x55)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(args[10], want)
        torch.randn(1000, device="cuda").sum().item()
    args[10].fill_(1.0)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call(args)
    s.synchronize()
    assert torch.equal(args[10], want)


def test_offsets_beyond_32_bits():
    """Caches of more than 4 GiB: rows a megabyte apart (views into one large buffer)."""
    import torch
    from paper_2605_19893_amd import binding as Bd
    dk, rows, pitch = 64, 2500, 1 << 20          # elements between rows: 2500 rows span 5 GB
    big = torch.empty(rows * pitch + 256, dtype=torch.bfloat16, device="cuda")
    kp = big.as_strided((1, 1, rows, dk), (0, 0, pitch, 1))
    vp = big.as_strided((1, 1, rows, dk), (0, 0, pitch, 1), dk)
    g = torch.Generator().manual_seed(17)
    hk, hv = torch.randn((rows, dk), generator=g).bfloat16(), torch.randn((rows, dk), generator=g).bfloat16()
    kp[0, 0], vp[0, 0] = hk.cuda(), hv.cuda()
    q = torch.randn((2, 1, 1, dk), generator=g).bfloat16()
    k, v = torch.randn((2, 1, 1, dk), generator=g).bfloat16(), torch.randn((2, 1, 1, dk), generator=g).bfloat16()
    p = Bd.make_prefix_params(B=2, T=1, H=1, H_kv=1, d_k=dk, d_v=dk, dtype=Bd.SSV_BF16, max_prefix_len=rows, max_seq_len=0,
                              kp_stride=kp.stride()[:3], vp_stride=vp.stride()[:3], k_stride=(dk, dk, dk), v_stride=(dk, dk, dk))
    need = Bd.ssv_prefix_workspace_bytes(p)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    out = torch.empty((2, 1, 1, dk), dtype=torch.bfloat16, device="cuda")
    args = [q.cuda(), kp, vp, k.cuda(), v.cuda(), ints([rows]), ints([0, 0]), None, None, p, out,
            torch.empty(need, dtype=torch.uint8, device="cuda"), need]
    call(args)
    f = lambda x: x.double().numpy()
    check(args, dict(q=f(q), kp=f(hk)[None, None], vp=f(hv)[None, None], k=f(k), v=f(v), plens=[rows], lens=[0, 0], nq=[1, 1], parents=None,
                     scale=dk ** -0.5, dk=dk, dt="bf16"))


@pytest.mark.parametrize("shape", ["bf16_192", "f32_64"])
@pytest.mark.parametrize("lens", [[1500, 0, 0, 1, 3, 700, 2], [0] * 7, [64, 128, 192, 65, 127, 1, 0], [5, 5, 5, 5, 5, 5, 1023]], ids=str)
def test_slices_dealt_out_by_length(shape, lens):
    """One sequence or prefix much longer than the others, none, and lengths on the tile borders; sequences without nodes."""
    nq = [2, 0, 1, 2, 2, 2, 0]
    args, h = setup(18, shape, B=7, T=2, H=4, Hk=2, G=7, plens=[lens[-1 - i] for i in range(7)], lens=lens, nq=nq, P=1500, S=1500)
    call(args)
    check(args, h)
    args, h = setup(19, shape, B=7, T=2, H=4, Hk=2, G=1, plens=[333], lens=lens, nq=nq, S=1500)
    call(args)
    check(args, h)


@pytest.mark.parametrize("B", [63, 64, 65, 130])
def test_batches_around_one_cache_per_lane(B):
    rng = np.random.default_rng(B)
    args, h = setup(20, "bf16_64", B=B, T=1, H=2, Hk=1, G=1, plens=[77], lens=[int(x) for x in rng.integers(0, 200, B)])
    call(args)
    check(args, h)
    args, h = setup(21, "bf16_64", B=B, T=1, H=2, Hk=2, G=B, plens=[int(x) for x in rng.integers(0, 150, B)], lens=[int(x) for x in rng.integers(0, 20, B)])
    call(args)
    check(args, h)


def test_long_prefix_of_few_rows_and_many_slices():
    """One row against many keys (as many slices as there are slots) and a window of nothing but the node itself."""
    args, h = setup(22, "bf16_192", B=1, T=1, H=1, Hk=1, G=1, plens=[9000], lens=[0])
    call(args)
    check(args, h)
    args, h = setup(23, "bf16_128", B=1, T=2, H=16, Hk=1, G=1, plens=[9000], lens=[5000])
    call(args)
    check(args, h)


def test_two_calls_on_two_streams():
    """Calls with workspaces of their own may overlap."""
    import torch
    sets = [setup(30 + k, "bf16_128", B=3, T=4, H=8, Hk=2, G=1, plens=[700 + k], lens=[40, 0, 9]) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        for (args, _), s in zip(sets, streams):
            with torch.cuda.stream(s):
                call(args)
    torch.cuda.synchronize()
    for args, h in sets:
        check(args, h)


def test_fuzz_of_small_problems():
    """Drawn shapes, lengths, trees and counts."""
    rng = np.random.default_rng(99)
    for case in range(40):
        shape = str(rng.choice(sorted(SHAPES)))
        G = int(rng.choice([1, 1, 2, 3]))
        B, T = G * int(rng.integers(1, 6)), int(rng.choice([1, 1, 2, 5, 17, 33]))
        Hk, Hg = int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 4, 8, 16]))
        par = None if rng.random() < 0.5 else [int(rng.integers(max(-1, i - 3), i)) for i in range(T)]
        top = int(rng.choice([3, 70, 300]))
        print("case", case, shape, B, T, Hk, Hg, G, top, flush=True)
        args, h = setup(1000 + case, shape, B=B, T=T, H=Hk * Hg, Hk=Hk, G=G, plens=[int(x) for x in rng.integers(0, top + 1, G)],
                        lens=[int(x) for x in rng.integers(0, top + 1, B)], nq=[int(x) for x in rng.integers(0, T + 1, B)], parents=par,
                        P=top, S=top, strided=bool(rng.random() < 0.3))
        call(args)
        check(args, h)


@pytest.mark.parametrize("shape", ["bf16_64", "f32_64"])
def test_smallest_scale_weighs_all_rows_alike(shape):
    args, h = setup(40, shape, B=2, T=3, H=16, Hk=1, G=1, plens=[300], lens=[50, 0], scale=2.0 ** -100)
    call(args)
    check(args, h)


@pytest.mark.parametrize("shape", ["bf16_128", "f32_64"])
@pytest.mark.parametrize("B, T", [(1, 1), (3, 9), (70, 1)])
def test_bounds_far_above_the_lengths(shape, B, T):
    """Slices are planned for the bounds; most of them get nothing."""
    args, h = setup(41, shape, B=B, T=T, H=4, Hk=1, G=1, plens=[129], lens=[(7 * b) % 90 for b in range(B)], P=60000, S=4000)
    call(args)
    check(args, h)


@pytest.mark.parametrize("shape, T", [("bf16_128", 70), ("bf16_64", 110), ("f32_64", 110)])
def test_more_rows_than_two_joining_workgroups_per_unit(shape, T):
    """Rows enough that their sums are fetched only where they count; sequences without nodes, slices without keys."""
    args, h = setup(42, shape, B=6, T=T, H=16, Hk=1, G=2, plens=[40, 200], lens=[0, 70, 1, 33, 5, 0], nq=[T, T, 0, T, T - 1, T], P=200, S=600)
    call(args)
    check(args, h)


@pytest.mark.parametrize("T", [2, 9])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_largest_scores_pick_the_largest(shape, T):
    """Scores of 2^25.6 after scaling, whole numbers before it: products and sums are exact, the keys of the largest score share the weight
    and all others vanish (the next is 2^15 lower).  The result is the mean of their values, rounded as probabilities and results are."""
    import torch
    scale = 2.0 ** 15
    args, h = setup(45, shape, B=2, T=T, H=4, Hk=1, G=1, plens=[300], lens=[150, 20], garbage=False, scale=scale)
    for at, name, top in ((0, "q", 9), (1, "kp", 8), (3, "k", 8)):
        h[name] = np.random.default_rng(at).integers(-top, top + 1, h[name].shape).astype(np.float64)
        h[name][..., 48:64], h[name][..., 64:] = top, 0.0
        args[at].copy_(torch.from_numpy(h[name]))
    call(args)
    torch.cuda.synchronize()
    got = args[10].double().cpu().numpy()
    want, mass, _ = ro.prefix_attention(h["q"], h["kp"], h["vp"], h["k"], h["v"], h["plens"], h["lens"], h["nq"], h["parents"], scale)
    assert scale * np.abs(h["kp"][0, 0] @ h["q"][0, 0, 0]).max() > 2.0 ** 25
    rnd = 2.0 ** -8 if h["dt"] == "bf16" else 2.0 ** -24
    assert (np.abs(got - want) <= rnd * (mass + np.abs(want)) + 2.0 ** -22 * mass).all()


def test_thousands_of_sequences():
    """A batch whose sequences and KV heads are 2^16 and more (compared on the device, in 64 bits)."""
    import torch
    from paper_2605_19893_amd import binding as Bd
    Bn, Hk, d, P, S = 8200, 8, 64, 70, 5
    g = torch.Generator(device="cuda").manual_seed(46)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    q, kp, vp, k, v = rnd(Bn, 1, Hk, d), rnd(1, Hk, P, d), rnd(1, Hk, P, d), rnd(Bn, Hk, S + 1, d), rnd(Bn, Hk, S + 1, d)
    lens = (torch.arange(Bn, device="cuda") % (S + 1)).int()
    p = Bd.make_prefix_params(B=Bn, T=1, H=Hk, H_kv=Hk, d_k=d, d_v=d, max_prefix_len=P, max_seq_len=S, kp_stride=kp.stride()[:3], vp_stride=vp.stride()[:3],
                              k_stride=k.stride()[:3], v_stride=v.stride()[:3])
    need = Bd.ssv_prefix_workspace_bytes(p)
    assert need > 0
    out, ws = torch.full_like(q, 7.0), torch.full((need,), 0x55, dtype=torch.uint8, device="cuda")
    call([q, kp, vp, k, v, torch.tensor([P - 1], dtype=torch.int32, device="cuda"), lens, None, None, p, out, ws, need])
    keys = torch.cat([kp[:, :, :P - 1].expand(Bn, -1, -1, -1), k], 2).double()
    vals = torch.cat([vp[:, :, :P - 1].expand(Bn, -1, -1, -1), v], 2).double()
    x = (keys * q[:, 0, :, None].double()).sum(3) * d ** -0.5
    x = x.masked_fill((torch.arange(P + S, device="cuda") - (P - 1) > lens[:, None])[:, None], float("-inf"))
    w = torch.softmax(x, 2)[..., None]
    want, mass = (w * vals).sum(2), (w * vals.abs()).sum(2)
    # (the tolerance of check())
    size = (keys.abs() * q[:, 0, :, None].double().abs()).sum(3).amax(2)[..., None] * d ** -0.5
    tol = 2 * ((d + 4) * 2.0 ** -24 * size + 2.0 ** -22 + (P + S) * 2.0 ** -24) * mass + 2.0 ** -8 * (mass + want.abs())
    assert ((out[:, 0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("shape", ["bf16_192", "bf16_128", "bf16_64"])
def test_sharp_scores_of_many_rows(shape):
    """As test_scale_and_sharp_scores, with rows enough in both parts that they share the key tiles."""
    args, h = setup(43, shape, B=2, T=9, H=8, Hk=2, G=1, plens=[300], lens=[50, 20], scale=0.9, sharp=4.0)
    call(args)
    check(args, h)


@pytest.mark.parametrize("shape", ["bf16_192", "bf16_128", "bf16_64"])
def test_scores_that_rise_from_tile_to_tile(shape):
    """Rows that share key tiles, their reference maximum too low in every tile but a slice's first: one head's scores rise by a factor of
    2^5.5 from one tile of 64 keys to the next (the tiles before keep a share of 2 %), one's by 2^14, one's fall, one's stay; the draft keys
    come highest.  The values tell even tiles from odd ones."""
    import torch
    B, T, H, Hk, P, lens, step = 2, 9, 8, 2, 1000, [700, 333], 8.0
    args, h = setup(44, shape, B=B, T=T, H=H, Hk=Hk, G=1, plens=[P], lens=lens, garbage=False, scale=0.0625, sharp=0.15)
    d, n_tiles = h["dk"], (P - 1) // 64
    factor = np.array([7.625, 19.5, -7.625, 0.0])
    h["q"][..., 0] = factor[np.arange(H) % 4]
    slot = np.arange(h["k"].shape[2])
    h["kp"][0, :, :, 0] = step * (np.arange(P) // 64 - n_tiles)
    h["vp"][0] += 2.0 * (1 - 2 * (np.arange(P) // 64 % 2))[:, None]
    for b in range(B):
        h["k"][b, :, :, 0] = np.where(slot < lens[b], step * (slot // 64 - lens[b] // 64), 2 * step)
        h["v"][b] += 2.0 * (1 - 2 * (slot // 64 % 2))[:, None]
    for at, name in ((0, "q"), (1, "kp"), (2, "vp"), (3, "k"), (4, "v")):
        args[at].copy_(torch.from_numpy(h[name]).bfloat16())
        h[name] = args[at].double().cpu().numpy()
    # a lane holds the keys 32 kb + 8 j + 4 hb + r (hb = 0, 1) of a tile; against the largest score before the tile they sum to more than 512
    for b in range(B):
        for head in (0, 1, 4, 5):
            for keys, n in ((h["kp"][0, head // 4], P), (h["k"][b, head // 4], lens[b])):
                x = h["scale"] / np.log(2.0) * (keys[:n] @ h["q"][b, :, head].T)
                for t in range(1, n // 64):
                    for hb in range(2):
                        mine = [64 * t + 32 * kb + 8 * j + 4 * hb + r for kb in range(2) for j in range(4) for r in range(4)]
                        assert (np.exp2(x[mine] - x[:64 * t].max(0)).sum(0) > 600).all()
    call(args)
    check(args, h)
