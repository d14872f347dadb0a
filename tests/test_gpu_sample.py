"""Sampling against its definition in 64 bits: the token is the definition's, except where the given number lies within the
rounding of a border (2^-40 of the kept sum, which 2^20 roundings of 2^-53 and the filters' fixed-point sums stay far below);
the probability is off by its one rounding to fp32 and 2^-40."""
import numpy as np
import pytest

import round_oracle as ro

pytestmark = pytest.mark.gpu


def run(x, t=None, k=None, p=None, m=None, u=None, nq=None, stride=(0, 0), probs=True):
    """x: device tensor [B, T, V] (or a view); per-sequence lists; u [B, T]."""
    import torch
    from paper_2605_19893_amd import binding as Bd
    B, T, V = x.shape
    dev = lambda v, dt: None if v is None else torch.tensor(v, dtype=dt, device="cuda")
    prm = Bd.make_sample_params(B=B, T=T, V=V, dtype=Bd.SSV_BF16 if x.dtype == torch.bfloat16 else Bd.SSV_F32,
                                logits_stride=stride)
    need = Bd.ssv_sample_workspace_bytes(prm)
    ws = torch.full((max(need, 1),), 0x55, dtype=torch.uint8, device="cuda")
    tokens = torch.full((B, T), -9, dtype=torch.int32, device="cuda")
    pr = torch.full((B, T), -9.0, device="cuda") if probs else None
    Bd.ssv_sample(x, dev(t, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32),
                  torch.as_tensor(np.asarray(u, np.float32)).cuda(), dev(nq, torch.int32), prm, tokens, pr, ws if need else None, need,
                  torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), None if pr is None else pr.double().cpu().numpy()


def check(x, t, k, p, m, u, nq=None, **kw):
    """x: device tensor; every row against the definition."""
    tok, pr = run(x, t, k, p, m, u, nq, **kw)
    h = x.double().cpu().numpy()
    f32 = lambda v, d: np.float64(np.float32(d if v is None else v))
    for b in range(h.shape[0]):
        for i in range(h.shape[1]):
            if nq is not None and i >= nq[b]:
                assert tok[b, i] == -1 and pr[b, i] == 0
                continue
            want, prob, margin = ro.sample(h[b, i], f32(None if t is None else t[b], 1), 0 if k is None else k[b], f32(None if p is None else p[b], 1),
                                           f32(None if m is None else m[b], 0), float(np.float32(u[b][i])))
            if margin > 2.0 ** -40:
                assert tok[b, i] == want, (b, i, tok[b, i], want, margin)
                assert abs(pr[b, i] - prob) <= (2.0 ** -24 + 2.0 ** -40) * prob, (b, i, pr[b, i], prob)


def logits(seed, shape, dtype, tail=0.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(shape, generator=g)
    return (2.0 * z + tail * z.clamp_min(0) ** 2).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.95, 0.0), (0.7, 40, 0.9, 0.02), (0.0, 0, 1.0, 0.0), (1.5, 1000, 0.99, 0.001), (2.0, 5, 1.0, 0.0),
            (1.0, 0, 1.0, 0.1), (0.3, 0, 0.5, 0.0), (1.0, 1, 1.0, 0.0), (5.0, 0, 0.999, 0.0), (1.0, 3000, 0.9999, 0.0), (0.01, 0, 0.9, 0.3)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 8191, 8192, 8193, 32000, 50001, 131071])
def test_settings_over_vocabularies(dtype, V):
    rng = np.random.default_rng(V)
    B = len(SETTINGS)
    x = logits(V, (B, 2, V), dtype)
    t, k, p, m = (list(c) for c in zip(*SETTINGS))
    check(x, t, k, p, m, rng.random((B, 2)))


def test_neutral_settings_by_null_pointers_and_no_probabilities():
    rng = np.random.default_rng(5)
    x = logits(5, (3, 4, 777), "f32")
    u = rng.random((3, 4))
    check(x, None, None, None, None, u)
    a, _ = run(x, u=u)
    b, none = run(x, u=u, probs=False)
    assert none is None and np.array_equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_go_to_the_lowest_index(dtype):
    """Values from a handful: the threshold falls inside a class of equal logits, whose first indices are kept."""
    import torch
    g = torch.Generator().manual_seed(3)
    x = torch.randint(0, 5, (8, 2, 20011), generator=g).float().to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    rng = np.random.default_rng(3)
    check(x, [1.0] * 8, [1, 7, 100, 4001, 9000, 0, 0, 4500], [1.0, 1.0, 1.0, 1.0, 0.7, 0.3, 0.9, 0.77], [0, 0, 0, 0, 0, 0, 0.2, 0.3], rng.random((8, 2)))


def test_all_equal_logits():
    import torch
    x = torch.full((5, 1, 640), -2.5, dtype=torch.bfloat16, device="cuda")
    u = [[0.05], [0.55], [0.95], [0.999], [0.0]]
    tok, pr = run(x, [1.0] * 5, [10] * 5, None, None, u)
    assert tok[:, 0].tolist() == [0, 5, 9, 9, 0] and np.allclose(pr, 0.1, rtol=1e-6)
    tok, _ = run(x, [1.0] * 5, None, None, None, u)
    assert tok[:, 0].tolist() == [32, 352, 607, 639, 0]      # (0.95 in fp32 is 0.94999999: 607.99999 of 640)


def test_masked_infinite_and_nan_logits():
    import torch
    inf, nan = float("inf"), float("nan")
    rows = [[-inf] * 9, [nan] * 9, [-inf, 1.0, -inf, 1.0, -inf, nan, 1.0, -inf, -inf], [0.0, inf, 3.0, inf, -inf, nan, 1.0, 2.0, 5.0],
            [-3.4028235e38, -inf, -3.4028235e38, -inf, -inf, -inf, -inf, -inf, nan], [-0.0, 0.0, -0.0, 0.0, -1.0, -1.0, -inf, -inf, -inf]]
    for dt in (torch.float32, torch.bfloat16):
        x = torch.tensor(rows, dtype=dt).reshape(6, 1, 9).repeat(1, 4, 1).cuda()
        u = [[0.0, 0.3, 0.7, 0.999]] * 6
        for t, k, p, m in [(1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.5, 2, 1.0, 0.0), (0.5, 0, 0.6, 0.0), (2.0, 0, 1.0, 0.5), (1.0, 8, 0.9, 0.9), (1.0, 3, 0.7, 1.0)]:
            check(x, [t] * 6, [k] * 6, [p] * 6, [m] * 6, u)
        tok, pr = run(x, [1.0] * 6, None, None, None, u)
        assert (tok[:2] == -1).all() and (pr[:2] == 0).all()
        assert set(tok[2]) <= {1, 3, 6} and set(tok[3]) <= {1, 3}
        # the lowest finite fp32 value lies beyond the largest of bf16, (2 - 2^-7) 2^127, and rounds to -inf there
        assert set(tok[4]) <= ({0, 2} if dt == torch.float32 else {-1})


def test_odd_settings():
    """What the documentation says of values out of range."""
    nan = float("nan")
    x = logits(9, (12, 1, 3001), "f32")
    t = [-1.0, nan, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1e-30, 1e30, float("inf"), 1e-45]
    k = [0, 0, -4, 99999, 0, 0, 0, 0, 0, 0, 0, 0]
    p = [1.0, 1.0, 1.0, 1.0, nan, -0.5, 0.0, 7.0, 0.9, 0.9, 1.0, 1.0]
    m = [0.0, 0.0, 0.0, 0.0, nan, 0.0, 0.0, 3.0, 0.0, 0.0, 0.0, 0.0]
    check(x, t, k, p, m, np.random.default_rng(9).random((12, 1)))


def test_random_numbers_at_the_ends():
    x = logits(10, (5, 1, 5000), "bf16")
    x[:, :, 4000:] = float("-inf")
    u = [[0.0], [1.0], [float("nan")], [-3.0], [np.nextafter(np.float32(1), np.float32(0))]]
    check(x, [1.0] * 5, [0] * 5, [1.0, 1.0, 0.9, 0.9, 0.9], [0.0] * 5, u)


def test_strides_ragged_counts_and_unaligned_rows():
    """Rows that start at every alignment, a padded vocabulary, nodes that do not exist (their logits are not read)."""
    import torch
    B, T, V = 4, 5, 1501
    for dt in ("bf16", "f32"):
        h = logits(21, (B, T, V), dt)
        for off in range(0, 8):
            buf = torch.full((B * T * (V + 13) + 64,), 50.0, dtype=h.dtype, device="cuda")
            x = buf[off:].as_strided((B, T, V), (T * (V + 13), V + 13, 1), off)
            x.copy_(h)
            x[1, 3:] = 1000.0
            check(x, [0.9] * B, [0, 20, 0, 0], [0.9, 1.0, 1.0, 0.5], [0.0, 0.0, 0.01, 0.0], np.random.default_rng(off).random((B, T)),
                  nq=[5, 3, 0, 1], stride=x.stride()[:2])


def test_graph_replays_and_another_stream():
    import torch
    from paper_2605_19893_amd import binding as Bd
    x = logits(31, (4, 3, 9001), "bf16")
    u = torch.rand((4, 3), device="cuda")
    t, p = torch.full((4,), 0.9, device="cuda"), torch.full((4,), 0.9, device="cuda")
    prm = Bd.make_sample_params(B=4, T=3, V=9001, dtype=Bd.SSV_BF16)
    need = Bd.ssv_sample_workspace_bytes(prm)
    ws = torch.full((max(need, 1),), 0x55, dtype=torch.uint8, device="cuda")
    tok, pr = torch.empty((4, 3), dtype=torch.int32, device="cuda"), torch.empty((4, 3), device="cuda")
    go = lambda s: Bd.ssv_sample(x, t, None, p, None, u, None, prm, tok, pr, ws, need, s.cuda_stream)
    go(torch.cuda.current_stream())
    want = tok.clone(), pr.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go(s)
    for _ in range(3):
        tok.fill_(-7)
        ws.fill_(0x55)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok, want[0]) and torch.equal(pr, want[1])
        torch.randn(1000, device="cuda").sum().item()


def test_frequencies_follow_the_probabilities():
    """Evenly spaced numbers give every kept token its share, to within one number."""
    n = 4096
    x = logits(41, (1, 1, 50), "f32").expand(1, n, 50)
    u = ((np.arange(n) + 0.5) / n)[None]
    tok, _ = run(x, [1.0], [0], [0.95], [0.0], u, stride=(50, 0))
    h = x[0, 0].double().cpu().numpy()
    order = np.argsort(-h, kind="stable")
    w = np.exp(h - h.max())
    keep = np.cumsum(w[order]) - w[order] < float(np.float32(0.95)) * w.sum()
    share = np.zeros(50)
    share[order[keep]] = w[order[keep]] / w[order[keep]].sum()
    assert (np.abs(np.bincount(tok[0], minlength=50) - n * share) <= 1.0 + 1e-6).all()


def test_lists_of_every_length():
    """Kept entries around what one wavefront solves, what is sorted and what is listed, and the general way beyond: flat rows, where
    the thresholds fall among thousands of candidates, by count, by mass and by both."""
    rng = np.random.default_rng(51)
    V = 50021
    for dt in ("f32", "bf16"):
        x = 0.3 * logits(51, (10, 2, V), dt, tail=0.0)
        k = [60, 64, 65, 500, 1100, 2047, 2600, 4000, 9000, 30000]
        check(x, [1.0] * 10, k, [1.0] * 10, [0.0] * 10, rng.random((10, 2)))
        check(x, [1.0] * 10, k, [0.8, 0.99, 0.5, 0.9, 0.7, 0.97, 0.3, 0.9, 0.6, 0.999], [0.0] * 5 + [0.2] * 5, rng.random((10, 2)))
        check(x, [1.0] * 10, [0] * 10, [0.0005, 0.002, 0.01, 0.04, 0.1, 0.3, 0.5, 0.8, 0.95, 0.9999], [0.0] * 10, rng.random((10, 2)))
        check(x, [1.0] * 10, [0] * 10, [1.0] * 10, [0.9, 0.8, 0.7, 0.6, 0.5, 0.4, 0.3, 0.2, 0.1, 0.01], rng.random((10, 2)))


def test_masked_vocabularies():
    """Most of the vocabulary at -inf: fewer entries than top-k, whole blocks without one."""
    import torch
    x = logits(52, (6, 1, 40000), "bf16")
    x[:, :, 100:39990] = float("-inf")
    x[3, :, 5:] = float("-inf")
    x[4, :, :39999] = float("-inf")
    x[5] = torch.where(torch.rand((1, 40000), device="cuda") < 0.9, float("-inf"), x[5])
    for s in SETTINGS:
        check(x, [s[0]] * 6, [s[1]] * 6, [s[2]] * 6, [s[3]] * 6, np.random.default_rng(52).random((6, 1)))


def test_largest_vocabulary_and_many_rows():
    import torch
    from paper_2605_19893_amd import binding as Bd
    V = Bd.SSV_SAMPLE_MAX_V
    x = logits(53, (4, 1, V), "f32")
    rng = np.random.default_rng(53)
    check(x, [1.0, 0.7, 0.9, 3.0], [0, 50, 0, 3000], [1.0, 0.9, 0.95, 0.9], [0.0, 0.0, 0.0, 0.0], rng.random((4, 1)))
    y = torch.zeros(V + 5, dtype=torch.bfloat16, device="cuda")[5:].reshape(1, 1, V)       # an unaligned row of equal logits
    check(y, [1.0], [0], [0.5], [0.0], [[0.7]])
    x = logits(54, (700, 3, 257), "bf16")
    n = 700
    check(x, [0.9] * n, [0 if i % 3 else 7 for i in range(n)], [0.9 if i % 2 else 1.0 for i in range(n)], [0.0] * n, rng.random((n, 3)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 16, 200, 3000, 12000])
def test_top_p_that_ends_on_a_border(n, dtype):
    """n equal logits, all others out of reach: half of the mass is n / 2 entries, neither more nor fewer, whatever the logit and the
    temperature (sums of equal weights are exact)."""
    import torch
    V = 3 * n + 5
    x = torch.full((8, 1, V), -2000.0)
    at = torch.randperm(V, generator=torch.Generator().manual_seed(n))[:n]
    tops = [1000.0, 0.1, -3.7, 7.3e4, 1e-3, 12.34, 1000.0, -1e-30]
    for b, top in enumerate(tops):
        x[b, 0, at] = top
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    t, p = [10.0, 0.7, 1.0, 3.0, 0.1, 1.3, 0.01, 1.0], [0.5, 0.25, 0.5, 0.75, 0.5, 0.5, 0.5, 0.25]
    p = p if n % 4 == 0 else [0.5] * 8
    for u in (0.3, 0.9999999):
        check(x, t, [0] * 8, p, [0.0] * 8, [[u]] * 8)
        check(x, t, [V - 1] * 8, p, [0.0] * 8, [[u]] * 8)


def test_extreme_temperatures():
    import torch
    x = logits(61, (10, 2, 9000), "f32")
    x[:, :, ::7] = float("-inf")
    x[:, :, 3] = float("nan")
    t = [float("inf"), 3e38, 1e30, 1e6, 1e-6, 1e-30, 1e-38, 1e-45, float("inf"), 1e-20]
    for k, p, m in ((0, 1.0, 0.0), (50, 1.0, 0.0), (0, 0.3, 0.0), (0, 1.0, 0.5), (3000, 0.9, 0.0)):
        check(x, t, [k] * 10, [p] * 10, [m] * 10, np.random.default_rng(61).random((10, 2)))
    check(torch.sign(x) * 3e38, t, [0] * 10, [1.0] * 10, [0.0] * 10, np.random.default_rng(62).random((10, 2)))


def kept_by_mass(x, top_k, top_p):
    """(entries that top_k and top_p keep of a row at temperature 1, distance of the target from the nearest border in entries), in
    numbers of 64 bits of mantissa: 2^20 roundings of a running sum of 53 are as large as a weight of e^-30."""
    big = np.longdouble
    ws = np.sort(np.exp(x.astype(big) - big(x.max())))[::-1]
    if 0 < top_k < len(ws):
        ws = ws[:top_k]
    upto = np.cumsum(ws)
    target = big(np.float32(top_p)) * upto[-1]
    n = int(np.sum(upto < target)) + 1
    return n, float(min(upto[n - 1] - target, target - (upto[n - 2] if n > 1 else 0)) / ws[n - 1])


@pytest.mark.parametrize("V, top_k", [(1 << 20, 0), (1 << 20, (1 << 20) - 1), (1 << 20, 700000), (60000, 0), (1 << 20, 4000), (1 << 20, 500)])
def test_top_p_near_one_behind_a_peak(V, top_k):
    """One likely token and a long tail of weights about 2^-43 (where top_k cuts the tail short: 2^-34 and more), in descending order:
    the last kept entry, which u = 1 asks for, says how many were kept.  The filters' sums are off by V 2^-63 of the whole at most, with a short
    list of top_k by 2^-40 (half a unit for every one of its entries, were they all rounded the same way), the target and the row's sum by 2^-50."""
    import torch
    few = 0 < top_k < 10000
    x = torch.full((V,), -100.0)
    x[0] = 0.0
    if few:        # as many alike as are kept at most
        x[1:top_k + 1] = -23.6 if top_k > 1000 else -21.5
    else:
        shift = np.log(2.0 ** 20 / V)
        x[1:] = torch.linspace(-29.0 + shift, -30.0 + shift, V - 1)
    x = x.reshape(1, 1, V)
    for top_p in (0.9999999, 1.0 - 2.0 ** -24):
        n, off = kept_by_mass(x[0, 0].numpy(), top_k, top_p)
        w = float(np.exp(x[0, 0, n - 1].double().item()))
        slack = ((2.0 ** -40 if few else V * 2.0 ** -63) + 2.0 ** -50) / w
        tok, pr = run(x.cuda(), [1.0], [top_k], [top_p], [0.0], [[1.0]])
        assert 1 < n < (top_k or V)
        assert abs(tok[0, 0] + 1 - n) <= (np.ceil(slack) if off < slack else 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_min_p_whose_border_is_zero(dtype):
    """Settings for which M + t ln(min_p) is zero but for a trillionth: its rounding in 64 bits is thousands of 32-bit steps there."""
    import torch
    rows = [(0.1, 1.2476844787597656, 0.5418624877929688), (0.1, 3.2534255981445312, 1.4129447937011719), (0.1, 41.04684829711914, 17.826419830322266),
            (0.05, 2.2117958068847656, 0.7383155822753906), (0.05, 11.779285430908203, 3.9320220947265625), (0.02, 13.251354217529297, 3.387340545654297),
            (0.7, 1.9285774230957031, 5.407100677490234), (0.7, 19.910770416259766, 55.82329177856445), (0.5, 31.799739837646484, 45.87732696533203),
            (0.25, 8.473453521728516, 6.1123046875), (0.9, 3.0236740112304688, 28.698352813720703), (0.0625, 4.0, 1.4426950408889634)]
    m, top, t = (list(c) for c in zip(*rows))
    B = len(rows)
    x = torch.linspace(-0.995, 0.975, 198).repeat(B, 4, 1) * torch.tensor(top)[:, None, None]      # (no value within a thousandth of the border)
    x = torch.cat([x, torch.tensor(top)[:, None, None].expand(B, 4, 1)], 2)
    x = x.bfloat16() if dtype == "bf16" else x
    u = [[0.05, 0.35, 0.65, 0.95]] * B
    check(x.cuda(), t, [0] * B, [1.0] * B, m, u)
    check(x.cuda(), t, [150] * B, [1.0] * B, m, u)
    check(x.cuda(), t, [0] * B, [0.9] * B, m, u)


def test_block_sums_are_good_to_64_bits():
    """A border at u = 1/2 to within 2e-13 of the sum, between two blocks: 2048 logits whose exponentials are alike, and as much and a
    little less (or more) beside the maximum itself.  The sums of a block take eleven additions and an exponential of
    4e-16, the row's a few more: together below 2e-15 of the sum."""
    import math
    import torch
    f32 = lambda v: float(np.float32(v))
    V = 8192
    for k, d in enumerate(f32(v) for v in -math.log(2) * np.array([0.02, 0.13, 0.25, 0.36, 0.47, 0.5, 0.62, 0.75, 0.88, 0.98, 1.3, 1.5])):
        for eta in (8e-13, -8e-13):
            # block 0: 0 and 2047 logits at d; blocks 1 and 2: as many of -0.05 as fit, then a few that make up the difference; block 3: nothing
            first = 1.0 + 2047.0 * math.exp(d)
            want = first * (1.0 - eta)
            y = f32(-0.05)
            count = int(want / math.exp(y))
            values, left = [y] * count, want - count * math.exp(y)
            while left > 1e-15 * want:
                v = float(np.nextafter(np.float32(math.log(left)), np.float32(-np.inf)))
                values.append(v)
                left -= math.exp(v)
            x = np.full(V, -np.inf, np.float32)
            x[0], x[1:2048] = 0.0, d
            x[2048:2048 + len(values)] = values
            big = np.exp(x.astype(np.longdouble))
            margin = float((big[:2048].sum() - big[2048:].sum()) / big.sum() / 2)
            assert 1e-13 < abs(margin) < 2.0 ** -40 and (margin > 0) == (eta > 0)
            tok, _ = run(torch.from_numpy(x).cuda().reshape(1, 1, V), [1.0], None, None, None, [[0.5]])
            assert (tok[0, 0] < 2048) == (margin > 0), (k, d, eta, tok[0, 0], margin)
