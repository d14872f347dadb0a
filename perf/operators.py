"""Performance cases of the operators around a verification round, and their plain forms.

A round of speculative verification is more than its sparse attention: a batch that shares a long prefix attends to it
densely (ssv_prefix_verify), the verifier's logits become tokens (ssv_sample), the tokens say which drafts are accepted
(ssv_accept), and the accepted rows move to the front of the draft slots of every layer's cache (ssv_commit).

Where `own` is false, run() computes these in elementary torch operations; where it is true, it makes the calls of the
package that a user makes.  exact() is the definition in 64 bits, written on its own.
"""
import math

import torch

own = False

FANOUTS = {"tree40": (4, 3, 2), "tree21": (3, 2, 2), "tree6": (2, 2)}


# ---- cases ----------------------------------------------------------------------------------------------------------
def _prefix(name, *, batch, queries, prefix, suffix, n_prefix=1, heads=64, kv_heads=4, d_k=192, d_v=128, dtype="bf16",
            drafts="chain", ragged=False):
    """prefix: rows of the longest prefix; suffix: committed tokens behind it of the longest sequence (the shortest has
    none); ragged: some sequences bring fewer queries than the batch's capacity."""
    case = {"op": "prefix", "batch": batch, "queries": queries, "prefix": prefix, "suffix": suffix, "n_prefix": n_prefix, "heads": heads,
            "kv_heads": kv_heads, "d_k": d_k, "d_v": d_v, "dtype": dtype, "drafts": drafts, "ragged": ragged}
    return {"name": name, **case} if name else case


def _sample(name, *, batch, queries, vocab, rule, dtype="bf16", masked=0.0, ragged=False):
    """rule: the settings of the batch (RULES); masked: share of the vocabulary that a constraint sets to -inf."""
    case = {"op": "sample", "batch": batch, "queries": queries, "vocab": vocab, "rule": rule, "dtype": dtype, "masked": masked,
            "ragged": ragged}
    return {"name": name, **case} if name else case


def _accept(name, *, batch, queries, drafts, agree, ragged=False):
    """agree: probability that the sampled token is the draft token of one of the children."""
    case = {"op": "accept", "batch": batch, "queries": queries, "drafts": drafts, "agree": agree, "ragged": ragged}
    return {"name": name, **case} if name else case


def _commit(name, *, layers, batch, drafts, queries, capacity, kv_heads=4, d_k=192, d_v=128, dtype="bf16"):
    case = {"op": "commit", "layers": layers, "batch": batch, "drafts": drafts, "queries": queries, "capacity": capacity,
            "kv_heads": kv_heads, "d_k": d_k, "d_v": d_v, "dtype": dtype}
    return {"name": name, **case} if name else case


def listed():
    return [
        # four samples of one prompt, one token each: the smallest call of a decoding loop, bound by latency
        _prefix("prefix_decode_small", batch=4, queries=1, prefix=2048, suffix=128),
        # a serving batch behind one system prompt, one token each, odd lengths: bound by memory and matrix cores alike
        _prefix("prefix_decode32", batch=32, queries=1, prefix=16411, suffix=1024),
        # draft trees of forty nodes, two prompts with two samples each, eight query heads per KV head of dimension 128
        _prefix("prefix_tree40", batch=4, queries=40, prefix=12345, suffix=700, n_prefix=2, heads=32, kv_heads=4, d_k=128, d_v=128,
                drafts="tree40", ragged=True),
        # the largest: chains of sixteen in 32 sequences behind a 32K document, bound by the matrix cores
        _prefix("prefix_chain16_32k", batch=32, queries=16, prefix=32768, suffix=2048),
        # a small fp32 model, chains of five, sixteen sequences
        _prefix("prefix_f32", batch=16, queries=5, prefix=4097, suffix=300, heads=8, kv_heads=2, d_k=64, d_v=64, dtype="f32"),
        # one user's chain of eight, nucleus sampling over a small vocabulary: bound by latency
        _sample("sample_chain8", batch=1, queries=8, vocab=32000, rule="nucleus"),
        # a batch with every sequence's own settings, over a large vocabulary of odd size
        _sample("sample_mixed", batch=32, queries=4, vocab=131071, rule="mixed", ragged=True),
        # the largest: pure temperature over the whole vocabulary for every node of a batch of chains, fp32 logits
        _sample("sample_whole_f32", batch=32, queries=16, vocab=100003, rule="temperature", dtype="f32"),
        # acceptance of one user's chain: the smallest call there is
        _accept("accept_chain8", batch=1, queries=8, drafts="chain", agree=0.8),
        # acceptance in a large batch of trees
        _accept("accept_trees", batch=256, queries=40, drafts="tree40", agree=0.7, ragged=True),
        # the accepted rows of four trees in one layer
        _commit("commit_layer", layers=1, batch=4, drafts="tree40", queries=40, capacity=4096),
        # the accepted rows of a batch of trees in every layer of a model
        _commit("commit_layers", layers=32, batch=16, drafts="tree40", queries=40, capacity=1024),
    ]


RULES = {  # temperature, top_k (0: all), top_p, min_p; a batch takes them in turn
    "temperature": [(0.9, 0, 1.0, 0.0)],
    "nucleus": [(0.8, 0, 0.95, 0.0)],
    "topk": [(1.0, 50, 1.0, 0.0), (0.7, 200, 0.9, 0.0)],
    "minp": [(1.2, 0, 1.0, 0.05)],
    "greedy": [(0.0, 0, 1.0, 0.0)],
    "mixed": [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.95, 0.0), (0.7, 40, 0.9, 0.02), (0.0, 0, 1.0, 0.0), (1.5, 1000, 0.99, 0.001)],
}


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _seconds(case):
    """A rough time of one pass, to keep drawn cases within the listed ones."""
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / (0.8e15 if case.get("dtype") == "bf16" else 0.03e15)


def draw(rng):
    """One more case of the same ranges, every operator in turn of chance."""
    op = rng.choices(["prefix", "sample", "accept", "commit"], [5, 3, 1, 2])[0]
    drafts, queries = "chain", _log_uniform(rng, 1, 64)
    if rng.random() < 0.35:
        drafts = rng.choice(sorted(FANOUTS))
        queries = len(_tree(drafts))
    shape = rng.choice([("bf16", 192, 128, 64, 4), ("bf16", 128, 128, 32, 4), ("bf16", 128, 128, 16, 8), ("bf16", 64, 64, 32, 8), ("f32", 64, 64, 8, 2)])
    dtype, d_k, d_v, heads, kv_heads = shape
    if op == "prefix":
        n_prefix = rng.choice([1, 1, 1, 2, 3])
        case = _prefix(None, batch=n_prefix * _log_uniform(rng, 1, 32 // n_prefix), queries=queries, prefix=_log_uniform(rng, 64, 32768),
                       suffix=_log_uniform(rng, 1, 2048), n_prefix=n_prefix, heads=heads, kv_heads=kv_heads, d_k=d_k, d_v=d_v, dtype=dtype,
                       drafts=drafts, ragged=rng.random() < 0.3)
        limit = 0.9 * max(_seconds(c) for c in listed() if c["op"] == "prefix")
        while _seconds(case) > limit or case["batch"] * case["queries"] * heads * (case["prefix"] + 2048) > 1.2e9:
            case = {**case, "prefix": case["prefix"] // 2 + 1}
        return case
    if op == "sample":
        case = _sample(None, batch=_log_uniform(rng, 1, 64), queries=min(16, queries), vocab=_log_uniform(rng, 1000, 131072),
                       rule=rng.choice(sorted(RULES)), dtype=rng.choice(["bf16", "bf16", "f32"]), masked=rng.choice([0.0, 0.0, 0.9]),
                       ragged=rng.random() < 0.3)
        while case["batch"] * case["queries"] * case["vocab"] > 5e7:
            case = {**case, "batch": case["batch"] // 2 + 1, "vocab": case["vocab"] // 2 + 1}
        return case
    if op == "accept":
        return _accept(None, batch=_log_uniform(rng, 1, 256), queries=queries, drafts=drafts, agree=rng.choice([0.5, 0.7, 0.9]), ragged=rng.random() < 0.5)
    drafts = rng.choice(sorted(FANOUTS))
    case = _commit(None, layers=_log_uniform(rng, 1, 32), batch=_log_uniform(rng, 1, 32), drafts=drafts, queries=len(_tree(drafts)),
                   capacity=_log_uniform(rng, 256, 4096), kv_heads=kv_heads, d_k=d_k, d_v=d_v, dtype=dtype)
    while case["layers"] * case["batch"] * case["capacity"] * kv_heads * (d_k + d_v) > 6e8:
        case = {**case, "capacity": max(128, case["capacity"] // 2), "layers": max(1, case["layers"] * 3 // 4)}
    return case


# ---- what a case holds besides values: trees, lengths, counts ---------------------------------------------------------
def _tree(drafts):
    """Parents of a tree of the given fan-outs, breadth first; -1: child of the last committed token."""
    parents, level = [], [-1]
    for f in FANOUTS[drafts]:
        first = len(parents)
        parents += [p for p in level for _ in range(f)]
        level = range(first, len(parents))
    return parents


def _depths(parents):
    depth = []
    for p in parents:
        depth.append(0 if p < 0 else depth[p] + 1)
    return depth


def _parents(case):
    return list(range(-1, case["queries"] - 1)) if case["drafts"] == "chain" else _tree(case["drafts"])


def _spread(n, lo, hi):
    """n whole numbers over [lo, hi] in no order, the first of them hi."""
    return [hi - int((hi - lo + 1) * ((k * 0.6180339887498949) % 1.0)) for k in range(n)]


def _prefix_lens(case):
    return _spread(case["n_prefix"], (case["prefix"] + 1) // 2, case["prefix"])


def _seq_lens(case):
    return _spread(case["batch"], 0, case["suffix"])


def _n_query(case):
    return _spread(case["batch"], (case["queries"] + 1) // 2, case["queries"]) if case.get("ragged") else [case["queries"]] * case["batch"]


def _accepted(case):
    depth = max(_depths(_parents(case))) + 1
    return _spread(case["batch"], 0, depth)


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    """Every input that is used read once, every output written once; the products of visible pairs."""
    b, t = case["batch"], case["queries"]
    if case["op"] == "prefix":
        depth = _depths(_parents(case))
        nq, lens, plens = _n_query(case), _seq_lens(case), _prefix_lens(case)
        d, per = case["d_k"] + case["d_v"], b // case["n_prefix"]
        pairs = sum(plens[k // per] + lens[k] + depth[i] + 1 for k in range(b) for i in range(nq[k]))
        rows = sum(plens) + sum(lens) + sum(nq)
        return {"bytes": rows * case["kv_heads"] * d * _elem(case) + b * t * case["heads"] * d * _elem(case),
                "flops": 2 * pairs * case["heads"] * d}
    if case["op"] == "sample":
        rows = sum(_n_query(case))
        return {"bytes": rows * case["vocab"] * _elem(case) + b * t * 12, "flops": rows * case["vocab"] * 20}
    if case["op"] == "accept":
        return {"bytes": b * t * 16 + b * 24, "flops": b * t}
    parents, per = _parents(case), _accepted(case)
    moved = sum(max(0, n - (1 if n and k % 2 == 0 else 0)) for k, n in enumerate(per))     # (half the first tokens are in place)
    return {"bytes": 2 * moved * case["layers"] * case["kv_heads"] * (case["d_k"] + case["d_v"]) * _elem(case) + b * len(parents) * 4, "flops": 0}


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case, "op": case["op"], **{"prefix": _prepare_prefix, "sample": _prepare_sample, "accept": _prepare_accept, "commit": _prepare_commit}[case["op"]](case, g)}
    if own:
        s["call"] = {"prefix": _own_prefix, "sample": _own_sample, "accept": _own_accept, "commit": _own_commit}[case["op"]](s)
    return s


def _prepare_prefix(case, g):
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    b, t, hk, n = case["batch"], case["queries"], case["kv_heads"], case["n_prefix"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)

    k_prefix, v_prefix = normal(n, hk, case["prefix"], case["d_k"]), normal(n, hk, case["prefix"], case["d_v"])
    k, v = normal(b, hk, case["suffix"] + t, case["d_k"]), normal(b, hk, case["suffix"] + t, case["d_v"])
    # queries with a direction of their sequence in common, long enough that some keys stand out
    q = (1.5 * (0.7 * torch.randn((b, 1, case["heads"], case["d_k"]), generator=g, device="cuda")
                + 0.7 * torch.randn((b, t, case["heads"], case["d_k"]), generator=g, device="cuda"))).to(dt)
    return {"q": q, "k_prefix": k_prefix, "v_prefix": v_prefix, "k": k, "v": v, "prefix_lens": _ints(_prefix_lens(case)),
            "seq_lens": _ints(_seq_lens(case)), "n_query": _ints(_n_query(case)),
            "parents": None if case["drafts"] == "chain" else _ints([_parents(case)] * b)}


def _prepare_sample(case, g):
    b, t, n = case["batch"], case["queries"], case["vocab"]
    z = torch.randn((b, t, n), generator=g, device="cuda")
    x = 2.0 * z + 0.5 * z.clamp_min(0.0) ** 2            # a bulk, and a tail of likely tokens
    if case["masked"]:
        x = torch.where(torch.rand((b, t, n), generator=g, device="cuda") < case["masked"], -math.inf, x)
    rules = [RULES[case["rule"]][k % len(RULES[case["rule"]])] for k in range(b)]
    columns = [torch.tensor([r[c] for r in rules], dtype=torch.int32 if c == 1 else torch.float32, device="cuda") for c in range(4)]
    return {"logits": x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32), "temperature": columns[0], "top_k": columns[1],
            "top_p": columns[2], "min_p": columns[3], "u": torch.rand((b, t), generator=g, device="cuda"), "n_query": _ints(_n_query(case))}


def _prepare_accept(case, g):
    b, t, parents = case["batch"], case["queries"], _parents(case)
    draft = torch.randint(0, 32000, (b, t), generator=g, device="cuda")
    other = torch.randint(0, 32000, (b, t + 1), generator=g, device="cuda")
    says_so = torch.rand((b, t + 1), generator=g, device="cuda") < case["agree"]
    children = [[c for c in range(t) if parents[c] == p] for p in range(-1, t)]
    width = max(len(c) for c in children)
    table = torch.tensor([[c[k % len(c)] if c else -1 for k in range(width)] for c in children], device="cuda")      # [t + 1, width]
    pick = torch.randint(0, width, (b, t + 1), generator=g, device="cuda")
    child = table.expand(b, -1, -1).gather(2, pick[..., None])[..., 0]
    target = torch.where(says_so & (child >= 0), draft.gather(1, child.clamp_min(0)), other).int()
    return {"draft": draft.int(), "root": target[:, 0].contiguous(), "sampled": target[:, 1:].contiguous(),
            "seq_lens": torch.randint(0, 131072, (b,), generator=g, device="cuda").int(), "n_query": _ints(_n_query(case)),
            "parents": None if case["drafts"] == "chain" else _ints([parents] * b)}


def _prepare_commit(case, g):
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    b, t, hk, cap, parents = case["batch"], case["queries"], case["kv_heads"], case["capacity"], _parents(case)
    k = torch.randn((case["layers"], b, hk, cap, case["d_k"]), generator=g, device="cuda").to(dt)
    v = torch.randn((case["layers"], b, hk, cap, case["d_v"]), generator=g, device="cuda").to(dt)
    counts = _accepted(case)
    pick = torch.randint(0, 1 << 20, (b, t), generator=g, device="cuda").tolist()
    path = []
    for n in range(b):
        at, row = -1, []
        for depth in range(counts[n]):
            children = [c for c in range(t) if parents[c] == at]
            at = children[0 if depth == 0 and n % 2 == 0 else pick[n][depth] % len(children)]
            row.append(at)
        path.append(row + [-1] * (t - len(row)))
    lens = torch.randint(cap // 2, cap - t + 1, (b,), generator=g, device="cuda").int()
    return {"k": k, "v": v, "path": _ints(path), "n_accepted": _ints(counts), "seq_lens": lens}


# ---- the calls that a user makes ----------------------------------------------------------------------------------------
def _own_prefix(s):
    from paper_2605_19893_amd import binding as B
    case, q = s["case"], s["q"]
    p = B.make_prefix_params(B=case["batch"], T=case["queries"], H=case["heads"], H_kv=case["kv_heads"], d_k=case["d_k"], d_v=case["d_v"],
                             n_prefix=case["n_prefix"], dtype=B.SSV_BF16 if case["dtype"] == "bf16" else B.SSV_F32, max_prefix_len=case["prefix"],
                             max_seq_len=case["suffix"], kp_stride=s["k_prefix"].stride()[:3], vp_stride=s["v_prefix"].stride()[:3],
                             k_stride=s["k"].stride()[:3], v_stride=s["v"].stride()[:3])
    need = B.ssv_prefix_workspace_bytes(p)
    out = torch.empty((*q.shape[:3], case["d_v"]), dtype=q.dtype, device=q.device)
    space = torch.empty(need, dtype=torch.uint8, device=q.device)

    def call():
        B.ssv_prefix_verify(q, s["k_prefix"], s["v_prefix"], s["k"], s["v"], s["prefix_lens"], s["seq_lens"], s["n_query"], s["parents"], p,
                            out, space, need, torch.cuda.current_stream().cuda_stream)
        return {"out": out}
    return call


def _own_sample(s):
    from paper_2605_19893_amd import binding as B
    case, x = s["case"], s["logits"]
    p = B.make_sample_params(B=case["batch"], T=case["queries"], V=case["vocab"], dtype=B.SSV_BF16 if case["dtype"] == "bf16" else B.SSV_F32,
                             logits_stride=x.stride()[:2])
    need = B.ssv_sample_workspace_bytes(p)
    tokens = torch.empty(x.shape[:2], dtype=torch.int32, device=x.device)
    probs = torch.empty(x.shape[:2], dtype=torch.float32, device=x.device)
    space = torch.empty(need, dtype=torch.uint8, device=x.device)

    def call():
        B.ssv_sample(x, s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"], s["n_query"], p, tokens, probs, space, need,
                     torch.cuda.current_stream().cuda_stream)
        return {"tokens": tokens, "probs": probs}
    return call


def _own_accept(s):
    from paper_2605_19893_amd import binding as B
    b, t = s["draft"].shape
    path = torch.empty((b, t), dtype=torch.int32, device="cuda")
    counts, following, lens = (torch.empty(b, dtype=torch.int32, device="cuda") for _ in range(3))

    def call():
        B.ssv_accept(s["draft"], s["root"], s["sampled"], s["seq_lens"], s["n_query"], s["parents"], b, t, path, counts, following, lens,
                     torch.cuda.current_stream().cuda_stream)
        return {"path": path, "n_accepted": counts, "next": following, "committed": lens}
    return call


def _own_commit(s):
    from paper_2605_19893_amd import binding as B
    case, k, v = s["case"], s["k"], s["v"]
    p = B.make_commit_params(layers=case["layers"], B=case["batch"], T=case["queries"], H_kv=case["kv_heads"], d_k=case["d_k"], d_v=case["d_v"],
                             dtype=B.SSV_BF16 if case["dtype"] == "bf16" else B.SSV_F32, kv_capacity=case["capacity"],
                             k_stride=k.stride()[:4], v_stride=v.stride()[:4])

    def call():
        B.ssv_commit(k, v, s["path"], s["n_accepted"], s["seq_lens"], p, torch.cuda.current_stream().cuda_stream)
        return {"k": k, "v": v}
    return call


# ---- the plain forms ----------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return s["call"]()
    return {"prefix": _plain_prefix, "sample": _plain_sample, "accept": _plain_accept, "commit": _plain_commit}[s["op"]](s)


def _ancestors(parents, b, t):
    """[b, t, t] truth values: draft token j is i or an ancestor of i."""
    if parents is None:
        return torch.ones((b, t, t), dtype=torch.bool, device="cuda").tril()
    step = (parents[:, :, None] == torch.arange(t, device="cuda")).double() + torch.eye(t, dtype=torch.float64, device="cuda")
    return torch.linalg.matrix_power(step, t) > 0


def _plain_prefix(s):
    case = s["case"]
    b, t, h, hk, dk, dv, n = (case[x] for x in ("batch", "queries", "heads", "kv_heads", "d_k", "d_v", "n_prefix"))
    hg, per = h // hk, b // n
    q = s["q"].float().reshape(b, t, hk, hg, dk).permute(0, 2, 1, 3, 4).reshape(b, hk, t * hg, dk) / math.sqrt(dk)
    stacked = q.reshape(n, per, hk, t * hg, dk).transpose(1, 2).reshape(n * hk, per * t * hg, dk)
    kp = s["k_prefix"].float().transpose(2, 3).reshape(n * hk, dk, -1).contiguous()
    vp = s["v_prefix"].float().reshape(n * hk, -1, dv)
    sp = torch.bmm(stacked, kp)
    ended = torch.arange(sp.shape[2], device="cuda") >= s["prefix_lens"].repeat_interleave(hk)[:, None]
    sp = sp.masked_fill_(ended[:, None, :], -math.inf)
    own_slots = torch.arange(s["k"].shape[2], device="cuda")
    at = own_slots[None, :] - s["seq_lens"][:, None]                                   # draft token of a slot; negative: committed
    drafted = _ancestors(s["parents"], b, t).gather(2, at.clamp(0, t - 1)[:, None, :].expand(b, t, -1).long())
    seen = (at < 0)[:, None, :] | (drafted & (at < t)[:, None, :])
    ss = torch.bmm(q.reshape(b * hk, t * hg, dk), s["k"].float().transpose(2, 3).reshape(b * hk, dk, -1).contiguous())
    ss = ss.reshape(b, hk, t, hg, -1).masked_fill(~seen[:, None, :, None, :], -math.inf).reshape(b * hk, t * hg, -1)
    top = torch.maximum(sp.amax(2).reshape(n, hk, per, t * hg).transpose(1, 2).reshape(b * hk, t * hg), ss.amax(2))
    wide = top.reshape(n, per, hk, t * hg).transpose(1, 2).reshape(n * hk, per * t * hg)
    sp = sp.sub_(wide[..., None]).exp_()
    ss = (ss - top[..., None]).exp()
    # rows of V that nobody sees may hold anything
    vp = vp.masked_fill(ended[..., None], 0.0)
    vs = s["v"].float().masked_fill((at >= t)[:, None, :, None], 0.0).reshape(b * hk, -1, dv)
    far = torch.bmm(sp, vp).reshape(n, hk, per, t * hg, dv).transpose(1, 2).reshape(b * hk, t * hg, dv)
    total = sp.sum(2).reshape(n, hk, per, t * hg).transpose(1, 2).reshape(b * hk, t * hg) + ss.sum(2)
    out = (far + torch.bmm(ss, vs)) / total[..., None]
    out = out.reshape(b, hk, t, hg, dv).permute(0, 2, 1, 3, 4).reshape(b, t, h, dv)
    asked = torch.arange(t, device="cuda") < s["n_query"][:, None]
    return {"out": out.masked_fill(~asked[..., None, None], 0.0).to(s["q"].dtype)}


def _plain_sample(s):
    x = s["logits"].double()
    n = x.shape[2]
    t, top_k, top_p, min_p = (s[c][:, None, None] for c in ("temperature", "top_k", "top_p", "min_p"))
    top = x.amax(2, keepdim=True)
    w = ((x - top) / torch.where(t > 0, t, 1.0).double()).exp()
    ws, order = x.sort(dim=2, descending=True, stable=True)
    ws = w.gather(2, order)
    rank = torch.arange(n, device="cuda")
    by_k = (rank < top_k) | (top_k <= 0)
    upto = (ws * by_k).cumsum(2)
    by_p = (upto - ws < top_p.double() * upto[..., -1:]) | (top_p >= 1)
    keep = by_k & by_p & (ws >= min_p.double()) & ((t > 0) | (rank == 0))
    kept = w * torch.zeros_like(keep).scatter(2, order, keep)
    upto = kept.cumsum(2)
    token = (upto <= s["u"].double()[..., None] * upto[..., -1:]).sum(2).clamp_max(n - 1)
    prob = kept.gather(2, token[..., None])[..., 0] / upto[..., -1]
    asked = torch.arange(x.shape[1], device="cuda") < s["n_query"][:, None]
    return {"tokens": torch.where(asked, token, -1).int(), "probs": torch.where(asked, prob, 0.0).float()}


def _plain_accept(s):
    b, t = s["draft"].shape
    index = torch.arange(t, device="cuda")
    parents = (index - 1).expand(b, t) if s["parents"] is None else s["parents"].long()
    asked = index < s["n_query"][:, None]
    says = torch.cat([s["root"][:, None], s["sampled"]], 1).gather(1, parents + 1)       # what the parent's sample says
    match = (s["draft"] == says) & asked
    twin = (parents[:, :, None] == parents[:, None, :]) & match[:, None, :] & (index < index[:, None])     # an earlier sibling that matches
    fine = match & ~twin.any(2)
    ok = torch.bmm(_ancestors(s["parents"], b, t).float(), (~fine).float()[..., None])[..., 0] == 0
    counts = ok.sum(1)
    path = torch.where(ok, index, t).sort(1).values
    path = torch.where(path < t, path, -1)
    last = path.gather(1, (counts - 1).clamp_min(0)[:, None])
    following = torch.cat([s["root"][:, None], s["sampled"]], 1).gather(1, torch.where(counts[:, None] > 0, last, -1) + 1)[:, 0]
    return {"path": path.int(), "n_accepted": counts.int(), "next": following.int(), "committed": (s["seq_lens"] + counts).int()}


def _plain_commit(s):
    b, t = s["path"].shape
    step = torch.arange(t, device="cuda")
    source = torch.where(step < s["n_accepted"][:, None], s["path"], step).long() + s["seq_lens"][:, None]
    target = step + s["seq_lens"][:, None]
    which = torch.arange(b, device="cuda")[:, None]
    k, v = s["k"].transpose(2, 3), s["v"].transpose(2, 3)                                # [layer, sequence, row, head, feature]
    k[:, which, target] = k[:, which, source]
    v[:, which, target] = v[:, which, source]
    return {"k": s["k"], "v": s["v"]}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------
def exact(case, seed):
    """Attention, probabilities and moved rows by their definitions, sequence by sequence and row by row; acceptance gives
    whole numbers only."""
    if case["op"] == "prefix":
        return _exact_prefix(case, prepare(case, seed))
    if case["op"] == "sample":
        return _exact_sample(prepare(case, seed))
    if case["op"] == "commit":
        return _exact_commit(prepare(case, seed))
    return None


def _exact_prefix(case, s):
    parents, lens, plens, nq = _parents(case), _seq_lens(case), _prefix_lens(case), _n_query(case)
    b, t, h, hk = case["batch"], case["queries"], case["heads"], case["kv_heads"]
    hg = h // hk
    out = torch.zeros((b, t, h, case["d_v"]), dtype=torch.float64, device="cuda")
    lines = []
    for i in range(t):
        line, at = [], i
        while at >= 0:
            line.append(at)
            at = parents[at]
        lines.append(line)
    for n in range(b):
        p = n // (b // case["n_prefix"])
        for c in range(hk):
            keys = torch.cat([s["k_prefix"][p, c, :plens[p]], s["k"][n, c, :lens[n] + t]]).double()
            values = torch.cat([s["v_prefix"][p, c, :plens[p]], s["v"][n, c, :lens[n] + t]]).double()
            hidden = torch.ones((nq[n], keys.shape[0]), dtype=torch.bool)
            hidden[:, :plens[p] + lens[n]] = False
            for i in range(nq[n]):
                hidden[i, [plens[p] + lens[n] + a for a in lines[i]]] = False
            x = s["q"][n, :nq[n], c * hg:(c + 1) * hg].double() @ keys.T.contiguous() * case["d_k"] ** -0.5
            x = x.masked_fill(hidden.cuda()[:, None, :], -math.inf)
            out[n, :nq[n], c * hg:(c + 1) * hg] = torch.softmax(x, 2) @ values
    return {"out": out}


def _exact_sample(s):
    b, t, n = s["logits"].shape
    if b * t * n > 1 << 26:
        return None
    rules = [s[c].double().tolist() for c in ("temperature", "top_k", "top_p", "min_p")]
    u, nq = s["u"].double().tolist(), s["n_query"].tolist()
    probs = torch.zeros((b, t), dtype=torch.float64)
    for i in range(b):
        temperature, top_k, top_p, min_p = (r[i] for r in rules)
        for j in range(nq[i]):
            x = s["logits"][i, j].double()
            if temperature <= 0:
                probs[i, j] = 1.0
                continue
            first = torch.argsort(x, descending=True, stable=True)
            if top_k > 0:
                first = first[:int(top_k)]
            p = torch.softmax(x[first] / temperature, 0)
            if top_p < 1:
                enough = int((p.cumsum(0) < top_p).sum()) + 1
                first, p = first[:enough], p[:enough]
            first = first[p >= min_p * p[0]]
            chosen = first.sort().values
            p = torch.softmax(x[chosen] / temperature, 0)
            probs[i, j] = p[min(int((p.cumsum(0) <= u[i][j]).sum()), len(p) - 1)]
    return {"tokens": None, "probs": probs}


def _exact_commit(s):
    moved = {"k": s["k"].double(), "v": s["v"].double()}
    path, counts, lens = (s[x].tolist() for x in ("path", "n_accepted", "seq_lens"))
    for name, at in moved.items():
        for n, line in enumerate(path):
            for j in range(counts[n]):
                at[:, n, :, lens[n] + j] = s[name][:, n, :, lens[n] + line[j]].double()
    return moved
