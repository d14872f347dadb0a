"""Host-side checks of include/ssv_round.h (no GPU, nothing launched): exports, struct layouts, refusals; and pins of the
definitions that the GPU tests compare with."""
import ctypes
import os
import re

import numpy as np
import pytest

import round_oracle as ro
from paper_2605_19893_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P16 = 1 << 20          # an address that is aligned and never used: every call below is refused before anything is launched


def prefix_params(**over):
    kw = dict(B=4, T=8, H=64, H_kv=4, d_k=192, d_v=128, n_prefix=2, dtype=B.SSV_BF16, max_prefix_len=1000, max_seq_len=100,
              kp_stride=(4 * 1000 * 192, 1000 * 192, 192), vp_stride=(4 * 1000 * 128, 1000 * 128, 128), k_stride=(4 * 108 * 192, 108 * 192, 192),
              v_stride=(4 * 108 * 128, 108 * 128, 128))
    kw.update(over)
    return B.make_prefix_params(**kw)


def test_exports_and_struct_layouts():
    lib = B.load_library()
    with open(os.path.join(ROOT, "include", "ssv_round.h")) as f:
        header = f.read()
    code = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    assert set(re.findall(r"\b(ssv_[a-z_]+)\s*\(", code)) == set(B.ROUND_EXPORTS)
    for name in B.ROUND_EXPORTS:
        assert getattr(lib, name) is not None
    for struct, cls, size in (("ssv_prefix_params", B.SsvPrefixParams, 12 * 4 + 18 * 8), ("ssv_sample_params", B.SsvSampleParams, 4 * 4 + 2 * 8),
                              ("ssv_commit_params", B.SsvCommitParams, 8 * 4 + 8 * 8)):
        body = code[code.index("typedef struct " + struct):code.index("} " + struct + ";")]
        names = re.findall(r"\b([A-Za-z_][A-Za-z0-9_]*)\s*(?:\[\d+\])?\s*[,;]", body)
        assert names == [n for n, _ in cls._fields_]
        assert ctypes.sizeof(cls) == size


def test_prefix_accepts_what_the_library_supports():
    for dt, dk, dv in ((B.SSV_BF16, 192, 128), (B.SSV_BF16, 128, 128), (B.SSV_BF16, 64, 64), (B.SSV_F32, 64, 64)):
        for hg in (1, 2, 4, 8, 16):
            p = prefix_params(dtype=dt, d_k=dk, d_v=dv, H=4 * hg)
            assert B.ssv_prefix_workspace_bytes(p) > 0
    assert B.ssv_prefix_workspace_bytes(prefix_params(max_prefix_len=0, kp_stride=(0, 0, 0), vp_stride=(0, 0, 0))) > 0
    assert B.ssv_prefix_workspace_bytes(prefix_params(max_seq_len=0)) > 0
    assert B.ssv_prefix_workspace_bytes(prefix_params(T=128, max_prefix_len=1 << 20)) > 0


@pytest.mark.parametrize("over, code", [
    (dict(B=0), B.SSV_EINVAL), (dict(T=0), B.SSV_EINVAL), (dict(H=0), B.SSV_EINVAL), (dict(H_kv=0), B.SSV_EINVAL), (dict(H=66), B.SSV_EINVAL),
    (dict(n_prefix=0), B.SSV_EINVAL), (dict(n_prefix=3), B.SSV_EINVAL), (dict(dtype=5), B.SSV_EINVAL), (dict(scale=-1.0), B.SSV_EINVAL),
    (dict(scale=float("nan")), B.SSV_EINVAL), (dict(scale=float("inf")), B.SSV_EINVAL), (dict(max_prefix_len=-1), B.SSV_EINVAL),
    (dict(max_seq_len=-1), B.SSV_EINVAL), (dict(k_stride=(0, 0, 191)), B.SSV_EINVAL), (dict(k_stride=(0, 0, 184)), B.SSV_EINVAL),
    (dict(vp_stride=(-128, 0, 128)), B.SSV_EINVAL), (dict(q_stride=(64 * 192, 64 * 192, 8)), B.SSV_EINVAL), (dict(out_stride=(4, 4, 129)), B.SSV_EINVAL),
    (dict(T=129), B.SSV_EUNSUPPORTED), (dict(H=12), B.SSV_EUNSUPPORTED), (dict(H=128), B.SSV_EUNSUPPORTED), (dict(d_k=96), B.SSV_EUNSUPPORTED),
    (dict(dtype=B.SSV_F32), B.SSV_EUNSUPPORTED), (dict(max_seq_len=2 ** 31 - 1), B.SSV_EUNSUPPORTED), (dict(v_stride=(0, 0, 1 << 26)), B.SSV_EUNSUPPORTED),
    (dict(B=1 << 30, n_prefix=1), B.SSV_EUNSUPPORTED)])
def test_prefix_refusals(over, code):
    p = prefix_params(**over)
    assert B.ssv_prefix_workspace_bytes(p) == 0
    with pytest.raises(B.SsvError) as e:
        B.ssv_prefix_verify(P16, P16, P16, P16, P16, P16, P16, None, None, p, P16, P16, 1 << 40, 0)
    assert e.value.code == code


def test_prefix_refuses_pointers_and_workspaces():
    p = prefix_params()
    need = B.ssv_prefix_workspace_bytes(p)

    def refused(args, ws=P16, size=need, prm=p):
        with pytest.raises(B.SsvError) as e:
            B.ssv_prefix_verify(*args[:9], prm, args[9], ws, size, 0)
        return e.value.code

    good = [P16] * 7 + [None, None, P16]
    for at in (0, 1, 2, 3, 4, 5, 6, 9):
        assert refused(good[:at] + [None] + good[at + 1:]) == B.SSV_EINVAL
    for at in (0, 1, 2, 3, 4, 9):
        assert refused(good[:at] + [P16 + 8] + good[at + 1:]) == B.SSV_EINVAL
    for at in (5, 6, 7, 8):
        assert refused(good[:at] + [P16 + 2] + good[at + 1:]) == B.SSV_EINVAL
    assert refused(good, ws=None) == refused(good, ws=P16 + 128) == refused(good, size=need - 1) == B.SSV_EWORKSPACE
    # without a prefix its pointers may be missing: the call gets as far as its workspace
    bare = prefix_params(max_prefix_len=0, kp_stride=(0, 0, 0), vp_stride=(0, 0, 0))
    assert refused([P16, None, None, P16, P16, None, P16, None, None, P16], ws=None, prm=bare) == B.SSV_EWORKSPACE


@pytest.mark.parametrize("over, code", [(dict(B=0), B.SSV_EINVAL), (dict(T=0), B.SSV_EINVAL), (dict(V=0), B.SSV_EINVAL), (dict(dtype=2), B.SSV_EINVAL),
                                        (dict(logits_stride=(-1, 0)), B.SSV_EINVAL), (dict(V=B.SSV_SAMPLE_MAX_V + 1), B.SSV_EUNSUPPORTED),
                                        (dict(B=1 << 20, T=1 << 20), B.SSV_EUNSUPPORTED)])
def test_sample_refusals(over, code):
    kw = dict(B=2, T=3, V=100, dtype=B.SSV_F32)
    kw.update(over)
    with pytest.raises(B.SsvError) as e:
        B.ssv_sample(P16, None, None, None, None, P16, None, B.make_sample_params(**kw), P16, None, P16, 1 << 40, 0)
    assert e.value.code == code


def test_sample_refuses_pointers():
    for dt, odd in ((B.SSV_F32, 2), (B.SSV_BF16, 1)):
        p = B.make_sample_params(B=2, T=3, V=100, dtype=dt)
        good = [P16, None, None, None, None, P16, None, p, P16, None]
        for at, bad in [(0, None), (5, None), (8, None), (0, P16 + odd)] + [(a, P16 + 2) for a in (1, 2, 3, 4, 5, 6, 8, 9)]:
            args = list(good)
            args[at] = bad
            with pytest.raises(B.SsvError) as e:
                B.ssv_sample(*args, P16, 1 << 40, 0)
            assert e.value.code == B.SSV_EINVAL


def test_sample_refuses_workspaces():
    for V in (1, 2041, 2042, 100003, B.SSV_SAMPLE_MAX_V):
        p = B.make_sample_params(B=2, T=3, V=V, dtype=B.SSV_F32)
        need = B.ssv_sample_workspace_bytes(p)
        assert need > 0
        for ws, size in ((None, need), (P16 + 128, need), (P16, need - 1)):
            with pytest.raises(B.SsvError) as e:
                B.ssv_sample(P16, None, None, None, None, P16, None, p, P16, None, ws, size, 0)
            assert e.value.code == B.SSV_EWORKSPACE
    assert B.ssv_sample_workspace_bytes(B.make_sample_params(B=0, T=3, V=8, dtype=B.SSV_F32)) == 0


def test_accept_refusals():
    def code(B_=2, T=3, at=None, to=None):
        args = [P16] * 6 + [B_, T] + [P16] * 4
        if at is not None:
            args[at] = to
        with pytest.raises(B.SsvError) as e:
            B.ssv_accept(*args, 0)
        return e.value.code

    assert code(B_=0) == code(T=0) == B.SSV_EINVAL and code(T=129) == B.SSV_EUNSUPPORTED
    for at in (0, 1, 2, 3, 8, 9, 10, 11):
        assert code(at=at, to=None) == B.SSV_EINVAL
    for at in (0, 1, 2, 3, 4, 5, 8, 9, 10, 11):
        assert code(at=at, to=P16 + 2) == B.SSV_EINVAL


@pytest.mark.parametrize("over, code", [(dict(layers=0), B.SSV_EINVAL), (dict(B=0), B.SSV_EINVAL), (dict(T=0), B.SSV_EINVAL), (dict(H_kv=0), B.SSV_EINVAL),
                                        (dict(d_k=4), B.SSV_EINVAL), (dict(d_v=0), B.SSV_EINVAL), (dict(dtype=9), B.SSV_EINVAL), (dict(kv_capacity=-1), B.SSV_EINVAL),
                                        (dict(k_stride=(0, 0, 0, 56)), B.SSV_EINVAL), (dict(v_stride=(0, 4, 0, 64)), B.SSV_EINVAL),
                                        (dict(v_stride=(-64, 0, 0, 64)), B.SSV_EINVAL), (dict(T=129), B.SSV_EUNSUPPORTED),
                                        (dict(layers=1 << 20, B=1 << 20), B.SSV_EUNSUPPORTED)])
def test_commit_refusals(over, code):
    kw = dict(layers=2, B=2, T=8, H_kv=2, d_k=64, d_v=64, dtype=B.SSV_BF16, kv_capacity=100, k_stride=(25600, 12800, 6400, 64), v_stride=(25600, 12800, 6400, 64))
    kw.update(over)
    with pytest.raises(B.SsvError) as e:
        B.ssv_commit(P16, P16, P16, P16, P16, B.make_commit_params(**kw), 0)
    assert e.value.code == code


def test_commit_refuses_pointers():
    p = B.make_commit_params(layers=1, B=2, T=8, H_kv=2, d_k=64, d_v=64, dtype=B.SSV_BF16, kv_capacity=100, k_stride=(0, 12800, 6400, 64),
                             v_stride=(0, 12800, 6400, 64))
    for at in range(5):
        for bad in (None, P16 + 2):
            args = [P16] * 5
            args[at] = bad
            with pytest.raises(B.SsvError) as e:
                B.ssv_commit(*args, p, 0)
            assert e.value.code == B.SSV_EINVAL


# ---- pins of the definitions ------------------------------------------------------------------------------------------
def test_definition_of_sampling():
    x = np.log([0.4, 0.1, 0.2, 0.3])
    assert [ro.sample(x, 1, 0, 1, 0, u)[0] for u in (0.0, 0.39, 0.41, 0.49, 0.51, 0.69, 0.71, 0.99)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [ro.sample(x, 1, 2, 1, 0, u)[0] for u in (0.0, 0.57, 0.58, 0.99)] == [0, 0, 3, 3]
    assert abs(ro.sample(x, 1, 2, 1, 0, 0.9)[1] - 0.3 / 0.7) < 1e-12
    assert [ro.sample(x, 1, 0, 0.71, 0, u)[0] for u in (0.45, 0.9)] == [2, 3]           # 0.4 + 0.3 < 0.71: three kept
    assert ro.sample(x, 1, 2, 0.5, 0, 0.99)[0] == 0                                    # 0.4 of 0.7 is over one half
    assert [ro.sample(x, 1, 0, 1, 0.6, u)[0] for u in (0.5, 0.9)] == [0, 3]             # 0.3 / 0.4 >= 0.6 > 0.2 / 0.4
    assert ro.sample(x, 0.5, 0, 1, 0, 0.0)[1] == pytest.approx(0.16 / 0.30)
    assert ro.sample([1.0, 3.0, 3.0], 0, 0, 1, 0, 0.9)[:2] == (1, 1.0)
    assert ro.sample([-np.inf] * 3, 1, 0, 1, 0, 0.5)[0] == -1


def test_definition_of_acceptance_and_commit():
    par = [-1, -1, 0, 0, 1]
    assert ro.accept([5, 6, 7, 7, 8], 5, [7, 0, 9, 1, 0], 10, 5, par) == ([0, 2], 9, 12)
    assert ro.accept([5, 6, 7, 7, 8], 6, [7, 8, 9, 1, 3], 10, 5, par) == ([1, 4], 3, 12)
    assert ro.accept([5, 6, 7, 7, 8], 4, [7, 8, 9, 1, 3], 10, 5, par) == ([], 4, 10)
    assert ro.accept([5, 6, 7, 7, 8], 6, [7, 8, 9, 1, 3], 10, 4, par) == ([1], 8, 11)
    rows = np.arange(10)[:, None]
    assert ro.commit(rows, [1, 3], 2, 4, 5, 10)[:, 0].tolist() == [0, 1, 2, 3, 5, 7, 6, 7, 8, 9]


def test_definition_of_attention_equals_one_softmax_over_all_rows():
    rng = np.random.default_rng(0)
    q, kp, vp = rng.normal(size=(2, 2, 2, 4)), rng.normal(size=(1, 1, 5, 4)), rng.normal(size=(1, 1, 5, 3))
    k, v = rng.normal(size=(2, 1, 6, 4)), rng.normal(size=(2, 1, 6, 3))
    out, mass, _ = ro.prefix_attention(q, kp, vp, k, v, [5], [3, 0], [2, 1], None, 0.5)
    keys, vals = np.concatenate([kp[0, 0], k[0, 0, :5]]), np.concatenate([vp[0, 0], v[0, 0, :5]])
    p = np.exp(0.5 * q[0, 1, 1] @ keys.T)
    assert np.allclose(out[0, 1, 1], p @ vals / p.sum())
    assert (out[1, 1] == 0).all() and (mass >= np.abs(out) - 1e-12).all()


@pytest.mark.parametrize("over, code", [
    (dict(out_stride=(0, 64 * 128, 128)), B.SSV_EINVAL), (dict(out_stride=(8 * 64 * 128, 0, 128)), B.SSV_EINVAL),
    (dict(B=1 << 14, T=128, n_prefix=1), B.SSV_EUNSUPPORTED), (dict(B=1 << 18, T=1, n_prefix=1 << 18), B.SSV_EUNSUPPORTED)])
def test_prefix_refuses_repeated_rows_and_launches_beyond_32_bits(over, code):
    test_prefix_refusals(over, code)


def test_prefix_accepts_broadcast_inputs():
    for over in (dict(k_stride=(0, 0, 192), v_stride=(0, 0, 128)), dict(kp_stride=(0, 0, 192), vp_stride=(0, 0, 128)), dict(q_stride=(0, 0, 192)),
                 dict(B=1, n_prefix=1, T=1, out_stride=(0, 0, 128))):
        assert B.ssv_prefix_workspace_bytes(prefix_params(**over)) > 0


def test_launches_beyond_32_bits_are_refused():
    """The threads of a launch are counted in 32 bits."""
    assert B.ssv_sample_workspace_bytes(B.make_sample_params(B=(1 << 23) - 1, T=1, V=1, dtype=B.SSV_F32)) > 0
    test_sample_refusals(dict(B=1 << 23, T=1, V=1), B.SSV_EUNSUPPORTED)
    test_sample_refusals(dict(B=1 << 21, T=1, V=60000), B.SSV_EUNSUPPORTED)
    with pytest.raises(B.SsvError) as e:
        B.ssv_accept(*[P16] * 6, 1 << 26, 3, *[P16] * 4, 0)
    assert e.value.code == B.SSV_EUNSUPPORTED
    test_commit_refusals(dict(layers=1 << 12, B=1 << 10, H_kv=1 << 6), B.SSV_EUNSUPPORTED)


@pytest.mark.parametrize("at", [0, 1, 2])
def test_commit_refuses_caches_at_one_place(at):
    good = (25600, 12800, 6400, 64)
    test_commit_refusals(dict(k_stride=good[:at] + (0,) + good[at + 1:]), B.SSV_EINVAL)
    test_commit_refusals(dict(v_stride=good[:at] + (0,) + good[at + 1:]), B.SSV_EINVAL)


def test_prefix_refuses_scales_below_2_to_the_minus_100():
    assert B.ssv_prefix_workspace_bytes(prefix_params(scale=2.0 ** -100)) > 0
    test_prefix_refusals(dict(scale=2.0 ** -101), B.SSV_EUNSUPPORTED)
    test_prefix_refusals(dict(scale=1e-40), B.SSV_EUNSUPPORTED)


def test_prefix_refuses_scales_above_2_to_the_100():
    """A scale whose product with log2(e) is not finite made every row a NaN."""
    assert B.ssv_prefix_workspace_bytes(prefix_params(scale=2.0 ** 100)) > 0
    test_prefix_refusals(dict(scale=2.0 ** 100 * (1 + 2.0 ** -23)), B.SSV_EUNSUPPORTED)
    test_prefix_refusals(dict(scale=2.5e38), B.SSV_EUNSUPPORTED)
    test_prefix_refusals(dict(scale=3.4e38), B.SSV_EUNSUPPORTED)


@pytest.mark.parametrize("over", [dict(B=8192, H=8, H_kv=8), dict(B=1 << 16, H=8, H_kv=8), dict(B=8192, H=8, H_kv=8, n_prefix=8192), dict(B=8192, H=64, H_kv=8, T=16),
                                  dict(B=1 << 16, H=8, H_kv=8, max_prefix_len=100000, max_seq_len=100000)])
def test_prefix_accepts_many_sequences(over):
    """Up to 2^19 sequences times KV heads: what counts is the launch that the call makes, not the one with the most slices."""
    kw = dict(T=1, n_prefix=1, d_k=64, d_v=64, kp_stride=(0, 0, 64), vp_stride=(0, 0, 64), k_stride=(0, 0, 64), v_stride=(0, 0, 64))
    kw.update(over)
    assert B.ssv_prefix_workspace_bytes(prefix_params(**kw)) > 0
    test_prefix_refusals({**kw, "B": kw["B"] * 64, "n_prefix": kw["n_prefix"] * 64}, B.SSV_EUNSUPPORTED)
