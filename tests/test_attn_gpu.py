"""Token attention on the GPU against the fp64 oracle: forward and gradients (tests/_attn.py has
the cases and derives the bounds)."""
import numpy as np
import pytest
import torch

import _attn
from oracle import operators_oracle as orc

pytestmark = pytest.mark.gpu

# B, H, Hkv, Gq, Gk, d
SIZES = [(1, 1, 1, 1, 1, 32), (1, 2, 1, 2, 2, 16), (2, 2, 2, 3, 3, 64), (1, 8, 8, 32, 32, 32), (2, 2, 2, 15, 15, 32),
         (2, 4, 2, 17, 17, 16), (1, 2, 1, 31, 31, 64), (1, 2, 2, 63, 63, 32), (1, 4, 4, 64, 64, 16), (3, 4, 2, 100, 100, 64),
         (1, 3, 3, 65, 65, 32), (1, 2, 1, 129, 129, 32), (1, 8, 2, 130, 130, 32), (1, 1, 1, 257, 257, 64),
         (1, 2, 2, 300, 300, 16), (2, 8, 2, 1, 700, 32), (1, 4, 1, 5, 1000, 64), (1, 2, 2, 40, 33, 32), (2, 4, 1, 1, 1, 32),
         # at least 128 rows and keys and 1.5 million pairs: tiles of 128 rows on tcgen05; several heads in a tile, one
         # tile, many, ragged ones, more queries than keys
         *[(*z, d) for z in ((1, 16, 4, 100, 1000), (1, 8, 8, 440, 440), (1, 8, 8, 600, 330), (12, 8, 8, 128, 128),
                             (2, 8, 2, 129, 760), (1, 1, 1, 1300, 1301), (1, 16, 1, 33, 3000)) for d in (32, 16, 64)],
         # just below: the same shapes by warps
         (1, 4, 1, 40, 300, 32), (2, 2, 2, 256, 256, 32), (1, 2, 2, 600, 129, 32)]
PLAIN = [dict(), dict(cap=5.0), dict(bias="index"), dict(bias="place", cap=2.0), dict(docs=2), dict(prefix=0),
         dict(prefix=1, bias="index"), dict(docs=3, prefix=1, cap=3.0, bias="place")]


@pytest.mark.parametrize("what", PLAIN, ids=lambda w: "-".join(f"{k}{v}" for k, v in w.items()) or "plain")
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_oracle(lib, size, what):
    if what.get("prefix") is not None and size[3] > size[4]:
        pytest.skip("the prefix mask has no more queries than keys")
    _attn.check(lib, _attn.make(sum(size), *size, **what))


@pytest.mark.parametrize("d", [16, 32, 64])
def test_large_scores(lib, d):
    """Scores of some tens, capped and not: the running maximum moves by much from tile to tile."""
    for cap in (0.0, 10.0):
        for H, G in ((2, 200), (4, 640)):
            c = _attn.make(d, 1, H, H, G, G, d, cap=cap)
            c["q"] *= 4
            c["k"] *= 3
            _attn.check(lib, c)


@pytest.mark.parametrize("scale", [-0.3, 0.0])
@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_negative_and_zero_scale(lib, scale, cap):
    for G in (50, 640):
        _attn.check(lib, {**_attn.make(G, 1, 4, 4, G, G, 32, cap=cap), "scale": scale})


def test_any_negative_document_is_none(lib):
    """Unused tokens see nothing, whatever negative numbers they carry."""
    for G in (60, 650):
        c = _attn.make(G, 2, 2, 2, G, G, 32, docs=2)
        rng = np.random.default_rng(G)
        for n in ("doc_q", "doc_k"):
            t = c["mask"][n]
            t[t < 0] = rng.choice([-1, -2, -(2 ** 31)], (t < 0).sum())
        got = _attn.check(lib, c)
        assert (got["lse"][np.broadcast_to((c["mask"]["doc_q"] < 0)[:, None], got["lse"].shape)] == -np.inf).all()


def test_tiny_and_huge_magnitudes(lib):
    """fp32's exponent range: no scale is assumed."""
    for f in (1e-20, 1e18):
        for G in (70, 900):
            c = _attn.make(5, 1, 2, 2, G, G, 32)
            c["v"] *= np.float32(f)
            c["dout"] *= np.float32(1 / f)
            _attn.check(lib, c)


@pytest.mark.parametrize("d", [32, 16, 64])
@pytest.mark.parametrize("G", [90, 460])
def test_rows_that_see_nothing(lib, G, d):
    c = _attn.make(6, 2, 4, 2, G, G, d, docs=2)
    c["mask"]["doc_q"][0, :40] = -1
    c["mask"]["doc_k"][1] = -1
    got = _attn.check(lib, c)
    assert (got["out"][1] == 0).all() and (got["lse"][1] == -np.inf).all()
    assert all((got[n][1] == 0).all() for n in ("dq", "dk", "dv"))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf, 3e38, -3.4e38])
@pytest.mark.parametrize("d", [16, 32, 64])
def test_what_masked_tokens_hold_reaches_no_result(lib, d, bad):
    """Documents: tokens of document 1 and unused ones hold `bad`; document 0's results are those
    of clean tokens."""
    for prefix, G in ((None, 150), (1, 150), (None, 460), (1, 460)):
        c = _attn.make(7, 2, 4, 2, G, G, d, docs=2, cap=4.0, bias="place", prefix=prefix)
        c["mask"]["doc_q"] = c["mask"]["doc_k"].copy()
        other = c["mask"]["doc_k"] != 0
        clean = {n: t.copy() for n, t in c.items() if n in ("q", "k", "v", "dout")}
        for n in ("q", "k", "v", "dout"):
            c[n][np.broadcast_to(other[:, None], c[n].shape[:3])] = bad
            clean[n][np.broadcast_to(other[:, None], c[n].shape[:3])] = 0
        got, ref = _attn.run(lib, c), {**c, **clean}
        res = _attn.want(ref)
        tol, _ = _attn.bounds(ref, res)
        for n in ("out", "lse", "dq", "dk", "dv"):
            mine = np.broadcast_to(~other[:, None], got[n].shape[:3])
            assert (np.abs(got[n][mine] - res[n][mine]) <= tol[n][mine])[np.isfinite(res[n][mine])].all(), n
            unused = np.broadcast_to((c["mask"]["doc_k"] < 0)[:, None], got[n].shape[:3])
            assert (got[n][unused] == (-np.inf if n == "lse" else 0)).all(), n


@pytest.mark.parametrize("d", [32, 16, 64])
@pytest.mark.parametrize("G", [150, 900])
def test_what_later_keys_hold_reaches_no_earlier_query(lib, G, d):
    c, cut = _attn.make(8, 1, 2, 2, G, G, d, prefix=0), G - 50
    for n in ("k", "v", "q", "dout"):
        c[n][:, :, cut:] = np.nan
    got = _attn.run(lib, c)
    ref = _attn.make(8, 1, 2, 2, G, G, d, prefix=0)
    for n in ("k", "v", "q", "dout"):
        ref[n][:, :, cut:] = 0
    res = _attn.want(ref)
    for n in ("out", "lse", "dq"):
        assert np.isfinite(got[n][:, :, :cut]).all()
        assert np.linalg.norm(got[n][:, :, :cut] - res[n][:, :, :cut]) <= 3e-6 * np.linalg.norm(res[n][:, :, :cut])
        assert np.isnan(got[n][:, :, cut:]).all()
    assert np.isnan(got["dk"]).all()  # every key is seen by the last queries


@pytest.mark.parametrize("d", [32, 16, 64])
@pytest.mark.parametrize("H, G", [(1, 40), (4, 640)])
def test_a_visible_nan_or_infinite_score(lib, H, G, d):
    c = _attn.make(9, 1, H, H, G, G, d, bwd=False)
    c["k"][0, :, 5, 0] = np.nan
    assert np.isnan(_attn.run(lib, c)["out"]).all()
    c = _attn.make(9, 1, H, H, G, G, d, bwd=False)
    c["k"][0, :, :, :] = 0
    c["k"][0, :, 5] = -np.inf
    c["q"][:] = np.abs(c["q"]) + 0.1  # key 5 scores -infinity for every query: weight 0
    got, clean = _attn.run(lib, c), {**c, "k": np.delete(c["k"], 5, 2), "v": np.delete(c["v"], 5, 2), "Gk": G - 1}
    assert np.abs(got["out"] - _attn.want(clean)["out"]).max() < 1e-6


def test_gradients_are_those_of_differences(lib):
    """The forward of the library, in fp32: central differences along random directions."""
    c = _attn.make(10, 1, 2, 1, 33, 33, 32, cap=2.0, bias="place", docs=1)
    got = _attn.run(lib, c)
    rng = np.random.default_rng(0)
    for n, gname in (("q", "dq"), ("k", "dk"), ("v", "dv")):
        step = rng.standard_normal(c[n].shape).astype(np.float32)
        h = 2.0 ** -6
        f = [(_attn.run(lib, {**c, n: (c[n] + s * h * step).astype(np.float32), "dout": None})["out"].astype(np.float64)
              * c["dout"]).sum() for s in (1, -1)]
        slope, scale = (got[gname].astype(np.float64) * step).sum(), np.linalg.norm(got[gname])
        # third derivatives of order one times h^2 / 6, over the norm of some 1000 entries
        assert abs((f[0] - f[1]) / (2 * h) - slope) < 2e-3 * max(abs(slope), scale)


def test_mask_tensors_may_be_views(lib):
    """Word-aligned positions, documents, slopes and prefix lengths: views into longer tensors."""
    for G in (70, 900):
        c = _attn.make(G, 1, 2, 2, G, G, 32, bias="place", docs=2, prefix=1)
        m = _attn.mask_of(lib, c)
        for n in ("slopes", "pos_q", "pos_k", "doc_q", "doc_k", "prefix"):
            t = getattr(m, n)
            long = torch.zeros(t.numel() + 3, dtype=t.dtype, device="cuda")
            view = long[1:1 + t.numel()].view(t.shape)
            view.copy_(t)
            assert view.data_ptr() % 16 == 4
            setattr(m, n, view)
        got = _attn.run(lib, c)
        again = _attn.run(lib, c, mask=m)
        assert all(np.array_equal(got[n], again[n]) for n in got)


def test_two_calls_streams_graphs_and_the_same_bits(lib):
    c = _attn.make(11, 2, 8, 8, 512, 512, 32, cap=20.0, docs=3)
    s, m = _attn.shape_of(lib, c), _attn.mask_of(lib, c)
    q, k, v, do = (_attn.dev(c[n]) for n in ("q", "k", "v", "dout"))
    o = [torch.empty_like(q), torch.empty_like(q[..., 0]), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]
    wf, wb = lib.attn_workspace(s), lib.attn_workspace(s, backward=True)

    def step(stream=None):
        lib.fs_attn_fwd(s, q, k, v, m, o[0], o[1], wf, stream=stream)
        lib.fs_attn_bwd(s, q, k, v, m, o[0], o[1], do, o[2], o[3], o[4], wb, stream=stream)

    step()
    first = [t.clone() for t in o]
    wf.random_(); wb.random_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, o))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in o:
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, o))


def test_splits_and_whole_rows_agree_with_the_oracle_at_a_large_size(lib):
    """4096 tokens, a few heads' rows against 64 bits."""
    c = _attn.make(12, 1, 2, 1, 4096, 4096, 32, prefix=1, bias="index", bwd=False)
    got = _attn.run(lib, c)
    rows = np.array([0, 1, 63, 64, 2047, 4000, 4095])
    for h in range(2):
        q, k, v = c["q"][0, h, rows].astype(np.float64), c["k"][0, 0].astype(np.float64), c["v"][0, 0].astype(np.float64)
        i, j = rows[:, None], np.arange(4096)[None, :]
        a = c["scale"] * q @ k.T - float(c["mask"]["slopes"][h]) * np.abs(i - j)
        a[(j > i) & (j >= c["mask"]["prefix"][0])] = -np.inf
        p = np.exp(a - a.max(1, keepdims=True))
        out = (p / p.sum(1, keepdims=True)) @ v
        assert np.linalg.norm(got["out"][0, h, rows] - out) <= 3e-6 * np.linalg.norm(out)


def test_one_query_over_a_long_cache(lib):
    """200,003 keys, split many ways: offsets and joins."""
    c = _attn.make(13, 2, 2, 1, 1, 200003, 16, bias="index", docs=3, bwd=False)
    c["mask"]["doc_q"][:] = [[1], [-1]]
    c["mask"]["slopes"] *= np.float32(1e-4)
    _attn.check(lib, c)


def test_many_units(lib):
    """More units than SMs, few tokens each."""
    _attn.check(lib, _attn.make(14, 40, 8, 4, 20, 20, 16, cap=2.0))
    _attn.check(lib, _attn.make(15, 20, 8, 8, 129, 130, 32, bwd=False))
