"""hgf_qk_norm_rotate and its gradients against the definition in 64 bits, element by element."""
import pytest
import torch

import rotate_reference as ref

pytestmark = pytest.mark.gpu
EPS, BASE = 1e-6, 10000.0


@pytest.fixture(scope="module")
def hgf():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    torch.cuda.set_device(0)
    return binding


def inputs(n, hq, hk, dh, seed=0, far=5000):
    r = torch.Generator().manual_seed(seed)
    x = lambda h, s: None if not h else (torch.randn(n, h * dh, generator=r) * s).to(torch.bfloat16).cuda()  # noqa: E731
    w = lambda: (1 + 0.3 * torch.randn(dh, generator=r)).cuda()  # noqa: E731
    return {"q": x(hq, 2.0), "k": x(hk, 0.1), "pos": torch.randint(0, far, (n,), generator=r, dtype=torch.int32).cuda(), "wq": w(), "wk": w(),
            "gq": x(hq, 0.03), "gk": x(hk, 0.03)}


def close(got, want):
    value, bound = want
    over = (got.double() - value).abs() - bound
    assert (over <= 0).all(), f"{over.max():.3e} over, largest value {value.abs().max():.3e}"


def check(hgf, s, dh, rot=None, pairs=False, eps=EPS, base=BASE):
    rot = dh if rot is None else rot
    how = {"eps": eps, "base": base, "rotary_dim": rot, "flags": hgf.FLAG_ROTATE_PAIRS if pairs else 0}
    out = hgf.qk_norm_rotate(s["q"], s["k"], s["pos"], dh, s["wq"], s["wk"], **how)
    g = hgf.qk_norm_rotate_backward(s["q"], s["k"], s["pos"], dh, s["gq"], s["gk"], s["wq"], s["wk"], **how)
    for name, y in zip("qk", out):
        if s[name] is None:
            assert y is None and "d" + name not in g
            continue
        close(y, ref.forward(s[name], s["pos"], dh, s["w" + name], eps, base, rot, pairs))
        want = ref.backward(s[name], s["g" + name], s["pos"], dh, s["w" + name], eps, base, rot, pairs)
        close(g["d" + name], want["dx"])
        close(g["dw" + name], want["dw"])
    return out, g


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,hq,hk", [(1, 1, 1), (1, 32, 8), (7, 5, 3), (33, 9, 17), (600, 6, 2)])
def test_shapes(hgf, dh, pairs, n, hq, hk):
    check(hgf, inputs(n, hq, hk, dh, seed=n), dh, pairs=pairs)


@pytest.mark.parametrize("dh", [64, 128])
def test_many_rows(hgf, dh):
    """Warps that take several heads of a token, and several tokens."""
    check(hgf, inputs(9001, 24, 7, dh, seed=1), dh)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("pairs", [False, True])
def test_some_of_the_dims_are_rotated(hgf, dh, pairs):
    s = inputs(13, 6, 4, dh, seed=2)
    for rot in range(0, dh + 1, 16):
        check(hgf, s, dh, rot=rot, pairs=pairs, base=500.0)


@pytest.mark.parametrize("dh", [64, 128])
def test_far_positions_and_negative_ones(hgf, dh):
    s = inputs(64, 4, 2, dh, seed=3)
    s["pos"][:8] = torch.tensor([0, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 10 ** 9 + 7, -123456789, 131071], dtype=torch.int32)
    check(hgf, s, dh)
    check(hgf, s, dh, base=5e5, pairs=True)


def test_one_side_alone_and_no_weights(hgf):
    s = inputs(50, 8, 4, 64, seed=4)
    both, _ = check(hgf, s, 64)
    for name, other in (("q", "k"), ("k", "q")):
        alone = {**s, other: None, "g" + other: None}
        out, g = check(hgf, alone, 64)
        assert torch.equal(out["qk".index(name)], both["qk".index(name)])
    check(hgf, {**s, "wq": None}, 64)
    check(hgf, {**s, "wq": None, "wk": None}, 64)


def test_zeros_small_and_large_values(hgf):
    s = inputs(8, 4, 4, 64, seed=5)
    s["q"][0] = 0
    s["q"][1] *= 1e-12
    s["q"][2] *= 1e12
    s["k"][3, 5] = 3e9
    check(hgf, s, 64, eps=1e-5)
    out, g = hgf.qk_norm_rotate(s["q"], s["k"], s["pos"], 64, s["wq"], s["wk"]), hgf.qk_norm_rotate_backward(s["q"], s["k"], s["pos"], 64, s["gq"], s["gk"])
    assert not out[0][0].any() and g["dq"][0].isfinite().all()


def test_a_head_that_is_not_finite_stays_alone(hgf):
    s = inputs(9, 8, 4, 64, seed=6)
    clean, grads = check(hgf, s, 64)
    x = s["q"].clone()
    x[4, 64:128] = float("nan")
    x[6, 3] = float("inf")
    bad = torch.zeros(9, 8, dtype=torch.bool, device="cuda")
    bad[4, 1] = bad[6, 0] = True
    y, _ = hgf.qk_norm_rotate(x, s["k"], s["pos"], 64, s["wq"], s["wk"], eps=EPS)
    g = hgf.qk_norm_rotate_backward(x, s["k"], s["pos"], 64, s["gq"], s["gk"], s["wq"], s["wk"], eps=EPS)
    for a, b in ((y, clean[0]), (g["dq"], grads["dq"])):
        a, b = a.view(9, 8, 64), b.view(9, 8, 64)
        assert torch.equal(a[~bad], b[~bad]) and not a[4, 1].isfinite().any() and not a[6, 0].isfinite().all()
    assert torch.equal(g["dk"], grads["dk"]) and torch.equal(g["dwk"], grads["dwk"]) and not g["dwq"].isfinite().any()


@pytest.mark.parametrize("dh", [64, 128])
def test_in_place_and_equal_bits(hgf, dh):
    s = inputs(300, 6, 10, dh, seed=7)
    one = hgf.qk_norm_rotate(s["q"], s["k"], s["pos"], dh, s["wq"], s["wk"])
    g = hgf.qk_norm_rotate_backward(s["q"], s["k"], s["pos"], dh, s["gq"], s["gk"], s["wq"], s["wk"])
    ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    for want in (None, ("dq",), ("dwk",), ("dk", "dwq"), ()):
        part = hgf.qk_norm_rotate_backward(s["q"], s["k"], s["pos"], dh, s["gq"], s["gk"], s["wq"], s["wk"], want=want, workspace=ws)
        assert set(part) - {"_workspace"} == set(("dq", "dk", "dwq", "dwk") if want is None else want)
        assert all(torch.equal(part[n], g[n]) for n in part if n != "_workspace")
    gq, gk = s["gq"].clone(), s["gk"].clone()
    same = hgf.qk_norm_rotate_backward(s["q"], s["k"], s["pos"], dh, gq, gk, s["wq"], s["wk"], out={**g, "dq": gq, "dk": gk})
    fresh = hgf.qk_norm_rotate_backward(s["q"], s["k"], s["pos"], dh, s["gq"], s["gk"], s["wq"], s["wk"])
    assert same["dq"] is gq and all(torch.equal(same[n], fresh[n]) for n in ("dq", "dk", "dwq", "dwk"))
    q, k = s["q"].clone(), s["k"].clone()
    hgf.qk_norm_rotate(q, k, s["pos"], dh, s["wq"], s["wk"], q_out=q, k_out=k)
    assert torch.equal(q, one[0]) and torch.equal(k, one[1])


def test_a_captured_decode_step_follows_its_positions(hgf):
    """Rotation, append and cached attention as one graph that is replayed token by token, against whole sequences at once."""
    S, n, h, dh, lam = 3, 70, 2, 64, 0.8
    s = inputs(S * n, 2 * h, 2 * h, dh, seed=8)
    v = torch.randn(S * n, h * dh, device="cuda").to(torch.bfloat16)
    s["pos"] = torch.arange(n, dtype=torch.int32, device="cuda").repeat(S)
    every = hgf.qk_norm_rotate(s["q"], s["k"], s["pos"], dh, s["wq"], s["wk"])
    cache = hgf.KVCache(h, dh, 2 * S, S, 2)
    slots, starts = torch.arange(S, dtype=torch.int32, device="cuda"), torch.arange(S + 1, dtype=torch.int32, device="cuda")
    hgf.cache_reserve(cache, slots, torch.full((S,), n, dtype=torch.int32, device="cuda"))
    q, k, x = (torch.empty(S, t.shape[1], dtype=t.dtype, device="cuda") for t in (s["q"], s["k"], v))
    qo, ko, out = torch.empty_like(q), torch.empty_like(k), torch.empty(S, h * dh, device="cuda")
    done, ws = torch.empty(S, dtype=torch.int32, device="cuda"), torch.empty(hgf.cached_workspace_bytes(cache, S, S, h), dtype=torch.uint8, device="cuda")

    def step():
        hgf.qk_norm_rotate(q, k, cache.length, dh, s["wq"], s["wk"], q_out=qo, k_out=ko)   # (a token's position: how many the sequence holds)
        hgf.cache_append(cache, ko, x, slots, starts, done=done)
        hgf.diff_attention_cached(cache, qo, slots, starts, lam, out=out, workspace=ws)

    graph = torch.cuda.CUDAGraph()
    step()
    cache.length.zero_()
    with torch.cuda.graph(graph):
        step()
    at = torch.arange(S, device="cuda") * n
    for t in range(n):
        q.copy_(s["q"][at + t])
        k.copy_(s["k"][at + t])
        x.copy_(v[at + t])
        graph.replay()
        assert torch.equal(qo, every[0][at + t]) and torch.equal(ko, every[1][at + t])
    hgf.check_status()
    assert cache.length.tolist() == [n] * S
    whole = hgf.diff_attention_forward(*every, v, S, n, h, dh, lam)
    # (the cache's codes are 8 bits: 2^-8 of a block's largest value in K and V)
    assert (out - whole[at + n - 1]).abs().max() <= 0.05 * v.float().abs().max()
