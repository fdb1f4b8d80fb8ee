"""The calls of a training step side by side: on two streams at once, captured graphs that share a workspace, outputs inside larger buffers, offsets beyond
32 bits, and what the entry points refuse."""
import math

import pytest
import torch

import attention_gradients as attention

pytestmark = pytest.mark.gpu
NAMES = ("dq", "dk", "dv", "dlambda")


@pytest.fixture(scope="module")
def hgf():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    torch.cuda.set_device(0)
    return binding


def rotation(n, h, dh, seed):
    r = torch.Generator(device="cuda").manual_seed(seed)
    x = lambda: torch.randn(n, h * dh, generator=r, device="cuda").to(torch.bfloat16)  # noqa: E731
    return x(), x(), torch.randint(0, 9000, (n,), generator=r, device="cuda", dtype=torch.int32), x(), x(), torch.rand(dh, generator=r, device="cuda"), torch.rand(dh, generator=r, device="cuda")


@pytest.mark.parametrize("B,L,h,dh", [(1, 4099, 1, 64), (1, 3001, 2, 128)])
def test_a_long_text(hgf, B, L, h, dh):
    q, k, v, g = attention.inputs(B, L, h, dh, 3, "cuda")
    out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, 0.8, 0.5, flags=hgf.FLAG_OUT_BF16)
    got = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, 0.8, 0.5)
    want = attention.reference(q, k, v, g, B, L, h, dh, 0.8, 0.5)
    for n, x in (("out", out), ("streams", streams), *((n, got[n]) for n in NAMES)):
        assert ((x.double() - want[n][0]).abs() <= want[n][1]).all(), n
    hgf.check_status()


def test_two_streams_at_once(hgf):
    """Calls with workspaces of their own, on two streams whose kernels run beside each other, give what each gives alone."""
    shapes = [(2, 300, 9, 64), (3, 190, 5, 128)]
    alone, steps = [], []
    for n, (B, L, h, dh) in enumerate(shapes):
        q, k, v, g = attention.inputs(B, L, h, dh, 20 + n, "cuda")
        rot = rotation(B * L, 2 * h, dh, n)
        grads = [torch.randn(100003 + n, device="cuda"), torch.randn(777, device="cuda")]
        scaled = [torch.empty_like(x) for x in grads]
        clip = hgf.GradList(grads, scaled)

        def step(stream, a=(q, k, v, g, B, L, h, dh), rot=rot, clip=clip, scaled=scaled):
            q, k, v, g, B, L, h, dh = a
            out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, 0.8, stream=stream)
            b = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, 0.8, stream=stream)
            x, y, pos, gx, gy, wx, wy = rot
            r = hgf.qk_norm_rotate_backward(x, y, pos, dh, gx, gy, wx, wy, stream=stream)
            norm = clip.clip(0.5, stream=stream)
            return [out, streams, lse, *(b[n] for n in NAMES), r["dq"], r["dk"], r["dwq"], r["dwk"], norm, *(s.clone() if stream is None else s for s in scaled)]
        steps.append(step)
        alone.append(step(None))
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [step(side) for step, side in zip(steps, sides)]
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(map(torch.equal, a, b))
    hgf.check_status()


def test_two_graphs_with_one_workspace(hgf):
    """One after the other on a stream, in any order."""
    graphs, want, kept, steps = [], [], [], []
    need = max(hgf.diff_attention_backward_workspace_bytes(2, 300, 3, 64), hgf.diff_attention_backward_workspace_bytes(1, 130, 4, 128),
               hgf.lib().hgf_qk_norm_rotate_workspace_bytes(128))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    for n, (B, L, h, dh) in enumerate([(2, 300, 3, 64), (1, 130, 4, 128)]):
        q, k, v, g = attention.inputs(B, L, h, dh, 30 + n, "cuda")
        x, y, pos, gx, gy, wx, wy = rotation(B * L, 2 * h, dh, n)
        _, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, 0.8)

        def step(out=None, rot=None, a=(q, k, v, g, streams, lse, B, L, h, dh, 0.8), r=(x, y, pos, dh, gx, gy, wx, wy)):
            return hgf.diff_attention_backward(*a, out=out, workspace=ws), hgf.qk_norm_rotate_backward(*r, out=rot, workspace=ws)
        one, two = step()
        names = [(d, m) for d, ms in ((one, NAMES), (two, ("dq", "dk", "dwq", "dwk"))) for m in ms]
        want.append([d[m].clone() for d, m in names])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(one, two)
        graphs.append(graph)
        steps.append(step)   # (its inputs live as long as the graph)
        kept.append(names)
    for n in (0, 1, 1, 0, 1, 0):
        for d, m in kept[n]:
            d[m].fill_(3.0)
        ws.fill_(255)
        graphs[n].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(d[m], w) for (d, m), w in zip(kept[n], want[n]))


@pytest.mark.parametrize("dh", [64, 128])
def test_rows_behind_the_last_stay_as_they_were(hgf, dh):
    B, L, h, more = 3, 45, 2, 40
    q, k, v, g = attention.inputs(B, L, h, dh, 40, "cuda")
    x, y, pos, gx, gy, wx, wy = rotation(B * L, 2 * h, dh, 5)
    room = lambda t: torch.full((t.shape[0] + more, *t.shape[1:]), 5.0, dtype=t.dtype, device="cuda")  # noqa: E731
    out, streams, lse = room(v), torch.full((B * L + more, 2 * h * dh), 5.0, device="cuda"), torch.full((B + 1, h, 2, L), 5.0, device="cuda")
    hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, 0.8, out=out[:B * L], streams=streams[:B * L], lse=lse[:B], flags=hgf.FLAG_OUT_BF16)
    grads = {"dq": room(q), "dk": room(k), "dv": room(v), "dlambda": torch.full((5,), 5.0, device="cuda")}
    ws = torch.empty(hgf.diff_attention_backward_workspace_bytes(B, L, h, dh) + 4096, dtype=torch.uint8, device="cuda").fill_(77)
    need = ws.numel() - 4096
    hgf.diff_attention_backward(q, k, v, g, streams[:B * L], lse[:B], B, L, h, dh, 0.8, out={n: t[:1 if n == "dlambda" else B * L] for n, t in grads.items()}, workspace=ws[:need])
    rot = {"dq": room(x), "dk": room(y), "dwq": torch.full((dh + 9,), 5.0, device="cuda"), "dwk": torch.full((dh + 9,), 5.0, device="cuda")}
    hgf.qk_norm_rotate_backward(x, y, pos, dh, gx, gy, wx, wy, out={n: t[:dh if n[1] == "w" else B * L] for n, t in rot.items()}, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    xo, yo = room(x), room(y)
    hgf.qk_norm_rotate(x, y, pos, dh, wx, wy, q_out=xo[:B * L], k_out=yo[:B * L])
    for t, n in ((out, B * L), (streams, B * L), (lse, B), (grads["dq"], B * L), (grads["dk"], B * L), (grads["dv"], B * L), (grads["dlambda"], 1),
                 (rot["dq"], B * L), (rot["dk"], B * L), (rot["dwq"], dh), (rot["dwk"], dh), (xo, B * L), (yo, B * L)):
        assert (t[n:] == 5.0).all() and not (t[:n] == 5.0).all()
    assert (ws[need:] == 77).all()


def test_rotation_offsets_beyond_32_bits(hgf):
    """More than 2^31 values of Q: the last rows are what they are alone."""
    n, h, dh, last = 66000, 512, 64, 9
    few, _, _, g, _, w, _ = rotation(600, h, dh, 6)
    q, dy = few.repeat(110, 1), g.repeat(110, 1)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    assert q.numel() > 2 ** 31
    y, _ = hgf.qk_norm_rotate(q, None, pos, dh, w)
    alone, _ = hgf.qk_norm_rotate(q[-last:], None, pos[-last:], dh, w)
    assert torch.equal(y[-last:], alone)
    del y
    b = hgf.qk_norm_rotate_backward(q, None, pos, dh, dy, None, w)
    alone = hgf.qk_norm_rotate_backward(q[-last:], None, pos[-last:], dh, dy[-last:], None, w)
    assert torch.equal(b["dq"][-last:], alone["dq"])


def test_attention_offsets_beyond_32_bits(hgf):
    """More than 2^31 values of Q, of the streams' outputs and of dQ: the last sequences are what they are alone."""
    B, L, h, dh, few, lam = 36000, 16, 16, 128, 100, 0.8
    some = attention.inputs(few, L, h, dh, 50, "cuda")
    q, k, v, g = (x.repeat(B // few, 1) for x in some)
    assert q.numel() > 2 ** 31
    out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam, flags=hgf.FLAG_OUT_BF16)
    got = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, lam)
    hgf.check_status()
    o, s, m = hgf.diff_attention_forward_train(*some[:3], few, L, h, dh, lam, flags=hgf.FLAG_OUT_BF16)
    alone = hgf.diff_attention_backward(*some, s, m, few, L, h, dh, lam)
    rows = few * L
    for a, b in ((out, o), (streams, s), *((got[n], alone[n]) for n in ("dq", "dk", "dv"))):
        assert torch.equal(a[-rows:], b) and torch.equal(a[:rows], b)
    assert torch.equal(lse[-few:], m)
    assert abs(float(got["dlambda"]) - B // few * float(alone["dlambda"])) <= 2.0 ** -20 * (B // few) * abs(float(alone["dlambda"]))


def test_a_gradient_of_more_than_two_to_the_31(hgf):
    n = 2 ** 31 + 77
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    x[-1] = 1024.0
    norm = hgf.GradList([x]).clip(2.0 ** 14)
    want = math.sqrt(n - 1 + 2.0 ** 20)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    f = 2.0 ** 14 / (want + 1e-6)
    assert abs(float(x[-1]) / (1024 * f) - 1) <= 2.0 ** -8 + 2.0 ** -22 and abs(float(x[0]) / f - 1) <= 2.0 ** -8 + 2.0 ** -22
    assert (x[:-1] == x[0]).all()


def test_an_infinite_limit_leaves_the_gradients(hgf):
    """Where only the norm is asked for, gradients stay as they are, whatever they hold."""
    for bad in (1.0, math.inf, math.nan):
        g = [torch.randn(5000, device="cuda"), torch.randn(33, device="cuda").to(torch.bfloat16)]
        g[0][77] = bad
        was, out = [x.clone() for x in g], [torch.zeros_like(x) for x in g]
        norm = float(hgf.GradList(g).clip(math.inf))
        assert math.isnan(norm) if math.isnan(bad) else (math.isinf(norm) == math.isinf(bad))
        hgf.GradList(g, out).clip(math.inf)
        for a, b, c in zip(was, g, out):
            assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) and torch.equal(a.nan_to_num(9.0), c.nan_to_num(9.0))


def test_a_closed_list(hgf):
    x = torch.ones(10, device="cuda")
    grads, norm = hgf.GradList([x]), torch.zeros(1, device="cuda")
    grads.close()
    grads.close()
    for where in (None, norm):
        with pytest.raises(hgf.HgfError):
            grads.clip(0.1, norm=where)
    assert (x == 1).all()


def test_refusals_leave_the_outputs(hgf):
    """Wrong tensors are refused by whichever way a call takes, before anything is enqueued."""
    B, L, h, dh = 2, 40, 2, 64
    q, k, v, g = attention.inputs(B, L, h, dh, 60, "cuda")
    out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, 0.8)
    grads = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, 0.8)
    kept = {"out": out, "streams": streams, "lse": lse, **{n: grads[n] for n in NAMES}}
    was = {n: t.clone() for n, t in kept.items()}
    aside = torch.empty(B * L * 2 * h * dh + 8, dtype=torch.bfloat16, device="cuda")[1:-7].view(B * L, -1)   # (not on 16 bytes)
    forward = {"q": q, "k": k, "v": v, "out": out, "streams": streams, "lse": lse}
    for name, bad, error in (("q", q.float(), AssertionError), ("k", k[:-1], AssertionError), ("v", v.t().contiguous().t(), AssertionError), ("q", q.cpu(), AssertionError),
                             ("k", aside, hgf.HgfError), ("out", out.double(), AssertionError), ("streams", streams.to(torch.bfloat16), AssertionError),
                             ("streams", streams[:, :-8], AssertionError), ("lse", lse[:, :, :1], AssertionError)):
        a = {**forward, name: bad}
        with pytest.raises(error):
            hgf.diff_attention_forward_train(a["q"], a["k"], a["v"], B, L, h, dh, 0.8, out=a["out"], streams=a["streams"], lse=a["lse"])
    inputs = {"q": q, "k": k, "v": v, "g": g, "streams": streams, "lse": lse}
    small = torch.empty(1024, dtype=torch.uint8, device="cuda")
    for name, bad, error in (("g", g.float(), AssertionError), ("g", None, (AssertionError, AttributeError)), ("lse", lse.double(), AssertionError), ("q", aside, hgf.HgfError),
                             ("dq", grads["dq"].float(), AssertionError), ("dv", grads["dv"][1:], AssertionError), ("dlambda", grads["dlambda"].double(), AssertionError),
                             ("dk", aside, hgf.HgfError), ("_workspace", small, hgf.HgfError), ("_workspace", grads["_workspace"][1:], hgf.HgfError)):
        a, o = {**inputs}, {**grads}
        (a if name in a else o)[name] = bad
        with pytest.raises(error):
            hgf.diff_attention_backward(a["q"], a["k"], a["v"], a["g"], a["streams"], a["lse"], B, L, h, dh, 0.8, out=o)
    with pytest.raises(hgf.HgfError):
        hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, 0.8, want=("dk",))
    torch.cuda.synchronize()
    assert all(torch.equal(kept[n], was[n]) for n in kept)
    hgf.check_status()


@pytest.mark.parametrize("B,L,h,dh", [(1, 61, 4, 64), (2, 300, 9, 64), (1, 200, 3, 128)])
def test_calls_close_behind_one_another(hgf, B, L, h, dh):
    """Launches start before the work in front of them has ended: passes whose inputs, outputs and workspaces the next one writes over, none waited for
    (once in a stream, once captured with the copies between them), give what they give one at a time."""
    inputs = [(*attention.inputs(B, L, h, dh, 70 + n, "cuda"), *rotation(B * L, 2 * h, dh, n)) for n in range(3)]
    a = [torch.empty_like(x) for x in inputs[0]]
    q, k, v, g, x, y, pos, gx, gy, wx, wy = a
    out, streams, lse = hgf.diff_attention_forward_train(q.zero_(), k.zero_(), v.zero_(), B, L, h, dh, 0.8)
    back = hgf.diff_attention_backward(q, k, v, g.zero_(), streams, lse, B, L, h, dh, 0.8)
    xo, yo = torch.empty_like(x), torch.empty_like(y)
    rot = hgf.qk_norm_rotate_backward(x, y, pos.zero_(), dh, gx, gy, wx, wy)
    clip, norm = hgf.GradList([back["dq"], back["dk"], back["dv"], back["dlambda"], rot["dwq"]]), torch.empty(1, device="cuda")

    def step(n):
        for to, new in zip(a, inputs[n]):
            to.copy_(new)
        hgf.qk_norm_rotate(x, y, pos, dh, wx, wy, q_out=xo, k_out=yo)
        hgf.diff_attention_forward_train(xo, yo, v, B, L, h, dh, 0.8, out=out, streams=streams, lse=lse)
        hgf.diff_attention_backward(xo, yo, v, g, streams, lse, B, L, h, dh, 0.8, out=back)
        hgf.qk_norm_rotate_backward(x, y, pos, dh, back["dq"], back["dk"], wx, wy, out=rot)
        clip.clip(1e-3, norm=norm)
        hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, 0.8, out=out, streams=streams, lse=lse)
        return [t.clone() for t in (xo, yo, out, streams, lse, back["dq"], back["dk"], back["dv"], back["dlambda"], rot["dq"], rot["dk"], rot["dwq"], rot["dwk"], norm)]
    alone = []
    for n in range(3):
        alone.append(step(n))
        torch.cuda.synchronize()
    got = [step(n % 3) for n in range(30)]
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for n, r in enumerate(got) for s, t in zip(r, alone[n % 3]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [step(n % 3) for n in range(6)]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for n, r in enumerate(got) for s, t in zip(r, alone[n % 3]))
    hgf.check_status()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("L", [1, 64, 65, 192, 320])
def test_sequences_at_the_ends_of_steps(hgf, L, dh):
    """Sequences that end with a step, inside one and inside a tile only: one whose values are not finite leaves the others as they are."""
    B, h = 3, 2
    q, k, v, g = attention.inputs(B, L, h, dh, 80, "cuda")

    def everything():
        plain = hgf.diff_attention_forward(q, k, v, B, L, h, dh, 0.8)
        out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, 0.8)
        b = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, 0.8)
        return plain, out, streams, lse.permute(0, 3, 1, 2).reshape(B * L, -1), b["dq"], b["dk"], b["dv"]
    clean = everything()
    for bad in (math.nan, math.inf):
        for x in (q, k, v, g):
            x[L:2 * L] = bad
        for a, b in zip(clean, everything()):
            assert torch.equal(a[:L], b[:L]) and torch.equal(a[2 * L:], b[2 * L:]) and not b[L:2 * L].isfinite().all()
    hgf.check_status()
