"""attnqat_rope_fwd, attnqat_rope_bwd and attnqat_kv_cache_append_rope against 64 bits.

Sine and cosine are off by at most 2^-23 + 2 pi 2^-32 < 2^-22.9 each, the two products and their sum by 2^-24 of the product's size each: together less than
(|a| + |b|) 2^-21 for a pair (a, b); the one rounding to bf16 is a relative 2^-8."""
import copy
import pickle

import numpy as np
import pytest
import torch

from tests import serve_util as S, sparse_util as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aq():
    import paper_2603_00040_amd as aq
    return aq


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def table(aq, dims, layout, theta=10000.0):
    freqs = [theta ** (-2.0 * i / n) for n in dims for i in range(n // 2)]
    axis = [a for a, n in enumerate(dims) for _ in range(n // 2)]
    return aq.rope_table(dims, theta=theta, layout=layout), freqs, axis


def check(got, x, positions, freqs, axis, layout, sign=1.0):
    """got, x [L, heads, d]; values that do not turn are the same bits."""
    y, size = P.turned(x.double().cpu().numpy(), positions, freqs, axis, layout, sign)
    g = got.double().cpu().numpy()
    err = np.abs(g - y) - (2.0 ** -8 * np.abs(y) + 2.0 ** -21 * size)
    assert not np.isnan(g).any() and err.max() <= 0.0, float(err.max())
    n = 2 * len(freqs)
    assert torch.equal(got[..., n:].view(torch.int16), x[..., n:].view(torch.int16))


def views(x, how):
    """x [B, H, L, d] on the GPU, same values, other strides."""
    B, H, L, d = x.shape
    if how == "plain":
        return x.contiguous()
    if how == "fused":                                            # a piece of a projection's output [B, L, heads, d]
        y = torch.full((B, L, H + 3, d), 9.0, dtype=x.dtype, device="cuda")
        y[:, :, 2:2 + H] = x.transpose(1, 2)
        return y[:, :, 2:2 + H].transpose(1, 2)
    y = torch.full((L, H, B, d + 8), 9.0, dtype=x.dtype, device="cuda")                       # everything the other way round, padded
    y[..., :d] = x.permute(2, 1, 0, 3)
    return y[..., :d].permute(2, 1, 0, 3)


def grid(B, L, axes, rng, far):
    p = rng.integers(-far, far + 1, (B, L, axes)) if far else np.stack([np.arange(L) // 3 ** a for a in range(axes)], -1)[None].repeat(B, 0)
    return p.astype(np.int32)


CASES = [((128,), "paired", 128), ((128,), "halves", 128), ((44, 42, 42), "paired", 128), ((32, 48, 48), "halves", 128), ((64,), "halves", 64), ((20, 22, 22), "paired", 64),
         ((2,), "paired", 64), ((16,), "halves", 64), ((30, 0, 12, 4), "paired", 128), ((48,), "halves", 128), ((16, 16, 0, 16), "halves", 128)]


@pytest.mark.parametrize("dims,layout,d", CASES)
@pytest.mark.parametrize("B,Hq,Hkv,L,how,far", [(1, 1, 1, 1, "plain", 0), (2, 5, 1, 33, "fused", 0), (3, 4, 2, 7, "other", 1 << 20), (1, 9, 9, 257, "fused", 2 ** 31 - 1)])
def test_forward_and_gradient(aq, dims, layout, d, B, Hq, Hkv, L, how, far):
    rng = np.random.default_rng(L + d)
    rope, freqs, axis = table(aq, dims, layout)
    pos = grid(B, L, len(dims), rng, far)
    shared = B == 1
    q, k = (S.bf16(rng.standard_normal((B, h, L, d)) * np.exp2(rng.integers(-20, 20, (B, h, L, 1)))).cuda() for h in (Hq, Hkv))
    qo, ko = aq.attnqat_rope_fwd(views(q, how), views(k, how), i32(pos[0] if shared else pos), rope)
    dq, dk = aq.attnqat_rope_bwd(qo, ko, i32(pos), rope, out=tuple(views(torch.full_like(t, 3.0), how) for t in (q, k)))
    assert qo.is_contiguous() and ko.is_contiguous()
    for x, y, g in ((q, qo, dq), (k, ko, dk)):
        for b in range(B):
            check(y[b].transpose(0, 1), x[b].transpose(0, 1), pos[b], freqs, axis, layout)
            check(g[b].transpose(0, 1), y[b].transpose(0, 1), pos[b], freqs, axis, layout, -1.0)


@pytest.mark.parametrize("dims,layout,d", CASES[:6])
def test_gradient_against_differences(aq, dims, layout, d):
    """Token l has +-1 in value l: the difference of the outputs, weighed by an upstream gradient, is the gradient of that value.  Outputs are rounded to bf16
    (2^-8 each, the two of a difference alike), the gradient too."""
    rng = np.random.default_rng(d)
    rope, _, _ = table(aq, dims, layout)
    pos = i32(rng.integers(-1000, 1000, (d, len(dims))))
    x = torch.eye(d, device="cuda", dtype=torch.bfloat16)[None, None]                           # [1, 1, d tokens, d]
    up, _ = aq.attnqat_rope_fwd(x, None, pos, rope)
    down, _ = aq.attnqat_rope_fwd(-x, None, pos, rope)
    dy = S.bf16(rng.standard_normal((1, 1, d, d))).cuda()
    g, _ = aq.attnqat_rope_bwd(dy, None, pos, rope)
    parts = dy.double() * (up.double() - down.double()) / 2.0
    want = parts.sum(-1)[0, 0]
    got = torch.diagonal(g[0, 0]).double()
    slack = 2.0 ** -8 * got.abs() + (2.0 ** -8 + 2.0 ** -8) * parts.abs().sum(-1)[0, 0] + 2.0 ** -21 * dy.double().abs().amax(-1)[0, 0]
    assert bool(((got - want).abs() <= slack).all())


def test_frequencies_and_axes_of_ones_own(aq):
    rng = np.random.default_rng(4)
    freqs, axis = [float(f) for f in rng.standard_normal(24) * 10.0 ** rng.integers(-6, 3, 24)], [int(a) for a in rng.integers(0, 3, 24)]
    rope = aq.rope_table((16, 16, 16), layout="halves", freqs=freqs, axis=axis)
    x = S.bf16(rng.standard_normal((1, 2, 50, 64))).cuda()
    pos = grid(1, 50, 3, rng, 5000)
    y, _ = aq.attnqat_rope_fwd(x, None, i32(pos[0]), rope)
    check(y[0].transpose(0, 1), x[0].transpose(0, 1), pos[0], freqs, axis, "halves")


def test_in_place_in_one_buffer_and_out_of_it(aq):
    """q and k turned where they lie, V between the tokens untouched; gradients into views of one buffer."""
    rng = np.random.default_rng(5)
    B, L, Hq, Hkv, d = 2, 40, 6, 2, 128
    for layout in ("paired", "halves"):
        rope, freqs, axis = table(aq, (128,), layout)
        buf = S.bf16(rng.standard_normal((B, L, Hq + 2 * Hkv, d))).cuda()
        old = buf.clone()
        q, k = buf[:, :, :Hq].transpose(1, 2), buf[:, :, Hq:Hq + Hkv].transpose(1, 2)
        pos = grid(1, L, 1, rng, 3000)[0]
        wq, wk = aq.attnqat_rope_fwd(q, k, i32(pos), rope)
        aq.attnqat_rope_fwd(q, k, i32(pos), rope, out=(q, k))
        assert torch.equal(q, wq) and torch.equal(k, wk) and torch.equal(buf[:, :, Hq + Hkv:], old[:, :, Hq + Hkv:])
        grad = torch.full_like(buf, 7.0)
        aq.attnqat_rope_bwd(wq, wk, i32(pos), rope, out=(grad[:, :, :Hq].transpose(1, 2), grad[:, :, Hq:Hq + Hkv].transpose(1, 2)))
        gq, gk = aq.attnqat_rope_bwd(wq, wk, i32(pos), rope)
        assert torch.equal(grad[:, :, :Hq].transpose(1, 2), gq) and torch.equal(grad[:, :, Hq:Hq + Hkv].transpose(1, 2), gk) and bool((grad[:, :, Hq + Hkv:] == 7.0).all())


def test_broadcast_inputs_and_what_does_not_turn(aq):
    """One row for every head; infinities and NaN behind the turned part stay as they are."""
    rope, freqs, axis = table(aq, (16,), "halves")
    x = S.bf16(np.random.default_rng(1).standard_normal((1, 1, 5, 64))).cuda()
    x[..., 16], x[..., 40], x[..., 63] = float("inf"), float("nan"), -0.0
    pos = np.arange(5)[:, None]
    y, _ = aq.attnqat_rope_fwd(x.expand(3, 4, 5, 64), None, i32(pos), rope)
    one, _ = aq.attnqat_rope_fwd(x, None, i32(pos), rope)
    assert torch.equal(y.view(torch.int16), one.expand(3, 4, 5, 64).view(torch.int16))
    assert torch.equal(y[0, 0, :, 16:].view(torch.int16), x[0, 0, :, 16:].view(torch.int16))
    paired, freqs, axis = table(aq, (6,), "paired")                # a thread's eight pairs turn in part
    y, _ = aq.attnqat_rope_fwd(x, None, i32(pos), paired)
    assert torch.equal(y[..., 6:].view(torch.int16), x[..., 6:].view(torch.int16))
    check(y[0, ..., :16].transpose(0, 1), x[0, ..., :16].transpose(0, 1), pos, freqs, axis, "paired")


def test_another_stream_and_a_graph(aq):
    rng = np.random.default_rng(6)
    rope, _, _ = table(aq, (44, 42, 42), "paired")
    q, k = (S.bf16(rng.standard_normal((1, h, 300, 128))).cuda() for h in (4, 2))
    pos = i32(grid(1, 300, 3, rng, 500)[0])
    want = aq.attnqat_rope_fwd(q, k, pos, rope)
    out = tuple(torch.zeros_like(t) for t in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        aq.attnqat_rope_fwd(q, k, pos, rope, out=out)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        aq.attnqat_rope_fwd(q, k, pos, aq.rope_table((44, 42, 42)), out=out)             # (the table is gone after the call)
    for i in range(3):
        q.add_(0.25)
        pos.add_(i)
        want = aq.attnqat_rope_fwd(q, k, pos, rope)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("d,dims,layout", [(128, (44, 42, 42), "paired"), (64, (64,), "halves")])
def test_training_step(aq, d, dims, layout):
    """Q and K of one projection turned, attention and its gradient, and from there to the projection's gradient; then the same in a captured graph, the inputs new at every replay."""
    rng = np.random.default_rng(8)
    B, L, Hq, Hkv = 2, 200, 4, 2
    rope, freqs, axis = table(aq, dims, layout)
    pos = grid(1, L, len(dims), rng, 40)[0]
    pd = i32(pos)
    qkv, do = S.bf16(rng.standard_normal((B, L, Hq + 2 * Hkv, d))).cuda(), S.bf16(rng.standard_normal((B, Hq, L, d))).cuda()
    heads = lambda t, a, n: t[:, :, a:a + n].transpose(1, 2)  # noqa: E731
    kept = {}

    def step(grad):
        q, k = aq.attnqat_rope_fwd(heads(qkv, 0, Hq), heads(qkv, Hq, Hkv), pd, rope)
        v = heads(qkv, Hq + Hkv, Hkv).contiguous()
        o, lse, o_hp = aq.attnqat_fwd(q, k, v, True)
        dq, dk, dv = aq.attnqat_bwd(q, k, v, do, lse, o_hp, True)
        aq.attnqat_rope_bwd(dq, dk, pd, rope, out=(heads(grad, 0, Hq), heads(grad, Hq, Hkv)))
        heads(grad, Hq + Hkv, Hkv).copy_(dv)
        kept.update(q=q, k=k, dq=dq, dk=dk, dv=dv, o=o)

    grad = torch.full_like(qkv, 9.0)
    step(grad)
    rows = lambda t: t.transpose(1, 2)  # noqa: E731
    for b in range(B):
        check(rows(kept["q"])[b], qkv[b, :, :Hq], pos, freqs, axis, layout)
        check(rows(kept["k"])[b], qkv[b, :, Hq:Hq + Hkv], pos, freqs, axis, layout)
        check(grad[b, :, :Hq], rows(kept["dq"])[b], pos, freqs, axis, layout, -1.0)
        check(grad[b, :, Hq:Hq + Hkv], rows(kept["dk"])[b], pos, freqs, axis, layout, -1.0)
    assert torch.equal(grad[:, :, Hq + Hkv:], rows(kept["dv"]))
    graph, out = torch.cuda.CUDAGraph(), torch.full_like(qkv, 9.0)
    with torch.cuda.graph(graph):
        step(out)
    for i in range(4):
        qkv.mul_(0.875)
        pd.add_(i)
        step(grad)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, grad), i


def test_nothing_to_do(aq):
    rope, _, _ = table(aq, (64,), "paired")
    q = torch.zeros((2, 3, 0, 64), dtype=torch.bfloat16, device="cuda")
    y, k = aq.attnqat_rope_fwd(q, None, torch.zeros((0, 1), dtype=torch.int32, device="cuda"), rope)
    assert y.shape == q.shape and k is None


# ------------------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dims,layout,d", CASES)
@pytest.mark.parametrize("T,Hq,Hkv,how", [(1, 1, 1, "plain"), (40, 6, 3, "fused"), (131, 10, 5, "heads"), (7, 0, 4, "plain")])
def test_append(aq, dims, layout, d, T, Hq, Hkv, how):
    """The bytes of attnqat_rope_fwd followed by attnqat_kv_cache_append; rows outside the cache turn q and write nothing else."""
    from tests.test_gpu_serve import _slots, _views, dev
    rng = np.random.default_rng(T + d)
    rope, freqs, axis = table(aq, dims, layout)
    num = S.pages(T) + 2
    cache0 = rng.integers(0, 256, num * aq.kv_cache_page_bytes_nvfp4(Hkv, d), dtype=np.uint8)
    slots = dev(_slots(T, num, rng))
    pos = rng.integers(-100000, 100000, (T, len(dims))).astype(np.int32)
    q, k, v = (S.bf16(rng.standard_normal((T, h, d))).cuda() for h in (Hq, Hkv, Hkv))
    got, want = dev(cache0), dev(cache0)
    qo = aq.attnqat_kv_cache_append_rope(_views(q, how) if Hq else None, _views(k, how), _views(v, how), i32(pos), rope, got, slots, num_pages=num)
    rows = lambda x: x.transpose(0, 1)[None]  # noqa: E731
    kt, _ = aq.attnqat_rope_fwd(rows(k), None, i32(pos), rope)
    aq.attnqat_kv_cache_append(kt[0].transpose(0, 1).contiguous(), v, want, slots, num_pages=num)
    assert torch.equal(got, want)
    if Hq:
        check(qo, q, pos, freqs, axis, layout)
        qt, _ = aq.attnqat_rope_fwd(rows(q), None, i32(pos), rope)
        assert torch.equal(qo, qt[0].transpose(0, 1))
        fused = torch.cat([q, k, v], dim=1)                        # q turned where it lies, beside k and v
        a, b, c = fused.split([Hq, Hkv, Hkv], dim=1)
        got = dev(cache0)
        assert aq.attnqat_kv_cache_append_rope(a, b, c, i32(pos), rope, got, slots, num_pages=num, out=a) is a
        assert torch.equal(a, qo) and torch.equal(b, k) and torch.equal(c, v) and torch.equal(got, want)
    else:
        assert qo is None


def test_append_takes_the_positions_of_a_plan(aq):
    """int32 [T] for one axis; a step in which every row belongs to nobody leaves the cache as it was."""
    rng = np.random.default_rng(2)
    rope, freqs, axis = table(aq, (64,), "halves")
    q, k, v = (S.bf16(rng.standard_normal((9, h, 64))).cuda() for h in (4, 2, 2))
    cache = torch.zeros(2 * aq.kv_cache_page_bytes_nvfp4(2, 64), dtype=torch.uint8, device="cuda")
    pos = np.arange(9) + 70
    qo = aq.attnqat_kv_cache_append_rope(q, k, v, i32(pos), rope, cache, torch.full((9,), -1, dtype=torch.int64, device="cuda"))
    assert not bool(cache.any())
    check(qo, q, pos[:, None], freqs, axis, "halves")
    empty = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert aq.attnqat_kv_cache_append_rope(q[:0], k[:0], v[:0], i32(pos[:0]), rope, cache, empty).shape == (0, 4, 64)


def test_copied_tables(aq):
    """A copy of a table, one that went through a pickle and one whose entries were put in by hand turn as the table itself does, the original gone or not."""
    q, pos = S.bf16(np.random.default_rng(6).standard_normal((1, 3, 50, 64))).cuda(), i32(np.arange(50)[:, None] * 77)
    want, _ = aq.attnqat_rope_fwd(q, None, pos, aq.rope_table((64,)))
    first = aq.rope_table((64,))
    by_hand = aq.Rope(first.pairs, first.axes, first.layout, 0, first.turns, first.axis)
    for other in (copy.copy(first), copy.deepcopy(first), pickle.loads(pickle.dumps(first)), by_hand):
        first = None
        got, _ = aq.attnqat_rope_fwd(q, None, pos, other)
        assert torch.equal(got, want)


def test_binding_refuses(aq):
    rope = aq.rope_table((64,), layout="halves")
    q, k = (torch.zeros((1, h, 6, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    pos = i32(np.zeros((6, 1)))
    good = dict(q=q, k=k, positions=pos, rope=rope)
    aq.attnqat_rope_fwd(**good)
    for kw in (dict(q=q.float()), dict(q=q[0]), dict(k=k[:, :, :5]), dict(k=k.cpu()), dict(positions=pos.long()), dict(positions=pos[:5]), dict(positions=i32(np.zeros((6, 2)))),
               dict(rope=None), dict(q=q.transpose(2, 3)), dict(out=(q.float(), k)), dict(out=(k, q)), dict(out=(q, q[:, :2])), dict(rope=aq.rope_table((128,)))):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_rope_fwd(**{**good, **kw})
    rows = lambda h, T=6: torch.zeros((T, h, 64), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    cache, slots = torch.zeros(aq.kv_cache_page_bytes_nvfp4(2, 64), dtype=torch.uint8, device="cuda"), torch.arange(6, device="cuda")
    good = dict(q=rows(4), k=rows(2), v=rows(2), positions=pos, rope=rope, cache=cache, slots=slots)
    aq.attnqat_kv_cache_append_rope(**good)
    for kw in (dict(q=rows(4, 5)), dict(q=rows(4)[0]), dict(k=rows(2, 5)), dict(v=rows(3)), dict(positions=i32(np.zeros((6, 2)))), dict(positions=pos.long()), dict(slots=slots.int()),
               dict(cache=cache[:100]), dict(rope=3), dict(out=rows(3)), dict(out=rows(4).float()), dict(num_pages=2)):
        with pytest.raises(aq.AttnQatError):
            aq.attnqat_kv_cache_append_rope(**{**good, **kw})
