"""Attention and rotary positions as a program calls them: refusals of the binding, autograd, tensors past 32 bits, and a
run of them together on merged tokens."""

from __future__ import annotations

import pytest
import torch

import exact_attention as exact

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def mpm():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2604_05718_gb300 as pkg
    from paper_2604_05718_gb300 import build

    build.build()
    return pkg


def tensors(tq=20, tk=30, heads=4, kv=2, dim=32, dtype=torch.bfloat16, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(dtype)  # noqa: E731
    return new(tq, heads, dim), new(tk, kv, dim), new(tk, kv, dim), new(tq, heads, dim)


def test_refused_tensors(mpm):
    q, k, v, g = tensors()
    off = torch.tensor([0, 10, 20], device=DEV)
    both = dict(q_offsets=off, k_offsets=torch.tensor([0, 10, 30], device=DEV))
    cases = [
        ((q[0], k, v), {}), ((q.cpu(), k, v), {}), ((q, k[:, :, :16], v), {}), ((q, k, v[:5]), {}), ((q[:, :3], k, v), {}),
        ((q.transpose(1, 2), k, v), {}), ((q.expand(20, 4, 32)[:, :1].expand(20, 4, 32), k, v), {}),
        ((q, k, v), dict(q_offsets=off)), ((q, k, v), dict(both, k_offsets=off[:2])),
        ((q, k, v), dict(both, q_offsets=off.cpu())), ((q, k, v), dict(both, q_offsets=off[::2])),
        ((q, k, v), dict(key_mask=torch.ones(29, dtype=torch.bool, device=DEV))),
        ((q, k, v), dict(key_mask=torch.ones(30, dtype=torch.bool))), ((q, k, v), dict(out=torch.empty_like(q[:5]))),
        ((q, k, v), dict(out=torch.empty(20, 4, 64, dtype=q.dtype, device=DEV)[:, :, :32])),
        ((q, k, v), dict(device_status=torch.zeros(1, dtype=torch.int32, device=DEV))),
    ]
    for args, kw in cases:
        with pytest.raises(ValueError):
            mpm.cross_attention(*args, **kw)
    for args, kw in [((q.float(), k, v), {}), ((q.half(), k.half(), v.half()), {}), ((q, k, v), dict(both, q_offsets=off.int())),
                     ((q, k, v), dict(key_mask=torch.ones(30, device=DEV))),
                     ((q, k, v), dict(out=torch.empty(20, 4, 32, device=DEV)))]:
        with pytest.raises(TypeError):
            mpm.cross_attention(*args, **kw)
    for kw, code in ((dict(scale=0.0), 1), (dict(scale=-2.0), 1), (dict(out=q), 8),
                     (dict(workspace=torch.empty(0, dtype=torch.uint8, device=DEV), out=k.new_empty(q.shape)), None)):
        if code is None:
            mpm.cross_attention(q, k, v, **kw)                       # none is needed here
            continue
        with pytest.raises(mpm.MPMError) as e:
            mpm.cross_attention(q, k, v, **kw)
        assert e.value.code == code
    wide = torch.zeros(4, 2, 136, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(mpm.MPMError) as e:
        mpm.cross_attention(wide, wide, wide)
    assert e.value.code == 2
    out, stats = mpm.cross_attention(q, k, v, with_lse=True)
    for bad in (dict(d_out=g[:5]), dict(out=out[:5]), dict(stats=mpm.AttentionStats(stats.lse[:, :2], stats.rest)),
                dict(stats=mpm.AttentionStats(stats.lse, stats.rest[:5]))):
        with pytest.raises(ValueError):
            mpm.cross_attention_backward(**{**dict(d_out=g, q=q, k=k, v=v, out=out, stats=stats), **bad})


def test_refused_positions(mpm):
    x, at = torch.zeros(6, 2, 16, device=DEV), torch.zeros(6, 2, device=DEV)
    f = mpm.rotary_frequencies((2, 3))
    assert mpm.rotary(x, at, f, (2, 3)).shape == x.shape and mpm.rotary(x, at, f, [2, 3]).shape == x.shape
    for args, kw in [((x[0], at, f, (2, 3)), {}), ((x, at[:5], f, (2, 3)), {}), ((x, at.t().contiguous().t(), f, (2, 3)), {}),
                     ((x, at, f[:4], (2, 3)), {}), ((x, at, f, ()), {}), ((x, at, f, (0, 5)), {}), ((x, at, f, (4, 5)), {}),
                     ((x, at, f, (1,) * 9), {}), ((x, at, f, (2, 3)), dict(layout="pairs")), ((x, at, f.cpu(), (2, 3)), {}),
                     ((x, at, f, (2, 3)), dict(out=torch.empty(6, 2, 15, device=DEV)))]:
        with pytest.raises(ValueError):
            mpm.rotary(*args, **kw)
    for args, kw in [((x, at.double(), f, (2, 3)), {}), ((x, at, f.float(), (2, 3)), {}), ((x, at, f, 5), {}),
                     ((x, at, f, (2.5, 3)), {}), ((x.half(), at, f, (2, 3)), {}), ((x, at, f, (2, 3)), dict(layout=1)),
                     ((x, at, f, (2, 3)), dict(out=torch.empty(6, 2, 16, device=DEV, dtype=torch.bfloat16)))]:
        with pytest.raises(TypeError):
            mpm.rotary(*args, **kw)
    with pytest.raises(mpm.MPMError) as e:
        mpm.rotary(x[:, :1], at, f, (2, 3), out=x[:, 1:])            # interleaved with x: the same run of memory
    assert e.value.code == 8


@pytest.mark.parametrize("which", [0, 1, 2])
def test_inputs_that_require_grad(mpm, which):
    t = list(tensors()[:3])
    t[which].requires_grad_()
    with pytest.raises(ValueError, match="qkv"[which] + ".*grad"):
        mpm.cross_attention(*t)
    with torch.no_grad():
        mpm.cross_attention(*t)
    with pytest.raises(ValueError, match="x.*grad"):
        mpm.rotary(t[which], torch.zeros(t[which].shape[0], 1, device=DEV), mpm.rotary_frequencies((4,)), (4,))


def test_within_a_function_of_autograd(mpm):
    """Turned queries and keys, attention, and its gradients to the leaves, eager and with a graph of the same leaves alive."""
    q, k, v, g = tensors(100, 140, dtype=torch.float32)
    at_q, at_k = torch.rand(100, 2, device=DEV) * 30, torch.rand(140, 2, device=DEV) * 30
    f, sections = mpm.rotary_frequencies((6, 8)), (6, 8)

    class Attend(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            tq, tk = mpm.rotary(q, at_q, f, sections), mpm.rotary(k, at_k, f, sections)
            out, stats = mpm.cross_attention(tq, tk, v, with_lse=True)
            ctx.save_for_backward(tq, tk, v, out, stats.lse)
            return out

        @staticmethod
        def backward(ctx, d_out):
            tq, tk, v, out, lse = ctx.saved_tensors
            d_q, d_k, d_v = mpm.cross_attention_backward(d_out, tq, tk, v, out, mpm.AttentionStats(lse, None))
            return (mpm.rotary_backward(d_q, at_q, f, sections, out=d_q), mpm.rotary_backward(d_k, at_k, f, sections, out=d_k), d_v)

    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    out = Attend.apply(*leaves)
    got = torch.autograd.grad(out, leaves, g)
    again = torch.autograd.grad(Attend.apply(*leaves), leaves, g)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # The same by torch's own autograd in 64 bits.
    wide = [x.double().requires_grad_() for x in (q, k, v)]
    tq = exact.rotary(wide[0].detach(), at_q, f, sections, "halves")
    tk = exact.rotary(wide[1].detach(), at_k, f, sections, "halves")
    tq.requires_grad_(), tk.requires_grad_()
    kk, vv = tk.repeat_interleave(2, 1), wide[2].repeat_interleave(2, 1)
    p = torch.softmax(torch.einsum("ihd,jhd->hij", tq, kk) / 32 ** 0.5, dim=-1)
    ref = torch.einsum("hij,jhd->ihd", p, vv)
    d_tq, d_tk, d_v = torch.autograd.grad(ref, [tq, tk, wide[2]], g.double())
    want = [exact.rotary(d_tq, at_q, f, sections, "halves", True), exact.rotary(d_tk, at_k, f, sections, "halves", True), d_v]
    for a, b in zip(got, want):
        # Sums of up to 140 x 2 terms of size about 1 in fp32, angles to 2^-22: 2^-14 of the gradients' size is ample.
        assert (a.double() - b).abs().max() <= 2.0 ** -14 * b.abs().max()


def test_writes_in_place_are_new_versions(mpm):
    q, k, v, g = tensors()
    out = torch.empty_like(q)
    mpm.cross_attention(q, k, v, out=out)
    assert out._version == 1 and all(x._version == 0 for x in (q, k, v))
    with pytest.raises(mpm.MPMError):
        mpm.cross_attention(q, k, v, out=out, scale=-1.0)
    assert out._version == 1


@pytest.mark.parametrize("dtype, queries", [(torch.bfloat16, 2), (torch.bfloat16, 300), (torch.float32, 70)],
                         ids=["few", "tensor_cores", "f32"])
def test_positions_past_32_bits(mpm, dtype, queries):
    """Keys, values and their gradients behind 2^31 elements, in a sequence of their own."""
    heads, dim, keys = 16, 128, 333
    before = (1 << 31) // (heads * dim) + 5
    q, small_k, small_v, g = tensors(queries, keys, heads, heads, dim, dtype)
    k = torch.zeros(before + keys, heads, dim, dtype=dtype, device=DEV)
    v = torch.zeros(before + keys, heads, dim, dtype=dtype, device=DEV)
    k[before:], v[before:] = small_k, small_v
    off = dict(q_offsets=torch.tensor([0, 0, queries], device=DEV), k_offsets=torch.tensor([0, before, before + keys], device=DEV))
    small = dict(q_offsets=torch.tensor([0, 0, queries], device=DEV), k_offsets=torch.tensor([0, 0, keys], device=DEV))
    out, stats = mpm.cross_attention(q, k, v, with_lse=True, **off)
    want, want_stats = mpm.cross_attention(q, small_k, small_v, with_lse=True, **small)
    # How keys are shared out goes by the buffers' sizes, so sums may be taken in another order.
    exact_one = exact.attention(q, small_k, small_v, g, [0, queries], [0, keys], None, dim ** -0.5, probabilities=torch.bfloat16 if dtype == torch.bfloat16 else None)
    exact.check(out, exact_one.out, exact_one.out_bound, "out")
    exact.check(stats.lse, exact_one.lse, exact_one.lse_bound, "lse")
    grads = mpm.cross_attention_backward(g, q, k, v, out, stats, **off)
    exact.check(grads.d_q, exact_one.d_q, exact_one.d_q_bound, "d_q")
    exact.check(grads.d_k[before:], exact_one.d_k, exact_one.d_k_bound, "d_k")
    exact.check(grads.d_v[before:], exact_one.d_v, exact_one.d_v_bound, "d_v")
    assert not grads.d_k[:before].any() and not grads.d_v[:before].any()
    assert want.shape == out.shape and want_stats.lse.shape == stats.lse.shape


def test_merged_tokens(mpm):
    """A merge's padded outputs go in as they are: queries of a pooling head and of the tokens themselves."""
    counts, dim, heads = [300, 1, 700, 129], 128, 2
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(sum(counts), dim, generator=gen, device=DEV).to(torch.bfloat16)
    off = torch.tensor([0] + counts, device=DEV).cumsum(0)
    merged, off1, _ = mpm.merge(x, off)
    live = int(off1[-1])
    assert live < merged.shape[0]
    merged[live:] = float("nan")
    tokens = merged.view(-1, heads, dim // heads)
    at = torch.rand(merged.shape[0], 2, generator=gen, device=DEV) * 32
    f, sections = mpm.rotary_frequencies((8, 8)), (8, 8)
    turned = torch.full_like(tokens, 5.0)
    mpm.rotary(tokens, at, f, sections, offsets=off1, out=turned)
    assert (turned[live:] == 5).all()
    pool = torch.randn(len(counts), heads, dim // heads, generator=gen, device=DEV).to(torch.bfloat16)
    each = torch.arange(len(counts) + 1, device=DEV)
    host = off1.tolist()
    for q, qo in ((pool, each), (turned, off1)):
        out = torch.full_like(q, 9.0)
        _, stats = mpm.cross_attention(q, turned, tokens, q_offsets=qo, k_offsets=off1, out=out, with_lse=True)
        rows = int(qo[-1])
        assert (out[rows:] == 9).all()
        want = exact.attention(q[:rows], turned[:live], tokens[:live], q[:rows], qo.tolist(), host, None, (dim // heads) ** -0.5,
                               probabilities=torch.bfloat16)
        exact.check(out[:rows], want.out, want.out_bound, "out")
        g = torch.full_like(q, float("nan"))
        g[:rows] = q[:rows]
        grads = mpm.cross_attention_backward(g, q, turned, tokens, out, stats, q_offsets=qo, k_offsets=off1)
        exact.check(grads.d_q[:rows], want.d_q, want.d_q_bound, "d_q")
        exact.check(grads.d_k[:live], want.d_k, want.d_k_bound, "d_k")
        exact.check(grads.d_v[:live], want.d_v, want.d_v_bound, "d_v")


def test_the_padded_batch(mpm):
    """pad_batch's layout and mask, with offsets of equal lengths, against the packed tokens."""
    counts, heads, dim, longest = [40, 0, 100, 77], 4, 64, 100
    off = torch.tensor([0] + counts, device=DEV).cumsum(0)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(sum(counts), heads * dim, generator=gen, device=DEV).to(torch.bfloat16)
    padded, mask = mpm.pad_batch(x, off, longest)[:2]
    q = torch.randn(8, heads, dim, generator=gen, device=DEV).to(torch.bfloat16)
    two = torch.arange(5, device=DEV) * 2
    packed = x.view(-1, heads, dim)
    flat = padded.reshape(-1, heads, dim)
    a, sa = mpm.cross_attention(q, packed, packed, q_offsets=two, k_offsets=off, with_lse=True)
    b, sb = mpm.cross_attention(q, flat, flat, q_offsets=two, k_offsets=torch.arange(5, device=DEV) * longest,
                                key_mask=mask.reshape(-1), with_lse=True)
    assert (sa.lse[2:4] == -float("inf")).all() and (sb.lse[2:4] == -float("inf")).all()
    want = exact.attention(q, packed, packed, q, two.tolist(), off.tolist(), None, dim ** -0.5, probabilities=torch.bfloat16)
    exact.check(a, want.out, want.out_bound, "packed")
    exact.check(b, want.out, want.out_bound, "padded")
