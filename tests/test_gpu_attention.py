"""cross_attention and its gradients against the 64-bit form, element by element, where they can go wrong."""

from __future__ import annotations

import math

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


def offsets(counts):
    got = [0]
    for n in counts:
        got.append(got[-1] + n)
    return got


def draw(gen, *shape, dtype, size=1.0):
    return (size * torch.randn(*shape, generator=gen, device=DEV)).to(dtype)


def problem(q_counts, k_counts, heads, kv_heads, dim, dtype, masked=0.0, seed=0, behind=(0, 0), size=1.0):
    """Tensors of a batch, with `behind` rows after the last sequence of either side; masked and such rows hold NaN."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    qo, ko = offsets(q_counts), offsets(k_counts)
    tq, tk = qo[-1] + behind[0], ko[-1] + behind[1]
    q, g = draw(gen, tq, heads, dim, dtype=dtype, size=size), draw(gen, tq, heads, dim, dtype=dtype)
    k, v = draw(gen, tk, kv_heads, dim, dtype=dtype, size=size), draw(gen, tk, kv_heads, dim, dtype=dtype)
    mask = None
    if masked > 0:
        mask = (torch.rand(tk, generator=gen, device=DEV) >= masked).to(torch.uint8)
        k[mask == 0], v[mask == 0] = float("nan"), float("inf")
    for x, n in ((q, qo[-1]), (g, qo[-1]), (k, ko[-1]), (v, ko[-1])):
        x[n:] = float("nan")
    return dict(q=q, k=k, v=v), g, dict(q_offsets=qo, k_offsets=ko), mask


def on_tensor_cores(q, k, v, g=None):
    """Whether the documentation promises the tensor cores: bf16 with 16-byte aligned rows and heads."""
    tensors = [x for x in (q, k, v, g) if x is not None]
    return all(x.dtype == torch.bfloat16 and x.data_ptr() % 16 == 0 and
               all(x.size(d) <= 1 or x.stride(d) % 8 == 0 for d in (0, 1)) for x in tensors)


def clean(x, mask, n):
    """Without what is masked or behind the sequences."""
    x = x.clone()
    x[n:] = 0
    if mask is not None:
        x[mask == 0] = 0
    return x


def run_and_check(mpm, t, g, off, mask, scale=None):
    q, k, v = t["q"], t["k"], t["v"]
    s = q.shape[2] ** -0.5 if scale is None else scale
    qo, ko = off["q_offsets"], off["k_offsets"]
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    got, stats = mpm.cross_attention(q, k, v, key_mask=mask, scale=scale, out=out, with_lse=True, device_status=status, **dev)
    assert got is out and (stats.rest is None) == (q.dtype == torch.float32)
    lse = stats.lse
    grads = mpm.cross_attention_backward(g, q, k, v, out, stats, key_mask=mask, scale=scale, device_status=status, **dev)
    assert status.tolist() == [0, 0]
    # Probabilities are bf16 on the tensor cores; a bound for fp32 ones is taken where the documentation says so.
    kind = torch.bfloat16 if on_tensor_cores(q, k, v, g) else torch.float32
    want = exact.attention(clean(q, None, qo[-1]), clean(k, mask, ko[-1]), clean(v, mask, ko[-1]), clean(g, None, qo[-1]), qo, ko,
                           mask, s, probabilities=kind)
    nq, nk = qo[-1], ko[-1]
    exact.check(out[:nq], want.out[:nq], want.out_bound[:nq], "out")
    exact.check(lse[:nq], want.lse[:nq], want.lse_bound[:nq], "lse")
    exact.check(grads.d_q[:nq], want.d_q[:nq], want.d_q_bound[:nq], "d_q")
    exact.check(grads.d_k[:nk], want.d_k[:nk], want.d_k_bound[:nk], "d_k")
    exact.check(grads.d_v[:nk], want.d_v[:nk], want.d_v_bound[:nk], "d_v")
    assert (out[nq:] == 7).all(), "rows behind the last sequence were written"
    return out, lse, grads


LENGTHS = {
    "one": ([1], [1]),
    "token": ([1, 1, 1], [5, 130, 0]),
    "few": ([3, 8, 2], [257, 64, 1000]),
    "tiles": ([128, 64, 256], [128, 64, 256]),
    "odd": ([130, 1, 0, 77, 300], [1, 129, 50, 0, 511]),
    "long_keys": ([40], [5000]),
    "long_queries": ([3000], [33]),
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_lengths(mpm, lengths, dim, dtype):
    q, k = LENGTHS[lengths]
    run_and_check(mpm, *problem(q, k, 2, 2, dim, dtype, behind=(3, 5), seed=dim))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dim", [1, 2, 7, 8, 24, 33, 40, 72, 80, 96, 127])
def test_head_widths(mpm, dim, dtype):
    run_and_check(mpm, *problem([70, 140], [150, 65], 2, 1, dim, dtype, seed=dim))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1), (6, 3), (8, 1), (12, 4)])
@pytest.mark.parametrize("lengths", [([1, 2], [300, 40]), ([190, 20], [140, 260])], ids=["few", "many"])
def test_shared_heads(mpm, lengths, heads, dtype):
    run_and_check(mpm, *problem(*lengths, *heads, 64, dtype, seed=heads[0]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dim", [40, 64, 128])
@pytest.mark.parametrize("masked", [0.1, 0.9, 1.0])
@pytest.mark.parametrize("lengths", [([1, 3], [200, 33]), ([150, 70, 1], [130, 3, 520])], ids=["few", "many"])
def test_masks(mpm, lengths, masked, dim, dtype):
    """Masked keys hold NaN and infinity; with all of them masked, rows are empty."""
    _, lse, grads = run_and_check(mpm, *problem(*lengths, 2, 2, dim, dtype, masked=masked, behind=(1, 1)))
    if masked == 1.0:
        assert (lse[:sum(lengths[0])] == -math.inf).all() and (grads.d_q[:sum(lengths[0])] == 0).all()


@pytest.mark.parametrize("queries", [20, 100, 140, 300])
@pytest.mark.parametrize("which", [(0, 1, 4), (0, 2, 4), (1, 3, 5), (0, 1, 2, 3, 4)])
def test_whole_tiles_that_are_masked(mpm, which, queries):
    t, g, off, _ = problem([queries], [700], 2, 2, 64, torch.bfloat16)
    mask = torch.ones(700, dtype=torch.bool, device=DEV)
    for tile in which:
        mask[128 * tile:128 * tile + 128] = False
    t["k"][~mask], t["v"][~mask] = float("nan"), float("nan")
    run_and_check(mpm, t, g, off, mask)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_scores_far_apart(mpm, dtype):
    """Maxima that grow by hundreds from tile to tile, and rows that one key decides."""
    t, g, off, mask = problem([130], [600], 1, 1, 64, dtype, size=4.0)
    t["k"][:] *= torch.linspace(0.05, 4.0, 600, device=DEV)[:, None, None].to(dtype)
    run_and_check(mpm, t, g, off, mask)
    t["k"] = t["k"].flip(0).contiguous()
    run_and_check(mpm, t, g, off, mask)


@pytest.mark.parametrize("scale", [1e-3, 1.0])
def test_scale(mpm, scale):
    run_and_check(mpm, *problem([100], [200], 2, 2, 64, torch.bfloat16), scale=scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["joint", "heads_first", "odd_rows", "shifted"])
def test_strides(mpm, kind, dtype):
    """Views: of a joint projection, of [H, T, D], of rows that are not 16-byte multiples, off by one element."""
    t, g, off, mask = problem([150, 61], [150, 61], 3, 3, 64, dtype)
    rows = 211

    def view(x):
        if kind == "joint":
            return torch.stack([x, x, x], 1)[:, 1]
        if kind == "heads_first":
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        if kind == "odd_rows":
            wide = torch.zeros(rows, 3 * 64 + 1, dtype=dtype, device=DEV)
            wide[:, :192] = x.reshape(rows, 192)
            return wide.as_strided((rows, 3, 64), (193, 64, 1))
        flat = torch.zeros(x.numel() + 1, dtype=dtype, device=DEV)
        flat[1:] = x.reshape(-1)
        return flat[1:].view(x.shape)
    t = {n: view(x) for n, x in t.items()}
    run_and_check(mpm, t, view(g), off, mask)


def test_one_row_and_one_head_with_odd_strides(mpm):
    """Strides that nothing goes by are not looked at."""
    t, g, off, mask = problem([1], [40], 1, 1, 64, torch.bfloat16)
    t["q"] = t["q"].as_strided((1, 1, 64), (3, 5, 1))
    run_and_check(mpm, t, g.as_strided((1, 1, 64), (7, 1, 1)), off, mask)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_without_offsets(mpm, dtype):
    t, g, off, _ = problem([77], [333], 4, 2, 64, dtype)
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    a, lse = mpm.cross_attention(t["q"], t["k"], t["v"], with_lse=True)
    b, _ = mpm.cross_attention(t["q"], t["k"], t["v"], **dev)
    assert torch.equal(a, b)
    x = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], a, lse)
    y = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], a, lse, **dev)
    assert all(torch.equal(i, j) for i, j in zip(x, y))


@pytest.mark.parametrize("shape", [(0, 5), (5, 0), (0, 0)])
def test_no_rows(mpm, shape):
    q, k = torch.zeros(shape[0], 2, 64, device=DEV), torch.zeros(shape[1], 2, 64, device=DEV)
    out, lse = mpm.cross_attention(q, k, k, with_lse=True)
    assert out.shape == q.shape and (out == 0).all() and (lse.lse == -math.inf).all()
    grads = mpm.cross_attention_backward(q, q, k, k, out, lse)
    assert all((x == 0).all() for x in grads) and grads.d_k.shape == k.shape


@pytest.mark.parametrize("heads", [(2, 2), (4, 1)])
@pytest.mark.parametrize("shape", [(0, 5), (5, 0), (0, 0), (300, 0), (0, 300)])
def test_no_rows_in_bf16(mpm, shape, heads):
    q = torch.zeros(shape[0], heads[0], 64, device=DEV, dtype=torch.bfloat16)
    k = torch.zeros(shape[1], heads[1], 64, device=DEV, dtype=torch.bfloat16)
    out, lse = mpm.cross_attention(q, k, k, with_lse=True)
    assert out.shape == q.shape and (out == 0).all() and (lse.lse == -math.inf).all()
    grads = mpm.cross_attention_backward(q, q, k, k, out, lse)
    assert all((x == 0).all() for x in grads) and grads.d_k.shape == k.shape


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("queries", [[3, 1, 9], [140, 300, 31]], ids=["few", "many"])
def test_one_key_a_sequence(mpm, queries, dim, dtype):
    """All weight on one key: gradients of q and k are 0 but for rounding."""
    run_and_check(mpm, *problem(queries, [1, 1, 1], 4, 2, dim, dtype, seed=dim))


@pytest.mark.parametrize("dim", [33, 64, 72, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_rows_of_any_alignment_over_many_tiles(mpm, dtype, dim):
    """Rows an odd number of elements apart: fp32's precision, in several tiles and parts either way."""
    t, g, off, mask = problem([700, 61], [200, 1100], 4, 2, dim, dtype, masked=0.2, seed=dim)
    odd = {}
    for name, x in t.items():
        odd[name] = torch.empty(x.shape[0], x.shape[1] * dim + 1, device=DEV, dtype=dtype)[:, :-1].view(x.shape[0], x.shape[1], dim)
        odd[name].copy_(x)
    run_and_check(mpm, odd, g, off, mask)


@pytest.mark.parametrize("where", ["q", "k", "v"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_nan_stays_with_what_it_touches(mpm, where, dtype):
    """A NaN in one sequence is seen in its rows, and in no other sequence's."""
    t, g, off, mask = problem([100, 90], [120, 140], 2, 2, 64, dtype)
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    clean_out, clean_lse = mpm.cross_attention(**t, with_lse=True, **dev)
    clean_grads = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], clean_out, clean_lse, **dev)
    t[where][3, 1, 5] = float("nan")
    out, lse = mpm.cross_attention(**t, with_lse=True, **dev)
    grads = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, lse, **dev)
    rows = slice(3, 4) if where == "q" else slice(0, 100)
    assert torch.isnan(out[rows, 1]).any(1).all()
    assert torch.equal(out[:, 0], clean_out[:, 0]) and torch.equal(out[100:], clean_out[100:])
    assert torch.equal(grads.d_q[100:], clean_grads.d_q[100:])
    assert torch.equal(grads.d_k[120:], clean_grads.d_k[120:]) and torch.equal(grads.d_v[120:], clean_grads.d_v[120:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lengths", [([1, 1], [3000, 500]), ([200, 31], [300, 260]), ([3000], [60])], ids=["few", "many", "keys"])
def test_the_same_bits_every_time(mpm, lengths, dtype):
    t, g, off, _ = problem(*lengths, 4, 2, 64, dtype)
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}

    def once():
        out, lse = mpm.cross_attention(**t, with_lse=True, **dev)
        return (out, lse.lse, *mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, lse, **dev))

    first = once()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, once()))


def test_given_workspaces_and_outputs(mpm):
    t, g, off, _ = problem([2], [4000], 4, 4, 64, torch.bfloat16)
    want, lse = mpm.cross_attention(**t, with_lse=True)
    ws = mpm.cross_attention_workspace(t["q"], t["k"])
    out = torch.empty_like(want)
    got, _ = mpm.cross_attention(**t, out=out, workspace=ws)
    assert got is out and torch.equal(out, want) and out._version == 1
    grads = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], want, lse)
    ws = mpm.cross_attention_workspace(t["q"], t["k"], backward=True)
    again = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], want, lse, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    with pytest.raises(mpm.MPMError) as e:
        mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], want, lse, workspace=ws[:ws.numel() - 256])
    assert e.value.code == 4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lengths", [([100, 17, 1, 64], [785, 197, 1, 0]), ([4000, 1, 0, 5], [3000, 2, 77, 400]), ([1, 1, 1], [9000, 3, 0])],
                         ids=["short", "long", "one"])
def test_nothing_is_read_that_was_not_written(mpm, lengths, dtype):
    """Workspaces full of NaN, where the sequences have unlike numbers of parts."""
    t, g, off, _ = problem(*lengths, 4, 2, 64, dtype)
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    out, stats = mpm.cross_attention(**t, with_lse=True, **dev)
    grads = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, stats, **dev)
    ws, back = (mpm.cross_attention_workspace(t["q"], t["k"], batch=len(lengths[0]), backward=b) for b in (False, True))
    for w in (ws, back):
        if w is not None:
            w.fill_(255)  # NaN in every type
    again, _ = mpm.cross_attention(**t, workspace=ws, **dev)
    assert torch.equal(out, again)
    dirty = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, stats, workspace=back, **dev)
    assert all(torch.equal(a, b) for a, b in zip(grads, dirty))
    run_and_check(mpm, t, g, off, None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lengths", [([1], [2000]), ([300, 40], [280, 120])], ids=["few", "many"])
def test_a_captured_graph_follows_its_inputs(mpm, lengths, dtype):
    """Lengths, tokens and masks of a later replay, while an eager call runs between."""
    t, g, off, _ = problem(*lengths, 4, 2, 64, dtype)
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    mask = torch.ones(sum(lengths[1]), dtype=torch.uint8, device=DEV)

    def step():
        out, lse = mpm.cross_attention(**t, key_mask=mask, with_lse=True, **dev)
        return (out, lse.lse, *mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, lse, key_mask=mask, **dev))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = step()
    for seed in (1, 2):
        fresh, g2, _, _ = problem(*lengths, 4, 2, 64, dtype, seed=seed)
        for n, x in fresh.items():
            t[n].copy_(x)
        g.copy_(g2)
        mask[::3] = seed % 2
        if len(lengths[1]) > 1:
            dev["k_offsets"][1] = 10 * seed
        eager = [x.clone() for x in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, made))


def test_two_streams_at_once(mpm):
    t, g, off, _ = problem([1, 300], [3000, 200], 4, 4, 64, torch.bfloat16)
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    want, lse = mpm.cross_attention(**t, with_lse=True, **dev)
    grads = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], want, lse, **dev)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                out, l = mpm.cross_attention(**t, with_lse=True, **dev)
                got.append((out, *mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, l, **dev)))
    torch.cuda.synchronize()
    assert all(torch.equal(x[0], want) and all(torch.equal(a, b) for a, b in zip(x[1:], grads)) for x in got)


@pytest.mark.parametrize("which", ["q_offsets", "k_offsets"])
@pytest.mark.parametrize("bad", [[0, 300, 80], [5, 50, 80], [0, 50, 999], [-4, 50, 80]])
def test_bad_offsets_are_reported(mpm, which, bad):
    t, g, off, _ = problem([50, 30], [50, 30], 2, 2, 64, torch.bfloat16)
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    dev[which] = torch.tensor(bad, device=DEV)
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    out, lse = mpm.cross_attention(**t, with_lse=True, device_status=status, **dev)
    assert status[0] == 6
    status.zero_()
    mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, lse, device_status=status, **dev)
    assert status[0] == 6


def test_gradients_against_differences(mpm):
    """d/dx of sum(out * g) by central differences in fp32, along random directions."""
    t, g, off, mask = problem([20, 9], [31, 14], 4, 2, 32, torch.float32, masked=0.2)
    mask_ok = mask != 0
    for n in ("k", "v"):
        t[n][~mask_ok] = 0
    dev = {n: torch.tensor(o, device=DEV) for n, o in off.items()}
    out, lse = mpm.cross_attention(**t, key_mask=mask, with_lse=True, **dev)
    grads = mpm.cross_attention_backward(g, t["q"], t["k"], t["v"], out, lse, key_mask=mask, **dev)
    gen = torch.Generator(device=DEV).manual_seed(5)
    for n, grad in zip(("q", "k", "v"), grads):
        step = torch.randn(t[n].shape, generator=gen, device=DEV)
        h = 1e-2
        ends = []
        for sign in (1, -1):
            moved = dict(t)
            moved[n] = t[n] + sign * h * step
            ends.append((mpm.cross_attention(**moved, key_mask=mask, **dev)[0].double() * g.double()).sum())
        want, got = (ends[0] - ends[1]) / (2 * h), (grad.double() * step.double()).sum()
        # The third derivative's part is h^2 / 6 of it, of the size of the terms' own sum; differences lose 2^-20 / h.
        size = (grad.double().abs() * step.double().abs()).sum()
        assert abs(want - got) <= size * (h * h + 2.0 ** -20 / h), n


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("shape", [(300, 160, 400), (700, 1, 300), (40, 1000, 1100)], ids=["one_or_two_tiles", "any", "many_tiles"])
def test_many_sequences_a_block(mpm, shape, dim):
    """More work items than SMs, of one and of two tiles of queries in turn: places and barriers are used over and over."""
    batch, low, high = shape
    gen = torch.Generator().manual_seed(batch)
    q = torch.randint(low, high, (batch,), generator=gen).tolist()
    k = torch.randint(low, high, (batch,), generator=gen).tolist()
    run_and_check(mpm, *problem(q, k, 2, 2, dim, torch.bfloat16, masked=0.1 if dim == 128 else 0.0))
