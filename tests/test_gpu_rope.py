"""skvq_rope_apply against the rotation in 64 bits: types, pair layouts, partial heads, strides and orders, positions far
out and negative, in place, the gradient; what it refuses; a captured and replayed call."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2405_06219_amd import binding
    return binding


def plain(x, positions, rope, rotary, interleaved, transpose=False):
    """x [B][T][H][d] (64 bits), positions [B][T]: the rotation, and the sizes |a| + |b| that its error goes by."""
    f, amplitude = rope.skvq_rope_frequencies()
    half = rotary // 2
    # turns in 64 bits of mantissa: a far position times a frequency keeps its fraction
    turns = positions[..., None].astype(np.longdouble) * (f.astype(np.longdouble) / (2 * np.longdouble("3.14159265358979323846264338327950288")))
    angle = ((turns - np.rint(turns)) * 2 * np.longdouble("3.14159265358979323846264338327950288"))
    c, s = (np.cos(angle) * amplitude).astype(np.float64)[:, :, None], (np.sin(angle) * amplitude).astype(np.float64)[:, :, None]
    s = -s if transpose else s
    first, second = ((slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, half), slice(half, rotary)))
    y, size = x.copy(), np.zeros_like(x)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size[..., first] = size[..., second] = (np.abs(a) + np.abs(b)) * amplitude
    return y, size


def check(got, x, positions, rope, rotary, interleaved, transpose=False):
    """Cosine, sine, the products and the sum round to fp32 (2^-24 of |a| + |b| each at most: three in a row), the result
    to its type (half a step)."""
    want, size = plain(x.double().cpu().numpy(), positions, rope, rotary, interleaved, transpose)
    err = 3 * 2.0 ** -24 * size
    bound = err + torch.finfo(x.dtype).eps / 2 * (np.abs(want) + err) + 2.0 ** -25 * (x.dtype == torch.float16)
    bound[size == 0] = 0
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= bound).all(), float((off - bound).max())


def tensor(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


SHAPES = [(1, 1, 4, 2), (2, 5, 8, 1), (3, 67, 3, 3), (1, 4100, 2, 1)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 64), (64, 32), (96, 48), (80, 20), (256, 256), (6, 2), (10, 10)])
@pytest.mark.parametrize("shape", SHAPES)
def test_types_and_heads(B, dtype, layout, d, rotary, shape):
    b, t, hq, hk = shape
    rope = B.SkvqRope(d, rotary, layout, 10000.0)
    q, k = tensor((b, t, hq, d), dtype, 1), tensor((b, t, hk, d), dtype, 2)
    oq, ok = rope.skvq_rope_apply(q, k, start=11)
    positions = np.broadcast_to(np.arange(t) + 11, (b, t))
    check(oq, q, positions, rope, rotary, layout == "interleaved")
    check(ok, k, positions, rope, rotary, layout == "interleaved")
    only = rope.skvq_rope_apply(q, start=11)
    assert torch.equal(only, oq)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("scaling", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=2.0),
                                     dict(scaling="yarn", factor=4.0, original_context=4096, low=1.0, high=32.0),
                                     dict(scaling="bands", factor=8.0, original_context=8192, low=1.0, high=4.0, amplitude=0.75)])
def test_positions_far_out(B, dtype, scaling):
    rope = B.SkvqRope(128, 128, "half", 10000.0, **scaling)
    far = np.array([[0, 1, -1, 4095, 1 << 20, (1 << 31) - 1, -(1 << 31), 123456789]], np.int32)
    x = tensor((2, 8, 3, 128), dtype, 3)
    both = np.concatenate([far, far[:, ::-1]])
    check(rope.skvq_rope_apply(x, positions=torch.from_numpy(both).to(DEV)), x, both, rope, 128, False)
    # one row of positions for all sequences; rows of a wider table
    check(rope.skvq_rope_apply(x, positions=torch.from_numpy(far[0]).to(DEV)), x, np.broadcast_to(far, (2, 8)), rope, 128, False)
    wide = torch.from_numpy(np.concatenate([both, both], 1)).to(DEV)
    check(rope.skvq_rope_apply(x, positions=wide[:, 8:]), x, both, rope, 128, False)
    check(rope.skvq_rope_apply(x, start=2 ** 31 - 8), x, np.broadcast_to(np.arange(8) + 2 ** 31 - 8, (2, 8)), rope, 128, False)
    check(rope.skvq_rope_apply(x, start=-2 ** 31), x, np.broadcast_to(np.arange(8) - 2 ** 31, (2, 8)), rope, 128, False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rotary", [128, 64])
def test_orders_and_strides(B, dtype, layout, rotary):
    rope = B.SkvqRope(128, rotary, layout)
    il = layout == "interleaved"
    positions = np.broadcast_to(np.arange(37), (2, 37))
    rows = tensor((2, 37, 7, 128), dtype, 4)                       # a fused projection: 4 query, 2 key, 1 value heads
    q, k = rows[:, :, :4], rows[:, :, 4:6]
    heads_first = torch.full((2, 4, 37, 128), 7.0, dtype=dtype, device=DEV)
    oq, ok = rope.skvq_rope_apply(q, k, out_q=heads_first.transpose(1, 2))
    check(oq, q, positions, rope, rotary, il)
    check(ok, k, positions, rope, rotary, il)
    assert oq.data_ptr() == heads_first.data_ptr()
    # rows that begin off 16 bytes: one channel at a time, the same values, nothing beside them
    wide = torch.full((2, 37, 4, 131), 3.0, dtype=dtype, device=DEV)
    rope.skvq_rope_apply(q, out_q=wide[..., 1:129])
    assert torch.equal(wide[..., 1:129], oq) and bool((wide[..., 0] == 3).all()) and bool((wide[..., 129:] == 3).all())
    # in place, the value head untouched
    before = rows.clone()
    rope.skvq_rope_apply(q, k, out_q=q, out_k=k)
    assert torch.equal(rows[:, :, :4], oq) and torch.equal(rows[:, :, 4:6], ok) and torch.equal(rows[:, :, 6], before[:, :, 6])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rotary", [(128, 128), (96, 48), (10, 6)])
def test_gradient(B, layout, d, rotary):
    rope = B.SkvqRope(d, rotary, layout, scaling="yarn", factor=4.0, original_context=64, low=1.0, high=8.0)
    x, g = tensor((2, 9, 2, d), torch.float32, 5), tensor((2, 9, 2, d), torch.float32, 6)
    positions = np.broadcast_to(np.arange(9) + 3, (2, 9))
    dx = rope.skvq_rope_apply(g, start=3, transpose=True)
    check(dx, g, positions, rope, rotary, layout == "interleaved", transpose=True)
    # the formula's gradient by differences in 64 bits: the call is linear, so one step of any size is exact
    rng = np.random.default_rng(7)
    for _ in range(5):
        at = tuple(int(rng.integers(n)) for n in x.shape)
        x64, e = x.double().cpu().numpy(), np.zeros(x.shape)
        e[at] = 1.0
        hi, lo = (plain(x64 + s * e, positions, rope, rotary, layout == "interleaved")[0] for s in (0.5, -0.5))
        want = float(((hi - lo) * g.double().cpu().numpy()).sum())
        # (three fp32 steps of two members of the pair, the result's own, and the differences' in 64 bits)
        assert abs(float(dx[at]) - want) <= 2.0 ** -21 * 2 * float(g.abs().max()) * 1.5


def test_refusals_of_tensors(B):
    rope = B.SkvqRope(128)
    x = tensor((2, 3, 4, 128), torch.float16, 8)
    for bad in (dict(q=x.double()), dict(q=x[..., :64]), dict(q=x.transpose(2, 3)), dict(q=x, k=x.float()), dict(q=x, k=x[:1]),
                dict(q=x, out_q=x.float()), dict(q=x, out_q=x[:, :2]), dict(q=x, positions=torch.zeros(4, dtype=torch.int32, device=DEV)),
                dict(q=x, positions=torch.zeros(3, dtype=torch.int64, device=DEV)), dict(q=x, positions=torch.zeros(3, dtype=torch.int32)),
                dict(q=x.cpu())):
        with pytest.raises(ValueError):
            rope.skvq_rope_apply(**bad)
    with pytest.raises(B.SkvqError) as e:
        rope.skvq_rope_apply(x, start=2 ** 31 - 2)
    assert e.value.status == B.SKVQ_ERR_INVALID_ARG
    with pytest.raises(B.SkvqError):    # in place with other strides
        rope.skvq_rope_apply(x[:, :2], out_q=x.view(-1)[:2 * 2 * 4 * 128].view(2, 2, 4, 128))
    for shape in ((0, 3, 4, 128), (2, 0, 4, 128), (2, 3, 0, 128)):
        assert rope.skvq_rope_apply(tensor(shape, torch.float16, 9)).shape == shape


def test_captured_calls_follow_their_positions(B):
    rope = B.SkvqRope(128, scaling="ntk", factor=2.0)
    x, out = tensor((1, 6, 4, 128), torch.bfloat16, 10), torch.empty((1, 6, 4, 128), dtype=torch.bfloat16, device=DEV)
    at = torch.arange(6, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        rope.skvq_rope_apply(x, positions=at, out_q=out)
        graph.capture_begin()
        rope.skvq_rope_apply(x, positions=at, out_q=out)
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    for step in range(4):
        at.copy_(torch.arange(6, dtype=torch.int32) + 1000 * step)
        x.add_(0.125)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, rope.skvq_rope_apply(x, start=1000 * step))
