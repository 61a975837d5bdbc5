"""Embedding lookup and the table's gradient against products and sums in 64 bits.

Tolerance of the lookup.  The product of two fp32 numbers has 48 bits, so it is exact in 64.  It is rounded to fp32, by at most u, and to its type, or to its type at once: the
compiler has an instruction that multiplies in fp32 and rounds to fp16 only.  Both are off by at most (u_T (1 + u) + u) of the product, or half the type's smallest number, and
u of it where the type is fp32; so (u_T + 2 u) |p| bounds them.  Without a scale there is nothing to round but the type.

Tolerance of the gradient.  u = 2^-24.  Whatever order n numbers are added in, the sum is off by at most (n - 1) u times the sum of their magnitudes (to first order);
the product with the scale adds u, an addition to what was there u of the result."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUNDING = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


@pytest.fixture(scope="module")
def rgc():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_1808_04357_amd as pkg
    pkg.load_library()
    return pkg


@pytest.fixture(scope="module")
def ctx(rgc):
    c = rgc.Context(1024, 1)
    yield c
    c.close()


def dtype_of(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def rows_of(n, width, dtype, strided, fill=math.nan):
    """[n, width] on the device, alone or as a part of wider rows at an odd place."""
    import torch
    if not strided:
        return torch.full((n, width), fill, dtype=dtype, device="cuda")
    return torch.full((n, 2 * width + 5), fill, dtype=dtype, device="cuda")[:, width + 1:2 * width + 1]


def check(rgc, ctx, tokens, vocab, width, dtype="f32", table_dtype="f32", scale=1.0, strided=False, add=False, stream=None, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed + vocab + width)
    rows = len(tokens)
    tokens = np.asarray(tokens, dtype=np.int32)
    table = torch.randn(vocab, width, generator=g).to(dtype_of(table_dtype))
    d_table, out = rows_of(vocab, width, table.dtype, strided), rows_of(rows, width, dtype_of(dtype), strided, 5.0)
    d_table.copy_(table)
    call = rgc.Embedding(d_table, torch.from_numpy(tokens).cuda(), out, scale=scale)
    known = (tokens >= 0) & (tokens < vocab)
    dout = torch.randn(rows, width, generator=g).to(dtype_of(dtype))
    dout[~torch.from_numpy(known)] = math.nan                  # not looked at
    d_dout = rows_of(rows, width, dout.dtype, strided)
    d_dout.copy_(dout)
    before = torch.randn(vocab, width, generator=g) if add else torch.full((vocab, width), 5.0)
    dtable = before.cuda()
    torch.cuda.synchronize()
    rgc.rgc_embed_tokens(ctx, call, stream)
    rgc.rgc_embed_tokens_backward(ctx, call, d_dout, dtable, rgc.RGC_ADD_TO_DST if add else rgc.RGC_OVERWRITE, stream)
    torch.cuda.synchronize()
    want = torch.zeros(rows, width, dtype=torch.float64)
    want[known] = table[tokens[known].astype(np.int64)].double() * float(np.float32(scale))
    if scale == 1.0:
        assert torch.equal(out.cpu(), want.to(out.dtype))
    assert bool(((out.cpu().double() - want).abs() <= (ROUNDING[dtype] + 2 * U) * want.abs() + SMALLEST[dtype] * (want != 0)).all())
    if strided:                                                # nothing beside the rows was written
        whole = out._base
        assert bool((whole[:, :width + 1] == 5.0).all()) and bool((whole[:, 2 * width + 1:] == 5.0).all())
    s = float(np.float32(scale))
    sums, sizes, n = np.zeros((vocab, width)), np.zeros((vocab, width)), np.zeros(vocab)
    d = dout.double().numpy()
    order = np.flatnonzero(known)
    np.add.at(sums, tokens[order], d[order])
    np.add.at(sizes, tokens[order], np.abs(d[order]))
    np.add.at(n, tokens[order], 1)
    got, b = dtable.double().cpu().numpy(), before.double().numpy()
    if add:
        assert np.array_equal(got[n == 0], b[n == 0])          # as they were
        wanted = b + s * sums
    else:
        assert not got[n == 0].any()
        wanted = s * sums
    slack = 1.01 * U * (abs(s) * sizes * np.maximum(n, 1)[:, None] + np.abs(wanted)) + 2.0 ** -140
    off = np.abs(got - wanted) > slack
    assert not off.any(), (np.argwhere(off)[0], got[off][0], wanted[off][0])
    return dtable


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32"), ("f32", "bf16"), ("f16", "bf16")]


@pytest.mark.parametrize("dtype,table_dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,width", [(1, 1, 1), (1, 10, 3), (2, 7, 4), (31, 5, 8), (32, 3, 65), (33, 100, 255), (64, 300, 1_500), (65, 40, 257), (700, 1_000, 513),
                                              (1_000, 70, 1_031)])
@pytest.mark.parametrize("strided", [False, True])
def test_sizes(rgc, ctx, dtype, table_dtype, rows, vocab, width, strided):
    g = np.random.default_rng(rows + width)
    check(rgc, ctx, g.integers(0, vocab, rows), vocab, width, dtype, table_dtype, 0.75, strided, add=rows % 2 == 0)


@pytest.mark.parametrize("rows,vocab,width", [(4_095, 300, 5), (4_096, 33_000, 3), (4_097, 255, 4), (4_097, 256, 4), (5_000, 257, 64), (20_000, 70_000, 6), (300_001, 1_000, 2),
                                              (9_000, 4_194_304, 1)])
@pytest.mark.parametrize("add", [False, True])
def test_many_rows(rgc, ctx, rows, vocab, width, add):
    g = np.random.default_rng(rows)
    tokens = np.minimum((np.exp(g.random(rows) * np.log(vocab + 1.0)) - 1).astype(np.int64), vocab - 1)
    tokens[g.random(rows) < 0.1] = -1
    check(rgc, ctx, tokens, vocab, width, "bf16", "f32", 2.5, add=add)


@pytest.mark.parametrize("rows", [10, 64, 1_000, 5_000])
def test_runs(rgc, ctx, rows):
    """One token for all, tokens in order, in the other order, each several segments long, and none that is known."""
    for tokens in (np.full(rows, 3), np.arange(rows) // 7, np.arange(rows)[::-1] // 40, np.arange(rows) % 2, np.full(rows, -1), np.full(rows, 2_000_000_000),
                   np.where(np.arange(rows) % 3 == 0, -(2 ** 31), 999)):
        check(rgc, ctx, tokens, 1_000, 70, "f16", "f16", add=False)
        check(rgc, ctx, tokens, 1_000, 70, "f32", "f32", -1.5, add=True)


def test_no_rows(rgc, ctx):
    import torch
    check(rgc, ctx, np.zeros(0, np.int32), 20, 9)
    check(rgc, ctx, np.zeros(0, np.int32), 20, 9, add=True)
    # RGC_OVERWRITE still clears the gradient
    dtable = torch.ones(20, 9, device="cuda")
    call = rgc.Embedding(torch.zeros(20, 9, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 9, device="cuda"))
    rgc.rgc_embed_tokens_backward(ctx, call, torch.zeros(0, 9, device="cuda"), dtable)
    assert not dtable.any()


def test_infinities_stay_in_their_rows(rgc, ctx):
    import torch
    table = torch.ones(4, 6, device="cuda")
    table[1, 2], table[2, 3] = math.inf, math.nan
    out = torch.empty(3, 6, device="cuda")
    call = rgc.Embedding(table, torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda"), out, scale=2.0)
    rgc.rgc_embed_tokens(ctx, call)
    assert out.tolist() == [[2.0] * 6, [2.0, 2.0, math.inf, 2.0, 2.0, 2.0], [0.0] * 6]
    dout, dtable = torch.ones(3, 6, device="cuda"), torch.empty(4, 6, device="cuda")
    dout[1, 4] = -math.inf
    rgc.rgc_embed_tokens_backward(ctx, call, dout, dtable)
    assert dtable.tolist() == [[2.0] * 6, [2.0, 2.0, 2.0, 2.0, -math.inf, 2.0], [0.0] * 6, [0.0] * 6]


def test_same_bits_every_time(rgc, ctx):
    g = np.random.default_rng(5)
    for rows in (900, 6_000):
        tokens = g.integers(0, 25, rows)
        first = check(rgc, ctx, tokens, 25, 130, "bf16", seed=1)
        for _ in range(3):
            assert bool((check(rgc, ctx, tokens, 25, 130, "bf16", seed=1) == first).all())


def test_a_gradient_of_one_row_for_all(rgc, ctx):
    """dout may be one row, expanded."""
    import torch
    dout, dtable = torch.randn(1, 40, device="cuda").expand(50, 40), torch.empty(3, 40, device="cuda")
    call = rgc.Embedding(torch.zeros(3, 40, device="cuda"), torch.ones(50, dtype=torch.int32, device="cuda"), torch.zeros(50, 40, device="cuda"))
    rgc.rgc_embed_tokens_backward(ctx, call, dout, dtable)
    assert torch.allclose(dtable[1], 50.0 * dout[0], rtol=50 * U, atol=0.0) and not dtable[0].any() and not dtable[2].any()


def test_a_table_longer_than_32_bits(rgc, ctx):
    import torch
    far = 2 ** 31 + 64
    memory = torch.empty(far + 100, dtype=torch.bfloat16, device="cuda")
    table = memory.as_strided((2, 100), (far, 1))
    table.copy_(torch.arange(200).view(2, 100))
    out = torch.empty(2, 100, dtype=torch.bfloat16, device="cuda")
    rgc.rgc_embed_tokens(ctx, rgc.Embedding(table, torch.tensor([1, 0], dtype=torch.int32, device="cuda"), out))
    assert torch.equal(out, table.flip(0))


def test_captured_and_on_another_stream(rgc, ctx):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    for rows in (200, 5_000):
        table, dout = torch.randn(50, 96, generator=g, device="cuda"), torch.randn(rows, 96, generator=g, device="cuda")
        tokens = torch.randint(-1, 50, (rows,), generator=g, device="cuda").to(torch.int32)
        out, dtable = torch.empty(rows, 96, device="cuda"), torch.empty(50, 96, device="cuda")
        call, stream = rgc.Embedding(table, tokens, out, scale=0.5), torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            rgc.rgc_embed_tokens(ctx, call, stream)
            rgc.rgc_embed_tokens_backward(ctx, call, dout, dtable, rgc.RGC_OVERWRITE, stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            rgc.rgc_embed_tokens(ctx, call, stream)
            rgc.rgc_embed_tokens_backward(ctx, call, dout, dtable, rgc.RGC_OVERWRITE, stream)
        for step in range(4):
            tokens.copy_(torch.randint(-1, 50, (rows,), generator=g, device="cuda"))
            dout.normal_(generator=g)
            out.fill_(7.0), dtable.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            eager_out, eager = torch.empty_like(out), torch.empty_like(dtable)
            again = rgc.Embedding(table, tokens, eager_out, scale=0.5)
            rgc.rgc_embed_tokens(ctx, again)
            rgc.rgc_embed_tokens_backward(ctx, again, dout, eager)
            torch.cuda.synchronize()
            assert torch.equal(out, eager_out) and torch.equal(dtable, eager)
            there = tokens >= 0
            want = torch.zeros(50, 96, dtype=torch.float64, device="cuda").index_add_(0, tokens[there].long(), dout[there].double()) * 0.5
            assert torch.allclose(dtable.double(), want, rtol=0.0, atol=1e-3)
        del graph


def test_refusals(rgc, ctx):
    import ctypes
    import torch
    from paper_1808_04357_amd import binding
    lib = rgc.load_library()
    table, out, tokens = torch.zeros(10, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    good = rgc.Embedding(table, tokens, out).desc

    def refused(**changes):
        a = binding.rgc_embedding.from_buffer_copy(good)
        for k, v in changes.items():
            setattr(a, k, v)
        return lib.rgc_embed_tokens(ctx.handle, ctypes.byref(a), None)

    assert refused() == 0
    for changes in (dict(rows=-1), dict(rows=2 ** 31), dict(vocab=0), dict(vocab=4_194_305), dict(width=0), dict(width=2 ** 21), dict(dtype=3), dict(table_dtype=-1),
                    dict(table=None), dict(out=None), dict(tokens=None), dict(out_stride=7), dict(table_stride=-1), dict(scale=math.inf), dict(scale=math.nan),
                    dict(table=good.table + 2), dict(tokens=good.tokens + 1), dict(out_stride=2 ** 60), dict(out=good.table, out_stride=8)):
        assert refused(**changes) == -1, changes
    dout, dtable = torch.zeros(4, 8, device="cuda"), torch.zeros(10, 8, device="cuda")
    call = rgc.Embedding(table, tokens, out)
    for flags in (0, rgc.RGC_OVERWRITE | rgc.RGC_ADD_TO_DST, 0x1):
        with pytest.raises(rgc.RgcError):
            rgc.rgc_embed_tokens_backward(ctx, call, dout, dtable, flags)
    for bad in (lambda: rgc.Embedding(table, tokens.long(), out), lambda: rgc.Embedding(table, tokens[:3], out), lambda: rgc.Embedding(table.t(), tokens, out),
                lambda: rgc.Embedding(table, tokens, out[:, :7]), lambda: rgc.Embedding(table.int(), tokens, out),
                lambda: rgc.rgc_embed_tokens_backward(ctx, call, dout.half(), dtable), lambda: rgc.rgc_embed_tokens_backward(ctx, call, dout, dtable.half()),
                lambda: rgc.rgc_embed_tokens_backward(ctx, call, dout, dtable[:9]), lambda: rgc.rgc_embed_tokens_backward(ctx, call, dtable[:4], dtable)):
        with pytest.raises(rgc.RgcError):
            bad()
    torch.cuda.synchronize()
