"""Token embedding against 64 bits: lookup, and the table's gradient with its fixed order."""
import pytest
import torch

import paper_1907_12205_b200 as dx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES}
U = 2.0 ** -24                                     # fp32's rounding
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}   # half a subnormal step


def matrix(rows, cols, pad, dtype, seed=0, offset=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    flat = torch.randn(rows * (cols + pad) + offset, generator=gen, device=DEV).to(dtype)
    return flat[offset:].view(rows, cols + pad)[:, :cols]


def as_bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols,pad,offset", [(1, 1, 1, 0, 0), (1, 300, 2048, 0, 0), (7, 50, 64, 8, 0), (33, 129, 257, 0, 0),
                                                        (130, 1000, 1000, 3, 1), (70, 40, 2049, 7, 3), (513, 77, 128, 0, 0)])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_lookup(dtype, rows, vocab, cols, pad, offset, index):
    w = matrix(vocab, cols, pad, dtype, 1, offset)
    tokens = torch.randint(0, vocab, (rows,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).to(index)
    tokens[0] = vocab - 1
    y = dx.detox_embedding(tokens, w, scale=2.75)
    want = w.double()[tokens.long()] * 2.75        # one fp32 product, then the type's rounding
    assert y.dtype == dtype and y.shape == (rows, cols)
    assert bool(((y.double() - want).abs() <= want.abs() * (HALF[dtype] + U) * 1.001 + TINY[dtype]).all())
    assert torch.equal(as_bits(dx.detox_embedding(tokens, w)), as_bits(w[tokens.long()]))   # scale 1: the rows themselves


@pytest.mark.parametrize("dtype", TYPES)
def test_padding_and_tokens_outside_the_vocabulary(dtype):
    w = matrix(20, 72, 0, dtype)
    w[3, 5] = float("inf")
    tokens = torch.tensor([-1, 3, 20, -2 ** 31, 2 ** 31 - 1, 19, 0], device=DEV, dtype=torch.int32)
    y = dx.detox_embedding(tokens, w, out=torch.full((7, 80), 9.0, device=DEV, dtype=dtype)[:, :72])
    assert bool((y[[0, 3]] == 0).all()) and bool(y[[2, 4]].isnan().all())
    assert torch.equal(y[[1, 5, 6]], w[[3, 19, 0]])
    far = torch.tensor([2 ** 40, -2 ** 40, 2 ** 32, 5], device=DEV)   # their low 32 bits are tokens
    y = dx.detox_embedding(far, w)
    assert bool(y[[0, 2]].isnan().all()) and bool((y[1] == 0).all()) and torch.equal(y[3], w[5])
    dy = matrix(4, 72, 0, dtype, 3)
    dw = dx.detox_embedding_backward(dy, far, 20)
    assert torch.equal(dw[5], dy[3]) and int((dw != 0).any(1).sum()) == 1


def gradient_bound(dy, tokens, vocab, scale, start=None):
    """The sums in 64 bits, and how far fp32 sums in any order may be off before they are rounded to their type: a rounding for each addition, one for the product."""
    keep = (tokens >= 0) & (tokens < vocab)
    t, d = tokens[keep].long(), dy.double()[keep]
    sums = torch.zeros((vocab, dy.shape[1]), dtype=torch.float64, device=DEV).index_add_(0, t, d * scale)
    size = torch.zeros_like(sums).index_add_(0, t, d.abs() * abs(scale))
    count = torch.bincount(t, minlength=vocab).double()[:, None]
    if start is not None:
        sums, size = sums + start.double(), size + start.double().abs()
    return sums, size * (2 * count + 3) * U, count[:, 0]


CASES = [(1, 1, 1), (5, 3, 8), (40, 7, 64), (100, 500, 72), (1000, 129, 257), (3000, 2000, 512), (17, 5000, 1030), (4096, 3, 96), (2500, 140000, 16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols", CASES)
@pytest.mark.parametrize("wide,add", [(False, False), (True, False), (False, True), (True, True)])
def test_gradient(dtype, rows, vocab, cols, wide, add):
    gen = torch.Generator(device=DEV).manual_seed(rows + vocab)
    # tokens as uneven as words: the first one takes up to a half
    tokens = (torch.rand(rows, generator=gen, device=DEV) ** 6 * vocab).long().clamp_(max=vocab - 1)
    tokens[torch.rand(rows, generator=gen, device=DEV) < 0.1] = -1
    out = torch.float32 if wide else dtype
    for pad, offset in ((0, 0), (3, 1)):
        dy = matrix(rows, cols, pad, dtype, 1, offset)
        dw = matrix(vocab, cols, pad, out, 2, offset)
        want, off, count = gradient_bound(dy, tokens, vocab, 1.5, dw if add else None)
        before = dw.clone()
        got = dx.detox_embedding_backward(dy, tokens.to(torch.int32), vocab, scale=1.5, dw=dw, accumulate=add)
        assert got.data_ptr() == dw.data_ptr()
        assert bool(((got.double() - want).abs() <= off + want.abs() * HALF[out] * 1.001 + TINY[out]).all())
        none = count == 0
        assert torch.equal(got[none], before[none] if add else torch.zeros_like(got[none]))
        again = dx.detox_embedding_backward(dy, tokens, vocab, scale=1.5, dw=before.clone() if add else None, dw_dtype=out, accumulate=add)
        assert torch.equal(as_bits(again), as_bits(got))                 # the same bits, whatever the layout and the index's type


@pytest.mark.parametrize("what", ["one token", "two tokens in turn", "all padding", "all beyond", "each once, backwards"])
@pytest.mark.parametrize("rows", [1, 9, 255, 5000])
def test_gradient_of_uneven_tokens(what, rows):
    vocab, cols = max(rows, 40), 300
    tokens = {"one token": lambda: torch.full((rows,), 17), "two tokens in turn": lambda: torch.arange(rows) % 2 * 38,
              "all padding": lambda: torch.full((rows,), -1), "all beyond": lambda: torch.full((rows,), vocab),
              "each once, backwards": lambda: torch.arange(rows).flip(0)}[what]().to(DEV)
    dy = matrix(rows, cols, 0, torch.bfloat16)
    want, off, count = gradient_bound(dy, tokens, vocab, 1.0)
    for add in (False, True):
        dw = torch.zeros((vocab, cols), device=DEV) if add else torch.full((vocab, cols), 7.0, device=DEV)
        dx.detox_embedding_backward(dy, tokens, vocab, dw=dw, accumulate=add)
        assert bool(((dw.double() - want).abs() <= off + want.abs() * HALF[torch.float32]).all())


def test_no_rows():
    dy, tokens = torch.empty((0, 24), device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    assert dx.detox_embedding(tokens, matrix(5, 24, 0, torch.float32)).shape == (0, 24)
    dw = torch.full((5, 24), 3.0, device=DEV)
    dx.detox_embedding_backward(dy, tokens, 5, dw=dw, accumulate=True)
    assert bool((dw == 3).all())
    assert bool((dx.detox_embedding_backward(dy, tokens, 5, dw=dw) == 0).all())


def test_gradient_against_differences():
    """dW of sum(c * Y) by the definition: Y is linear in W, so a difference is exact but for its roundings."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    w, c = torch.randn((11, 24), generator=gen, device=DEV), torch.randn((60, 24), generator=gen, device=DEV)
    tokens = torch.randint(-1, 11, (60,), generator=gen, device=DEV)
    dw = dx.detox_embedding_backward(c, tokens, 11, scale=0.5)
    for v, k in ((0, 0), (3, 7), (10, 23)):
        step = torch.zeros_like(w)
        step[v, k] = 1.0
        up, down = (dx.detox_embedding(tokens, w + s * step, scale=0.5).double() for s in (1, -1))
        diff = float(((up - down) * c.double()).sum() / 2)
        assert abs(diff - float(dw[v, k])) <= 60 * 4 * U * 4 * float(c.abs().max()) * (1 + float(w.abs().max()))


def test_outside_and_behind_nothing_is_written():
    """Columns behind a row's last one, rows behind the last, bytes behind the workspace."""
    rows, vocab, cols = 333, 100, 203
    tokens = torch.randint(0, vocab, (rows,), device=DEV)
    dy = matrix(rows, cols, 5, torch.bfloat16)
    buffer = torch.full((vocab + 2, 211), 7.0, device=DEV)
    size = dx.detox_embedding_backward_workspace_bytes(rows, vocab, cols)
    ws = torch.full((size + 512,), 0x5A, dtype=torch.uint8, device=DEV)
    dx.detox_embedding_backward(dy, tokens, vocab, dw=buffer[1:-1, :cols], ws=ws[256:256 + size])
    assert bool((buffer[[0, -1]] == 7).all()) and bool((buffer[:, cols:] == 7).all())
    # (7 itself is a sum that bf16 rows can have, so written rows are told by a call without a buffer)
    assert torch.equal(buffer[1:-1, :cols], dx.detox_embedding_backward(dy, tokens, vocab, dw_dtype=torch.float32))
    assert bool((ws[:256] == 0x5A).all()) and bool((ws[256 + size:] == 0x5A).all())
    out = torch.full((rows + 2, 211), 7.0, device=DEV, dtype=torch.bfloat16)
    dx.detox_embedding(tokens, matrix(vocab, cols, 0, torch.bfloat16), out=out[1:-1, :cols])
    assert bool((out[[0, -1]] == 7).all()) and bool((out[:, cols:] == 7).all())


def test_offsets_beyond_32_bits():
    """A table and a gradient of more than 2^31 entries."""
    vocab, cols = 140_000, 16384
    w = torch.empty((vocab, cols), dtype=torch.bfloat16, device=DEV)
    w[[0, 131_072, vocab - 1]] = matrix(3, cols, 0, torch.bfloat16)
    tokens = torch.tensor([vocab - 1, 131_072, 0, vocab - 1], device=DEV)
    assert torch.equal(dx.detox_embedding(tokens, w), w[tokens])
    dy = matrix(4, cols, 0, torch.bfloat16, 4)
    dx.detox_embedding_backward(dy, tokens, vocab, dw=w)
    assert torch.equal(w[131_072], dy[1]) and torch.equal(w[0], dy[2])
    assert torch.equal(w[vocab - 1], (dy[0].float() + dy[3].float()).to(torch.bfloat16))
    assert bool((w[1:131_072:997] == 0).all()) and bool((w[131_073:vocab - 1:97] == 0).all())
