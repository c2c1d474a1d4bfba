"""The MXFP4 operators on the GPU against their definition in 64 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_1910_06188_b200 import binding as q8
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
NAMES = {torch.float32: "fp32", torch.float16: "fp16", torch.bfloat16: "bf16"}


def values(shape, seed, dtype=torch.float32, spread=2.0):
    """Blocks of very different magnitude, an outlier here and there."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    x = x * torch.exp(spread * torch.randn((*shape[:-1], 1), generator=g)).clamp(1e-2, 1e2)
    x = x * (1 + 7 * (torch.rand(shape, generator=g) < 0.02))
    return x.to(dtype).cuda()


def weights(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return (0.02 * torch.randn(shape, generator=g)).cuda()


def status_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def check_codes(t, x, group=0):
    code, E, blocks = ref.unpack(t, group)
    want_code, want_E = ref.quantize(ref.as_numpy(x))
    assert np.array_equal(E[:, :blocks], want_E)
    assert not E[:, blocks:].any(), "scales behind the last block"
    assert np.array_equal(code[:, :32 * blocks], want_code) and not code[:, 32 * blocks:].any()


# ---------------------------------------------------------------- quantisation
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (3, 33), (31, 256), (33, 257), (100, 31), (128, 128), (129, 1000), (300, 4104)])
def test_quantize(rows, K, dtype):
    x = values((rows, K), rows + K, dtype)
    word = status_word()
    t = q8.q8_mx4_quantize(x, dev_status=word)
    assert t.tiles.numel() == q8.q8_mx4_bytes(1, rows, K) and t.shape == (rows, K)
    check_codes(t, x)
    assert word.item() == 0
    for out in TYPES:
        got = q8.q8_mx4_dequantize(t, out)
        assert got.dtype == out and torch.equal(got.double().cpu(), torch.from_numpy(ref.rounded(x)).to(out).double())


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("offset,ld", [(0, 600), (8, 616), (1, 601), (3, 640)])
def test_quantize_rows_of_a_wider_tensor(offset, ld, dtype):
    x = values((70, ld), ld, dtype)[:, offset:offset + 520]
    check_codes(q8.q8_mx4_quantize(x), x)


@pytest.mark.parametrize("shape", [(3, 5, 40), (2, 128, 256), (4, 200, 130)])
def test_quantize_groups(shape):
    x = values(shape, 7)
    t = q8.q8_mx4_quantize(x)
    back = q8.q8_mx4_dequantize(t)
    for g in range(shape[0]):
        check_codes(t, x[g], g)
        assert np.array_equal(ref.as_numpy(back[g]), ref.rounded(x[g]))


def test_quantize_ties_and_borders():
    steps = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.9999995])
    rows = []
    for s in (1.0, 2.0 ** -20, 2.0 ** 90):
        for sign in (1, -1):
            row = torch.zeros(32)
            row[:10], row[10:20], row[20:30] = steps, torch.nextafter(steps, torch.tensor(9.0)), torch.nextafter(steps, torch.tensor(0.0))
            row[30], row[31] = 4.0, -4.0
            rows.append(sign * s * row.clamp(max=7.9999995))
    x = torch.stack(rows).cuda()
    t = q8.q8_mx4_quantize(x)
    check_codes(t, x)
    E = ref.unpack(t)[1][:, 0]
    assert E.tolist() == [127, 127, 107, 107, 217, 217]


def test_quantize_smallest_and_largest():
    top, tiny = torch.finfo(torch.float32).max, 2.0 ** -149
    x = torch.zeros(6, 64)
    x[0, :32] = torch.linspace(-top, top, 32)
    x[1, 3], x[1, 40] = tiny, -3 * tiny
    x[2, :32] = torch.linspace(0, 2.0 ** -126, 32)
    x[3, :32] = torch.linspace(0, 2.0 ** -123, 32)
    x[4, 0], x[4, 1] = 2.0 ** -125, 2.0 ** 100
    x = x.cuda()
    check_codes(q8.q8_mx4_quantize(x), x)
    assert np.array_equal(ref.as_numpy(q8.q8_mx4_fake_quantize(x)), ref.rounded(x))


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_quantize_what_is_not_a_number(dtype):
    x = values((40, 96), 3, dtype, 0.0)
    x[0, 5], x[1, 40], x[2, 70] = float("nan"), float("inf"), -float("inf")
    x[3, :32], x[4, 32:64], x[5] = float("nan"), float("inf"), 0
    word = status_word()
    t = q8.q8_mx4_quantize(x, dev_status=word)
    check_codes(t, x)
    assert word.item() == 1 << q8.Q8_ERR_SCALE
    code, E, _ = ref.unpack(t)
    assert code[0, 5] == 0 and code[1, 40] == 7 and code[2, 70] == 15
    assert not code[3, :32].any() and E[3, 0] == 0 and (code[4, 32:64] == 7).all() and E[4, 1] == 0 and not E[5].any()
    word.zero_()
    q8.q8_mx4_fake_quantize(x[6:], dev_status=word)
    assert word.item() == 0
    y = q8.q8_mx4_fake_quantize(x, dev_status=word)
    assert word.item() == 1 << q8.Q8_ERR_SCALE and torch.isfinite(y).all()


# ---------------------------------------------------------------- training
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("rows,K", [(1, 1), (5, 33), (64, 768), (33, 1001)])
def test_fake_quantize(rows, K, dtype):
    x = values((rows, K), K, dtype)
    before = x.clone()
    y = q8.q8_mx4_fake_quantize(x)
    want = torch.from_numpy(ref.rounded(x)).to(dtype)
    assert y.dtype == dtype and torch.equal(y.cpu(), want) and torch.equal(x, before)
    wide = torch.full((rows, K + 9), 3.0, dtype=dtype, device="cuda")
    q8.q8_mx4_fake_quantize(x, wide[:, 4:4 + K])
    assert torch.equal(wide[:, 4:4 + K].cpu(), want) and (wide[:, :4] == 3).all() and (wide[:, 4 + K:] == 3).all()
    assert q8.q8_mx4_fake_quantize(x, x) is x and torch.equal(x.cpu(), want)
    assert torch.equal(q8.q8_mx4_fake_quantize(x.clone()), x), "values on the grid stay"


class FakeQuantized(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x):
        return q8.q8_mx4_fake_quantize(x)

    @staticmethod
    def backward(ctx, g):
        return q8.q8_ste_backward(g.contiguous())


def test_training_step():
    """A fake-quantised layer's gradients are those of the layer on the rounded values (Eq. 5: the rounding has slope 1)."""
    x, w = values((48, 96), 1, spread=0.5).requires_grad_(), weights((80, 96), 2).requires_grad_()
    g = values((48, 80), 3, spread=0.0)
    (FakeQuantized.apply(x) @ FakeQuantized.apply(w).t()).backward(g)
    x_hat, w_hat, g64 = ref.rounded(x), ref.rounded(w), ref.as_numpy(g)
    for got, want, size in ((x.grad, g64 @ w_hat, np.abs(g64) @ np.abs(w_hat)), (w.grad, g64.T @ x_hat, np.abs(g64).T @ np.abs(x_hat))):
        assert (np.abs(ref.as_numpy(got) - want) <= 100 * 2.0 ** -24 * size).all()  # up to 96 fp32 additions


def test_slope_of_the_rounding():
    """Differences over whole steps: from one end of the grid to the other the rounded values rise as the values do."""
    t = torch.linspace(-6, 6, 961)[:, None].expand(-1, 32).contiguous()
    t[:, 31] = 6.0
    y = q8.q8_mx4_fake_quantize(t.cuda())[:, 0].cpu()
    assert (y[1:] >= y[:-1]).all() and y[0] == -6 and y[-1] == 6
    assert (y[-1] - y[0]) / (t[-1, 0] - t[0, 0]) == 1


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("K", [1, 7, 8, 9, 31, 100, 255, 256, 257, 263, 264, 511, 770, 1035])
def test_rows_at_any_address(K, dtype):
    """Every place of a row's beginning and end in the 16 bytes that are read and written at once: values, and nothing beside them."""
    for offset in range(0, 9):
        for ld in (K + 9, K + 10, 2 * K + 12, 16 * (K // 16 + 2)):
            x = values((9, ld), K + offset, dtype)
            x[:, :offset], x[:, offset + K:] = float("nan"), float("nan")  # what is not of the rows does not reach them
            rows = x[:, offset:offset + K]
            word = status_word()
            t = q8.q8_mx4_quantize(rows, dev_status=word)
            check_codes(t, rows)
            out = torch.full((11, ld + 3), 5.0, dtype=dtype, device="cuda")
            inner = out[1:10, offset + 1:offset + 1 + K]
            q8.q8_mx4_fake_quantize(rows, inner, dev_status=word)
            want = torch.from_numpy(ref.rounded(rows)).to(dtype)
            assert torch.equal(inner.cpu(), want) and word.item() == 0
            rest = out.clone()
            rest[1:10, offset + 1:offset + 1 + K] = 5.0
            assert (rest == 5.0).all()
            assert torch.equal(q8.q8_mx4_dequantize(t, dtype).cpu(), want)


# ---------------------------------------------------------------- the layer
def run_layer(M, N, K, dtype, act, with_bias, seed=0, ld=None, out=None):
    x = values((M, ld or K), seed, dtype, 0.5)[:, :K]
    w, b = weights((N, K), seed + 1), weights((N,), seed + 2) if with_bias else None
    W = q8.q8_mx4_quantize(w)
    word = status_word()
    pad, out = 7, out or dtype
    whole = torch.full((M + 2, N + pad), 77.0, dtype=out, device="cuda")
    Y = whole[1:-1, :N]
    got = q8.q8_mx4_linear(x, W, b, act, Y=Y, dev_status=word)
    assert got is Y and word.item() == 0
    ref.assert_layer(Y, ref.rounded(x), ref.rounded(w), b, act)
    assert (whole[:, N:] == 77).all() and (whole[0] == 77).all() and (whole[-1] == 77).all()
    plain = q8.q8_mx4_linear(x, W, b, act, dtype=out)
    assert torch.equal(plain, Y)
    assert torch.equal(q8.q8_mx4_linear_q(q8.q8_mx4_quantize(x), W, b, act, dtype=out), Y)


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 8, 32), (1, 1000, 33), (2, 129, 64), (3, 128, 96), (15, 200, 130), (16, 256, 256),
                                   (17, 127, 257), (33, 384, 512), (64, 128, 1000), (65, 300, 777), (127, 130, 2000), (128, 512, 160)])
def test_linear_few_tokens(M, N, K):
    run_layer(M, N, K, torch.float32, q8.Q8_ACT_NONE, True, seed=M)


@pytest.mark.parametrize("M,N,K", [(129, 128, 128), (191, 256, 300), (192, 640, 512), (193, 1000, 1024), (320, 4096, 256), (500, 777, 1000),
                                   (1000, 1024, 520), (2100, 2048, 264), (1500, 4100, 96)])
@pytest.mark.parametrize("act", [q8.Q8_ACT_NONE, q8.Q8_ACT_GELU], ids=["none", "gelu"])
def test_linear(M, N, K, act):
    run_layer(M, N, K, torch.float32, act, act == q8.Q8_ACT_GELU, seed=M)


@pytest.mark.parametrize("M", [1, 24, 200, 1300])
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("out", TYPES, ids=NAMES.get)
def test_linear_types(M, dtype, out):
    run_layer(M, 333, 700, dtype, q8.Q8_ACT_GELU, True, seed=5, out=out)
    run_layer(M, 256, 512, dtype, q8.Q8_ACT_NONE, False, seed=6, out=out)


@pytest.mark.parametrize("ld", [1000, 1008, 1001])
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_linear_rows_of_a_wider_tensor(ld, dtype):
    for M in (1, 3, 13, 100):
        run_layer(M, 256, 1000, dtype, q8.Q8_ACT_NONE, True, ld=ld)


def test_linear_long_rows():
    run_layer(5, 130, 30000, torch.float32, q8.Q8_ACT_NONE, False)
    run_layer(200, 300, 20001, torch.bfloat16, q8.Q8_ACT_NONE, True)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 7, 8, 15, 31, 33, 63, 64, 65, 100, 128])
@pytest.mark.parametrize("N,K", [(1, 2048), (130, 2049), (300, 4096), (1000, 8100), (40, 20000)])
def test_linear_few_tiles_with_a_long_sum(M, N, K):
    """The K axis of a tile shared by CTAs, which finish shares of its tokens: more tokens than CTAs, fewer, and none for some."""
    run_layer(M, N, K, (torch.float32, torch.bfloat16)[M % 2], M % 3 == 0, M % 2 == 1, seed=M)


def test_linear_scales_of_all_sizes():
    """Scales from the smallest to the largest exponent; products outside fp32's range are left to it."""
    x, w = values((70, 256), 1, spread=0.0), weights((160, 256), 2)
    x = x * torch.pow(2.0, torch.arange(70).cuda().float()[:, None] - 35)
    w = w * torch.pow(2.0, 40 - torch.arange(160).cuda().float()[:, None] / 2)
    Y = q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w))
    ref.assert_layer(Y, ref.rounded(x), ref.rounded(w), None, q8.Q8_ACT_NONE)


@pytest.mark.parametrize("M,K", [(3, 2048), (200, 4096), (300, 96)])
def test_linear_blocks_of_all_sizes_in_a_row(M, K):
    """Sums in which some blocks are far larger than others, so that fp32 cannot hold them exactly."""
    g = torch.Generator().manual_seed(K)
    x = torch.randn(M, K // 32, 32, generator=g) * torch.exp(4 * torch.randn(M, K // 32, 1, generator=g))
    w = torch.randn(260, K // 32, 32, generator=g) * torch.exp(4 * torch.randn(260, K // 32, 1, generator=g))
    x, w = x.flatten(1).cuda(), w.flatten(1).cuda()
    ref.assert_layer(q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w)), ref.rounded(x), ref.rounded(w), None, q8.Q8_ACT_NONE)


def test_linear_columns_of_one_matrix():
    """Input and output side by side in one buffer; an output on top of the input is refused."""
    for M in (3, 40, 300):
        both = torch.zeros(M, 512 + 384, device="cuda")
        both[:, :512] = values((M, 512), M, spread=0.5)
        x, w = both[:, :512].clone(), weights((384, 512), 2)
        q8.q8_mx4_linear(both[:, :512], q8.q8_mx4_quantize(w), Y=both[:, 512:])
        assert torch.equal(both[:, :512], x)
        ref.assert_layer(both[:, 512:], ref.rounded(x), ref.rounded(w), None, q8.Q8_ACT_NONE)
        with pytest.raises(q8.Q8Error) as e:
            q8.q8_mx4_linear(both[:, :512], q8.q8_mx4_quantize(w), Y=both[:, 500:884])
        assert e.value.status == q8.Q8_ERR_ARG


def test_linear_zero_rows_and_infinities():
    x, w = values((40, 192), 1, spread=0.0), weights((130, 192), 2)
    x[3], x[4, 64:96] = 0, 0
    x[7, 10], x[8, 100] = float("inf"), float("nan")
    w[5] = 0
    word = status_word()
    Y = q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w), dev_status=word)
    assert word.item() == 1 << q8.Q8_ERR_SCALE
    assert (Y[3] == 0).all() and (Y[:, 5] == 0).all()
    ref.assert_layer(Y, ref.rounded(x), ref.rounded(w), None, q8.Q8_ACT_NONE)


def test_linear_nothing_to_do():
    W = q8.q8_mx4_quantize(weights((16, 64), 1))
    assert q8.q8_mx4_linear(torch.empty(0, 64, device="cuda"), W).shape == (0, 16)
    none = q8.q8_mx4_quantize(torch.empty(0, 64, device="cuda"))
    assert q8.q8_mx4_linear(values((3, 64), 1), none).shape == (3, 0)
    assert q8.q8_mx4_dequantize(none).shape == (0, 64)


# ---------------------------------------------------------------- grouped by expert
def run_grouped(offsets, T, N, K, dtype=torch.float32, act=q8.Q8_ACT_NONE, with_bias=True, tokens=None, seed=0):
    E = len(offsets) - 1
    g = torch.Generator().manual_seed(seed)
    x = values((tokens or T, K), seed, dtype, 0.5)
    w, b = weights((E, N, K), seed + 1), weights((E, N), seed + 2) if with_bias else None
    rows = torch.randint(0, tokens, (T,), generator=g, dtype=torch.int32).cuda() if tokens else None
    W = q8.q8_mx4_quantize(w)
    word = status_word()
    whole = torch.full((T + 2, N), 55.0, dtype=dtype, device="cuda")
    Y = whole[1:-1]
    q8.q8_mx4_linear_grouped(x, torch.tensor(offsets, dtype=torch.int32).cuda(), W, b, act, rows, Y, dev_status=word)
    assert word.item() == 0 and (whole[0] == 55).all() and (whole[-1] == 55).all()
    taken = x if rows is None else x[rows.long()]
    assert (Y[:offsets[0]] == 55).all() and (Y[offsets[-1]:] == 55).all()
    for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        if hi > lo:
            ref.assert_layer(Y[lo:hi], ref.rounded(taken[lo:hi]), ref.rounded(w[e]), None if b is None else b[e], act)


@pytest.mark.parametrize("offsets,T", [
    ([0, 1], 1), ([0, 0, 1, 1], 1), ([0, 5, 5, 12], 12), ([0, 16, 32, 48, 64], 64), ([3, 10, 40], 50), ([0, 0, 0, 0], 9),
    ([0, 130, 131, 400], 400), ([0, 127, 255, 384, 513], 600), ([0, 500, 500, 517, 1000], 1000)])
@pytest.mark.parametrize("N,K", [(128, 128), (300, 520), (65, 33)])
def test_grouped(offsets, T, N, K):
    run_grouped(offsets, T, N, K)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("counts", [[8, 8, 14, 34], [0, 70, 0, 0, 1, 0], [33, 0, 0, 5], [2, 0, 96, 1, 0, 0, 0, 3], [31, 32, 33, 0, 0, 0, 0, 0, 0]])
def test_grouped_few_slots_unevenly(counts, dtype):
    """Experts with more slots than the others have on average."""
    offsets = [0, *np.cumsum(counts).tolist()]
    run_grouped(offsets, offsets[-1], 200, 600, dtype, q8.Q8_ACT_GELU)
    run_grouped([v + 3 for v in offsets], offsets[-1] + 10, 128, 256, dtype, tokens=9)


@pytest.mark.parametrize("counts", [[700, 0, 1300], [256, 257, 255, 1, 0, 900], [1023, 1025]])
def test_grouped_many_slots(counts):
    """Enough for pairs of CTAs: full and cut tiles of experts, features that end in the first half of a pair's tile."""
    offsets = [0, *np.cumsum(counts).tolist()]
    for dtype, N in ((torch.float32, 2400), (torch.bfloat16, 2500), (torch.float16, 2305)):
        run_grouped(offsets, offsets[-1] + 5, N, 520, dtype, q8.Q8_ACT_GELU, tokens=offsets[-1] // 2)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("E,T", [(7, 20), (64, 40), (64, 3000), (5, 4000), (1, 100)])
def test_grouped_routed(E, T, dtype):
    cuts = np.sort(np.random.RandomState(E).randint(0, T + 1, E - 1)).tolist()
    run_grouped([0, *cuts, T], T, 200, 264, dtype, q8.Q8_ACT_GELU, tokens=T // 2 + 1, seed=T)


def test_grouped_many_experts():
    for E in (31, 32, 33, 1000, 1024):
        cuts = np.sort(np.random.RandomState(E).randint(0, 701, E - 1)).tolist()
        run_grouped([0, *cuts, 700], 700, 40, 64, with_bias=E != 33)


def test_grouped_is_the_plain_layer_for_one_expert():
    x, w = values((300, 512), 1, torch.bfloat16), weights((1, 384, 512), 2)
    W = q8.q8_mx4_quantize(w)
    one = q8.Mx4(W.tiles, W.shape[1:])
    offsets = torch.tensor([0, 300], dtype=torch.int32).cuda()
    assert torch.equal(q8.q8_mx4_linear_grouped(x, offsets, W), q8.q8_mx4_linear(x, one))


@pytest.mark.parametrize("offsets", [[0, 30, 20, 50], [0, -5, 30, 50], [0, 20, 70, 50], [60, 10, 20, 30], [0, 2 ** 31 - 1, -2 ** 31, 7]])
def test_grouped_bad_offsets(offsets):
    """Moved to the nearest offsets that rise from 0 to T, and flagged."""
    T, N, K = 50, 140, 96
    x, w = values((T, K), 1), weights((3, N, K), 2)
    word = status_word()
    whole = torch.full((T + 2, N), 55.0, device="cuda")
    Y = whole[1:-1]
    q8.q8_mx4_linear_grouped(x, torch.tensor(offsets, dtype=torch.int64).to(torch.int32).cuda(), q8.q8_mx4_quantize(w), Y=Y, dev_status=word)
    assert word.item() == 1 << q8.Q8_ERR_INDEX and (whole[0] == 55).all() and (whole[-1] == 55).all()
    ends = np.maximum.accumulate(np.clip(offsets, 0, T))
    for e in range(3):
        lo, hi = ends[e], ends[e + 1]
        if hi > lo:
            ref.assert_layer(Y[lo:hi], ref.rounded(x[lo:hi]), ref.rounded(w[e]), None, q8.Q8_ACT_NONE)
    assert (Y[:ends[0]] == 55).all() and (Y[ends[-1]:] == 55).all()


def test_grouped_bad_rows():
    x, w = values((10, 96), 1), weights((2, 60, 96), 2)
    rows = torch.tensor([0, 9, 10, -1, 3, 3, 2 ** 31 - 1, 5], dtype=torch.int32).cuda()
    offsets = torch.tensor([0, 5, 7], dtype=torch.int32).cuda()
    word = status_word()
    Y = torch.full((8, 60), 55.0, device="cuda")
    q8.q8_mx4_linear_grouped(x, offsets, q8.q8_mx4_quantize(w), rows=rows, Y=Y, dev_status=word)
    assert word.item() == 1 << q8.Q8_ERR_INDEX
    assert (Y[[2, 3, 6]] == 0).all() and (Y[7] == 55).all()
    taken = x[rows.long().clamp(0, 9)].clone()
    taken[[2, 3, 6]] = 0
    ref.assert_layer(Y[:5], ref.rounded(taken[:5]), ref.rounded(w[0]), None, 0)
    ref.assert_layer(Y[5:7], ref.rounded(taken[5:7]), ref.rounded(w[1]), None, 0)
    word.zero_()
    rows[:7] = 0
    rows[7] = 99  # of a slot that no expert owns
    q8.q8_mx4_linear_grouped(x, offsets, q8.q8_mx4_quantize(w), rows=rows, Y=Y, dev_status=word)
    assert word.item() == 0


# ---------------------------------------------------------------- as they are used
def test_feed_forward_of_experts():
    """Top-2 routing, two grouped layers with GELU between them, and the tokens put together again."""
    tokens, E, H, F = 150, 6, 256, 520
    g = torch.Generator().manual_seed(0)
    x = values((tokens, H), 1, torch.bfloat16, 0.0)
    choice = torch.rand(tokens, E, generator=g).topk(2, dim=1)
    expert = choice.indices.flatten()
    order = expert.argsort(stable=True)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), expert.bincount(minlength=E).cumsum(0)]).to(torch.int32).cuda()
    rows = (order // 2).to(torch.int32).cuda()
    w1, w2 = weights((E, F, H), 2), weights((E, H, F), 3)
    h = q8.q8_mx4_linear_grouped(x, offsets, q8.q8_mx4_quantize(w1), None, q8.Q8_ACT_GELU, rows)
    y = q8.q8_mx4_linear_grouped(h, offsets, q8.q8_mx4_quantize(w2))
    out = torch.zeros(tokens, H, device="cuda").index_add_(0, rows.long(), y.float() * choice.values.flatten()[order].cuda()[:, None])
    want, size = np.zeros((tokens, H)), np.zeros((tokens, H))
    ends = offsets.tolist()
    for e in range(E):
        lo, hi = ends[e], ends[e + 1]
        if lo == hi:
            continue
        taken = rows[lo:hi].long().cpu()
        ref.assert_layer(h[lo:hi], ref.rounded(x[taken]), ref.rounded(w1[e]), None, q8.Q8_ACT_GELU)
        ref.assert_layer(y[lo:hi], ref.rounded(h[lo:hi]), ref.rounded(w2[e]), None, q8.Q8_ACT_NONE)
        part = ref.as_numpy(y[lo:hi]) * choice.values.flatten()[order][lo:hi, None].double().numpy()
        np.add.at(want, taken.numpy(), part)
        np.add.at(size, taken.numpy(), np.abs(part))
    assert (np.abs(ref.as_numpy(out) - want) <= 4 * 2.0 ** -24 * size).all()  # a product and up to two additions in fp32


def test_captured_and_replayed():
    """Two layers and a grouped one in a graph, replayed on new inputs, one workspace for all of them."""
    M, H, F, E = 70, 256, 384, 3
    x = values((M, H), 1, torch.bfloat16, 0.0)
    W1, W2, W3 = q8.q8_mx4_quantize(weights((F, H), 2)), q8.q8_mx4_quantize(weights((H, F), 3)), q8.q8_mx4_quantize(weights((E, F, H), 4))
    offsets = torch.tensor([0, 20, 20, 65], dtype=torch.int32).cuda()
    ws = torch.empty(max(q8.q8_mx4_linear_workspace_bytes(M, F), q8.q8_mx4_linear_grouped_workspace_bytes(M, E, H)), dtype=torch.uint8, device="cuda")
    Y = torch.full((M, F), 9.0, dtype=torch.bfloat16, device="cuda")

    def step():
        h = q8.q8_mx4_linear(x, W1, None, q8.Q8_ACT_GELU, workspace=ws)
        y = q8.q8_mx4_linear(h, W2, workspace=ws)
        q8.q8_mx4_linear_grouped(y, offsets, W3, Y=Y, workspace=ws)
        return y

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    for seed in (5, 6):
        x.copy_(values((M, H), seed, torch.bfloat16, 0.0))
        offsets.copy_(torch.tensor([0, 20, 20, 65] if seed == 5 else [0, 0, 50, 60], dtype=torch.int32))
        Y.fill_(9.0)
        graph.replay()
        replayed = (y.clone(), Y.clone())
        Y.fill_(9.0)
        assert torch.equal(step(), replayed[0]) and torch.equal(Y, replayed[1])


def test_other_streams_and_repeated_calls():
    x, w = values((200, 512), 1), weights((640, 512), 2)
    W = q8.q8_mx4_quantize(w)
    want = q8.q8_mx4_linear(x, W)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    results = [q8.q8_mx4_linear(x, W, stream=side) for _ in range(20)] + [q8.q8_mx4_linear(x, W) for _ in range(20)]
    with torch.cuda.stream(side):
        results.append(q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w)))
        results.append(q8.q8_mx4_linear_q(q8.q8_mx4_quantize(x), q8.q8_mx4_quantize(w)))
    torch.cuda.synchronize()
    assert all(torch.equal(r, want) for r in results)


def test_weights_made_right_before_the_layer():
    """The layer starts while the kernel before it still runs; weights and offsets that earlier kernels write are there in time."""
    x = values((64, 1024), 1)
    ws = [weights((2048, 1024), s) for s in range(6)]
    want = []
    for w in ws:
        W = q8.q8_mx4_quantize(w)
        torch.cuda.synchronize()
        want.append(q8.q8_mx4_linear(x, W))
        torch.cuda.synchronize()
    W = q8.q8_mx4_quantize(ws[0])
    got = []
    for w in ws:
        fresh = q8.q8_mx4_quantize(w)
        W.tiles.copy_(fresh.tiles)
        got.append(q8.q8_mx4_linear(x, W))
        fresh = q8.q8_mx4_quantize(w)
        got.append(q8.q8_mx4_linear(x, fresh))
    assert all(torch.equal(a, b) for a, b in zip(got, [v for v in want for _ in range(2)]))



@pytest.mark.parametrize("M,K,N,act,dtype", [(4096, 2048, 2048, q8.Q8_ACT_NONE, torch.bfloat16), (2304, 512, 1000, q8.Q8_ACT_GELU, torch.float32),
                                             (300, 1024, 768, q8.Q8_ACT_NONE, torch.float16), (24, 4096, 512, q8.Q8_ACT_NONE, torch.bfloat16)])
def test_calls_one_after_the_other(M, K, N, act, dtype):
    """Hundreds of calls that nothing waits between, two inputs in turn: no wait runs out, and each gives what it gave alone."""
    word = status_word()
    xs = [values((M, K), s, dtype) for s in (1, 2)]
    W = q8.q8_mx4_quantize(weights((N, K), 3))
    want = []
    for x in xs:
        want.append(q8.q8_mx4_linear(x, W, act=act, dev_status=word))
        torch.cuda.synchronize()
    for _ in range(4):
        for i in range(200):
            y = q8.q8_mx4_linear(xs[i % 2], W, act=act, dev_status=word)
            if i in (0, 63, 198, 199):
                assert torch.equal(y, want[i % 2])
        torch.cuda.synchronize()
    assert word.item() == 0


def test_offsets_and_experts_made_right_before_the_layer():
    """The product reads offsets and weights before its own quantise pass ends, but after the kernels that wrote them."""
    x = values((700, 512), 1)
    layers = []
    for seed, counts in enumerate([(300, 0, 400), (0, 700, 0), (1, 2, 697), (233, 234, 233)]):
        w = torch.stack([weights((384, 512), 10 * seed + e) for e in range(3)])
        layers.append((w, torch.tensor(counts, dtype=torch.int32, device="cuda")))

    def offsets_of(counts):
        return torch.cat([counts.new_zeros(1), counts.cumsum(0, dtype=torch.int32)])

    want = []
    for w, counts in layers:
        W, offsets = q8.q8_mx4_quantize(w), offsets_of(counts)
        torch.cuda.synchronize()
        want.append(q8.q8_mx4_linear_grouped(x, offsets, W))
        torch.cuda.synchronize()
    offsets, W = offsets_of(layers[0][1]), q8.q8_mx4_quantize(layers[0][0])
    got = []
    for _ in range(10):
        for w, counts in layers:
            fresh = q8.q8_mx4_quantize(w)
            W.tiles.copy_(fresh.tiles)
            offsets.copy_(offsets_of(counts))
            got.append(q8.q8_mx4_linear_grouped(x, offsets, W))
            offsets.copy_(offsets_of(counts))
            got.append(q8.q8_mx4_linear_grouped(x, offsets, q8.q8_mx4_quantize(w)))
    assert all(torch.equal(a, want[i // 2 % 4]) for i, a in enumerate(got))



@pytest.mark.parametrize("M", [1, 3, 40, 200])
def test_everything_made_right_before_the_layer(M):
    """Activation, bias and weights come from kernels of the library right before, call after call in the same memory."""
    K, N, sets = 256, 384, 5
    xs, bs, ws = ([q8.q8_mx4_quantize(f(shape, 3 * i + j)) for i in range(sets)] for j, (f, shape) in enumerate(((values, (M, K)), (weights, (1, N)), (weights, (N, K)))))
    want = []
    for x, b, w in zip(xs, bs, ws):
        x, b, w = (q8.q8_mx4_dequantize(t) for t in (x, b, w))
        torch.cuda.synchronize()
        w = q8.q8_mx4_quantize(w)
        torch.cuda.synchronize()
        want.append(q8.q8_mx4_linear(x, w, b[0]))
        torch.cuda.synchronize()
    got = []
    for i in range(300):
        x, b, w = (q8.q8_mx4_dequantize(t[i % sets]) for t in (xs, bs, ws))
        got.append(q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w), b[0]))
        x = b = w = None  # the next call's are in the same places
    assert all(torch.equal(y, want[i % sets]) for i, y in enumerate(got))


def test_tiles_rewritten_between_readings():
    tiles = torch.empty(q8.q8_mx4_bytes(1, 200, 512), dtype=torch.uint8, device="cuda")
    xs = [values((200, 512), s) for s in range(4)]
    lib, stream = q8.load(), torch.cuda.current_stream().cuda_stream
    want = [q8.q8_mx4_dequantize(q8.q8_mx4_quantize(x)) for x in xs]
    torch.cuda.synchronize()
    got = torch.empty(200, 200, 512, device="cuda")
    for i in range(200):
        assert lib.q8_mx4_quantize(xs[i % 4].data_ptr(), q8.Q8_F32, 1, 200, 512, 512, tiles.data_ptr(), None, stream) == q8.Q8_OK
        assert lib.q8_mx4_dequantize(tiles.data_ptr(), 1, 200, 512, got[i].data_ptr(), q8.Q8_F32, 512, stream) == q8.Q8_OK
    assert all(torch.equal(got[i], want[i % 4]) for i in range(200))


def test_refusals_on_the_device():
    x, w = values((4, 64), 1), weights((8, 64), 2)
    W = q8.q8_mx4_quantize(w)
    with pytest.raises(ValueError, match="rows of 64"):
        q8.q8_mx4_linear(values((4, 65), 1), W)
    with pytest.raises(ValueError, match="bias has 7"):
        q8.q8_mx4_linear(x, W, weights((7,), 1))
    with pytest.raises(ValueError, match="Y must be"):
        q8.q8_mx4_linear(x, W, Y=torch.empty(4, 9, device="cuda"))
    with pytest.raises(TypeError, match="asked for"):
        q8.q8_mx4_linear(x, W, Y=torch.empty(4, 8, device="cuda"), dtype=torch.float16)
    with pytest.raises(TypeError, match="float32, float16 or bfloat16"):
        q8.q8_mx4_linear(x.double(), W)
    with pytest.raises(TypeError, match="side by side"):
        q8.q8_mx4_linear(values((64, 4), 1).t(), W)
    with pytest.raises(TypeError, match="overlap"):
        q8.q8_mx4_linear(values((1, 64), 1).expand(4, 64), W)
    with pytest.raises(ValueError, match="bytes of tiles"):
        q8.q8_mx4_linear(x, q8.Mx4(W.tiles[:17407], W.shape))
    with pytest.raises(ValueError, match="bytes of tiles"):
        q8.q8_mx4_linear(values((4, 257), 1), q8.Mx4(W.tiles, (8, 257)))
    with pytest.raises(q8.Q8Error) as e:
        q8.q8_mx4_linear(values((130, 64), 1), W, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == q8.Q8_ERR_WORKSPACE
    with pytest.raises(q8.Q8Error) as e:
        q8.q8_mx4_linear(x, W, act=3)
    assert e.value.status == q8.Q8_ERR_ARG
    G = q8.q8_mx4_quantize(weights((2, 8, 64), 2))
    with pytest.raises(ValueError, match="dimensions"):
        q8.q8_mx4_linear(x, G)
    with pytest.raises(ValueError, match="for 2 experts"):
        q8.q8_mx4_linear_grouped(x, torch.zeros(2, dtype=torch.int32, device="cuda"), G)
    with pytest.raises(TypeError, match="offsets must be torch.int32"):
        q8.q8_mx4_linear_grouped(x, torch.zeros(3, dtype=torch.int64, device="cuda"), G)
    torch.cuda.synchronize()


# ---------------------------------------------------------------- what is not finite, behind the product
@pytest.mark.parametrize("out", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("M,N,K,tokens,ctas", [(2, 300, 64, 32, {1}), (2, 200, 8192, 32, {2, 4, 8}), (5, 200, 8192, 64, {2, 4, 8}), (40, 300, 200, 64, {1}),
                                               (4096, 2400, 96, 128, {1}), (4096, 2400, 2100, 256, {2})])
def test_gelu_of_what_is_not_finite(M, N, K, tokens, ctas, out):
    """A NaN in the bias, or of sums of opposite infinities, stays NaN; +inf stays; of -inf the limit, 0.  In each way a sum takes to Y."""
    x, w, b = values((M, K), 1, spread=0.0), weights((N, K), 2), weights((N,), 3)
    b[0], b[1], b[2], b[N - 1] = float("nan"), float("inf"), -float("inf"), float("nan")
    # row 1: features 5 and 6 overflow to either side, feature 7 has both signs in its sum, and in feature 2 the sum's infinity meets the bias's
    x[1] = 2.0 ** 101
    w[2], w[5], w[6], w[7] = 2.0 ** 101, 2.0 ** 101, -2.0 ** 101, 2.0 ** 101
    w[7, : K // 2] *= -1
    W = q8.q8_mx4_quantize(w)
    plain, got = (q8.q8_mx4_linear(x, W, b, act, dtype=out) for act in (q8.Q8_ACT_NONE, q8.Q8_ACT_GELU))
    info = q8.q8_last_launch_info()
    assert info["block_n"] == tokens and info["ctas"] in ctas
    others = [0, *range(2, M)]
    assert torch.isnan(plain[:, [0, N - 1]]).all() and torch.isposinf(plain[others, 1]).all() and torch.isneginf(plain[others, 2]).all()
    assert torch.isposinf(plain[1, 5]) and torch.isneginf(plain[1, 6]) and torch.isnan(plain[1, 2])
    assert torch.equal(torch.isnan(got), torch.isnan(plain)), "NaN where the sums are, and nowhere else"
    assert torch.equal(torch.isposinf(got), torch.isposinf(plain))
    low = torch.isneginf(plain)
    assert low[1, 6] and (got[low].abs() <= 1e-7).all()


def test_gelu_of_what_is_not_finite_grouped():
    x, w, b = values((300, 128), 1, spread=0.0), weights((3, 200, 128), 2), weights((3, 200), 3)
    b[0, 7], b[2, 199], b[2, 3] = float("nan"), float("nan"), -float("inf")
    offsets = torch.tensor([0, 100, 140, 300], dtype=torch.int32).cuda()
    y = q8.q8_mx4_linear_grouped(x, offsets, q8.q8_mx4_quantize(w), b, q8.Q8_ACT_GELU)
    want = torch.zeros(300, 200, dtype=torch.bool, device="cuda")
    want[:100, 7], want[140:, 199] = True, True
    assert torch.equal(torch.isnan(y), want) and (y[140:, 3].abs() <= 1e-7).all()


def test_bias_between_the_rows_of_the_output():
    """What lies between two rows of Y is not Y's: a bias there is read and stays."""
    for M in (2, 40):
        x, w, b = values((M, 256), M, spread=0.5), weights((100, 256), 2), weights((100,), 3)
        both = torch.zeros(M, 512, device="cuda")
        both[1, 200:300] = b
        q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w), both[1, 200:300], Y=both[:, :100])
        ref.assert_layer(both[:, :100], ref.rounded(x), ref.rounded(w), b, q8.Q8_ACT_NONE)
        assert torch.equal(both[1, 200:300], b) and (both[0, 100:] == 0).all()
        with pytest.raises(q8.Q8Error) as e:
            q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w), both[1, 50:150], Y=both[:, :100])
        assert e.value.status == q8.Q8_ERR_ARG


# ---------------------------------------------------------------- many rows at any address
MANY_ROWS = 33 * 128  # whole tiles, so that every byte of them is defined; with K >= 256 over 2^20 values, from which on the kernels move bytes to their places


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("K", [256, 257, 263, 264, 511, 1035])
def test_many_rows_at_any_address(K, dtype):
    """test_rows_at_any_address for the kernels that large tensors take: every place of a row in its 16 bytes, rows that all begin at another one, values, and
    nothing beside them read as theirs or written."""
    assert K >= 256 and MANY_ROWS * K >= 1 << 20
    x0 = values((MANY_ROWS, K), K, dtype)
    aligned = torch.zeros(MANY_ROWS, (K + 31) // 32 * 32, dtype=dtype, device="cuda")
    aligned[:, :K] = x0
    t0 = q8.q8_mx4_quantize(aligned[:, :K])  # rows at multiples of 32 bytes: checked against the definition, the others against it
    check_codes(t0, x0)
    want = torch.from_numpy(ref.rounded(x0)).to(dtype).cuda()
    assert torch.equal(q8.q8_mx4_fake_quantize(aligned[:, :K]), want)
    lib, stream = q8.load(), torch.cuda.current_stream().cuda_stream
    for offset in range(0, 9):
        for ld in (K + 9, K + 10, K + 16 - K % 8):
            whole = torch.full((MANY_ROWS + 2, ld), float("nan"), dtype=dtype, device="cuda")
            rows = whole[1:-1, offset:offset + K]
            rows.copy_(x0)
            word = status_word()
            t = q8.q8_mx4_quantize(rows, dev_status=word)
            assert word.item() == 0, "a NaN beside the rows was taken for one of theirs"
            assert torch.equal(t.tiles, t0.tiles)
            out = torch.full((MANY_ROWS + 2, ld + 3), 5.0, dtype=dtype, device="cuda")
            place = (slice(1, -1), slice((offset + 1) % 9, (offset + 1) % 9 + K))
            guard = out.clone()
            guard[place] = want
            q8.q8_mx4_fake_quantize(rows, out[place], dev_status=word)
            assert torch.equal(out, guard) and word.item() == 0
            out.fill_(5.0)
            st = lib.q8_mx4_dequantize(t.tiles.data_ptr(), 1, MANY_ROWS, K, out[place].data_ptr(), q8._MX4_DTYPES[dtype], ld + 3, stream)
            assert st == q8.Q8_OK and torch.equal(out, guard)
            q8.q8_mx4_fake_quantize(rows, rows, dev_status=word)  # in place
            assert word.item() == 0 and torch.equal(rows, want)
            assert torch.isnan(whole[[0, -1]]).all() and torch.isnan(whole[1:-1, :offset]).all() and torch.isnan(whole[1:-1, offset + K:]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_many_rows_of_odd_length_side_by_side(dtype):
    """Contiguous tensors whose rows end anywhere, matrices of experts among them, with what is not a number at both ends of rows."""
    for shape in ((3, 1413, 301), (5000, 257)):
        x = values(shape, 3, dtype)
        t = q8.q8_mx4_quantize(x)
        back = q8.q8_mx4_dequantize(t, dtype)
        for g in range(shape[0] if len(shape) == 3 else 1):
            one, again = (x[g], back[g]) if len(shape) == 3 else (x, back)
            check_codes(t, one, g)
            assert torch.equal(again, torch.from_numpy(ref.rounded(one)).to(dtype).cuda())
    for column in (0, 7, 8, 255, 256):
        y = x.clone()
        y[::7, column] = float("nan")
        word = status_word()
        got = q8.q8_mx4_fake_quantize(y, dev_status=word)
        assert word.item() == 1 << q8.Q8_ERR_SCALE and torch.equal(got, torch.from_numpy(ref.rounded(y)).to(dtype).cuda())


# ---------------------------------------------------------------- sums without rounding
def on_the_grid(shape, seed):
    """Values that are their own codes at scale 1: every block has one of 4 or 6."""
    g = torch.Generator().manual_seed(seed)
    x = torch.tensor(ref.GRID, dtype=torch.float32)[torch.randint(0, 8, shape, generator=g)] * (torch.randint(0, 2, shape, generator=g) * 2 - 1)
    x[..., ::32] = torch.tensor([4.0, 6.0])[torch.randint(0, 2, x[..., ::32].shape, generator=g)]
    return x.cuda()


@pytest.mark.parametrize("M,N,K", [(2, 130, 20001), (20, 130, 20001), (40, 300, 33), (500, 300, 4100), (1000, 1030, 20001), (4096, 2400, 2100)])
def test_sums_that_fp32_holds_are_exact(M, N, K):
    """Products are multiples of 1/4 and their absolute sum is below 36 K <= 720036 < 2^20, so 22 bits hold every partial sum, in whatever order: a wrong code,
    scale or place of a single value shows, which the tolerance of a long sum hides."""
    x, w, b = on_the_grid((M, K), 1), on_the_grid((N, K), 2), on_the_grid((N,), 3)
    W = q8.q8_mx4_quantize(w / 1024)
    want = (x.double() @ w.double().t() / 1024).float()
    for dtype in TYPES:
        assert torch.equal(q8.q8_mx4_linear(x.to(dtype), W, dtype=torch.float32), want)
    assert torch.equal(q8.q8_mx4_linear(x * 2.0 ** 20, W, b * 1024.0), want * 2.0 ** 20 + b * 1024)
    cuts = [0, M // 3, M // 3, M - 1, M]
    W4 = q8.q8_mx4_quantize(torch.stack([w / 1024, w, w / 2, -w / 1024]))
    y = q8.q8_mx4_linear_grouped(x, torch.tensor(cuts, dtype=torch.int32).cuda(), W4)
    for (lo, hi), factor in zip(zip(cuts, cuts[1:]), (1, 1024, 512, -1)):
        assert torch.equal(y[lo:hi], want[lo:hi] * factor)


# ---------------------------------------------------------------- conditions without a word of the caller's
def test_status_of_calls_without_a_word():
    """What the device finds is to be had of calls that were given no word, and of no others."""
    x, w = values((40, 192), 1, spread=0.0), weights((130, 192), 2)
    bad = x.clone()
    bad[3, 5] = float("nan")
    W, many = q8.q8_mx4_quantize(w), q8.q8_mx4_quantize(weights((2, 130, 192), 3))
    offsets, falling = (torch.tensor(v, dtype=torch.int32).cuda() for v in ([0, 20, 40], [0, 30, 20]))
    outside = torch.full((40,), 40, dtype=torch.int32, device="cuda")
    scale, index = (q8.Q8_ERR_SCALE, 1 << q8.Q8_ERR_SCALE), (q8.Q8_ERR_INDEX, 1 << q8.Q8_ERR_INDEX)
    q8.q8_mx4_status()
    for call, found in (
            (lambda v, s: q8.q8_mx4_quantize(v, dev_status=s), scale), (lambda v, s: q8.q8_mx4_fake_quantize(v, dev_status=s), scale),
            (lambda v, s: q8.q8_mx4_linear(v, W, dev_status=s), scale), (lambda v, s: q8.q8_mx4_linear(v[2:5], W, dev_status=s), scale),
            (lambda v, s: q8.q8_mx4_linear_grouped(v, offsets, many, dev_status=s), scale),
            (lambda v, s: q8.q8_mx4_linear_grouped(x, offsets if v is x else falling, many, dev_status=s), index),
            (lambda v, s: q8.q8_mx4_linear_grouped(x, offsets, many, rows=None if v is x else outside, dev_status=s), index)):
        call(x, None)
        assert q8.q8_mx4_status() == (q8.Q8_OK, 0)
        call(bad, None)
        assert q8.q8_mx4_status() == found and q8.q8_mx4_status() == (q8.Q8_OK, 0)
        word = status_word()
        call(bad, word)
        assert word.item() == found[1] and q8.q8_mx4_status() == (q8.Q8_OK, 0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(bad, None)
            assert q8.q8_mx4_status() == found


# ---------------------------------------------------------------- the gradient in every type
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2049, 100_003])
def test_straight_through_gradient(n, dtype):
    """Bit for bit the incoming one, NaN and infinities too, at any address, nothing beside it written, in place, in a graph."""
    g = values((n,), n, dtype)
    g[n // 2] = float("nan")
    bits = {4: torch.int32, 2: torch.int16}[g.element_size()]
    got = q8.q8_mx4_ste_backward(g)
    assert q8.q8_last_launch_info()["launches"] == 1 and got.dtype == dtype and got.data_ptr() != g.data_ptr()
    assert torch.equal(got.view(bits), g.view(bits)) and torch.equal(q8.q8_mx4_ste_backward(g, stream=torch.cuda.current_stream()).view(bits), g.view(bits))
    assert q8.q8_mx4_ste_backward(g, g) is g
    for off_in, off_out in ((0, 0), (1, 0), (0, 1), (2, 2), (3, 5)):
        src, room = torch.zeros(n + 8, dtype=dtype, device="cuda"), torch.full((n + 16,), 9.0, dtype=dtype, device="cuda")
        src[off_in:off_in + n] = g
        q8.q8_mx4_ste_backward(src[off_in:off_in + n], room[off_out:off_out + n])
        assert torch.equal(room[off_out:off_out + n].view(bits), g.view(bits))
        assert (room[:off_out] == 9).all() and (room[off_out + n:] == 9).all()
    moved, graph = torch.zeros_like(g), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q8.q8_mx4_ste_backward(g, moved)
    g.copy_(values((n,), n + 1, dtype))
    graph.replay()
    assert torch.equal(moved, g)
    assert q8.q8_mx4_ste_backward(torch.empty(0, 5, dtype=dtype, device="cuda")).shape == (0, 5)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_training_step_in_every_type(dtype):
    """test_training_step with leaves, rounded values and gradients in their own type, the product between them in fp32."""
    class Rounded(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return q8.q8_mx4_fake_quantize(x)

        @staticmethod
        def backward(ctx, g):
            return q8.q8_mx4_ste_backward(g.contiguous())

    x, w = values((48, 96), 1, dtype, 0.5).requires_grad_(), weights((80, 96), 2).to(dtype).requires_grad_()
    g = values((48, 80), 3, spread=0.0)
    (Rounded.apply(x).float() @ Rounded.apply(w).float().t()).backward(g)
    x_hat, w_hat, g64 = ref.rounded(x), ref.rounded(w), ref.as_numpy(g)
    for leaf, want, size in ((x, g64 @ w_hat, np.abs(g64) @ np.abs(w_hat)), (w, g64.T @ x_hat, np.abs(g64).T @ np.abs(x_hat))):
        far = 100 * 2.0 ** -24 * size  # up to 96 fp32 additions
        far = far + ref.HALF_STEP[dtype] * (np.abs(want) + far) + ref.SMALLEST[dtype]  # and the rounding to the leaf's type
        assert leaf.grad.dtype == dtype and (np.abs(ref.as_numpy(leaf.grad) - want) <= far).all()


def test_straight_through_gradient_refusals():
    g = values((40,), 1, torch.bfloat16)
    with pytest.raises(TypeError, match="float32, float16 or bfloat16"):
        q8.q8_mx4_ste_backward(g.double())
    with pytest.raises(TypeError):
        q8.q8_mx4_ste_backward(g, torch.empty(40, dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError, match="grad_in must be"):
        q8.q8_mx4_ste_backward(g, torch.empty(39, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError, match="contiguous"):
        q8.q8_mx4_ste_backward(g[::2])
    with pytest.raises(q8.Q8Error) as e:
        q8.q8_mx4_ste_backward(g[:30], g[5:35])
    assert e.value.status == q8.Q8_ERR_ARG


# ---------------------------------------------------------------- far offsets, streams at once, a first call that is captured
def test_tensors_of_more_than_two_to_the_31_values():
    rows, K = 525_000, 4100  # 2.15e9 values, rows that end inside a block and are not aligned
    x = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda")
    part = values((1000, K), 1, torch.bfloat16)
    for i in range(0, rows, 1000):
        torch.mul(part, 1 + i // 1000 % 3, out=x[i:i + 1000])
    assert x.numel() > 2 ** 31
    want = [torch.from_numpy(ref.rounded(part * f)).to(torch.bfloat16).cuda() for f in (1, 2, 3)]
    t = q8.q8_mx4_quantize(x)
    for back in (lambda: q8.q8_mx4_dequantize(t, torch.bfloat16), lambda: q8.q8_mx4_fake_quantize(x, x)):
        y = back()
        assert all(torch.equal(y[i:i + 1000], want[i // 1000 % 3]) for i in range(0, rows, 1000))
        del y


@pytest.mark.parametrize("grouped", [False, True], ids=["plain", "grouped"])
def test_outputs_of_more_than_two_to_the_31_values(grouped):
    M, N, K = 70_000, 32_000, 64
    x, w = values((M, K), 1, torch.bfloat16, 0.0), weights((2 if grouped else 1, N, K), 2)
    cut = 69_900
    if grouped:
        Y = q8.q8_mx4_linear_grouped(x, torch.tensor([0, cut, M], dtype=torch.int32).cuda(), q8.q8_mx4_quantize(w))
    else:
        Y = q8.q8_mx4_linear(x, q8.q8_mx4_quantize(w[0]))
    assert Y.numel() > 2 ** 31
    for lo in (0, 33_000, 67_100, cut - 60, cut, M - 60):  # on both sides of value 2^31
        ref.assert_layer(Y[lo:lo + 60], ref.rounded(x[lo:lo + 60]), ref.rounded(w[1 if grouped and lo >= cut else 0]), None, q8.Q8_ACT_NONE)


def test_calls_on_two_streams_at_once():
    """Products of every form on one stream while others run on a second one, each with what it gives alone."""
    sizes = [(4096, 2400, 2100), (2, 200, 8192), (24, 1000, 4096), (1300, 1000, 96), (700, 384, 512)]
    calls = []
    for M, N, K in sizes:
        x, W = values((M, K), M, torch.bfloat16), q8.q8_mx4_quantize(weights((N, K), 2))
        calls.append(lambda word, x=x, W=W: q8.q8_mx4_linear(x, W, act=q8.Q8_ACT_GELU, dev_status=word))
    x, W = values((500, 512), 1), q8.q8_mx4_quantize(weights((6, 300, 512), 2))
    offsets = torch.tensor([0, 100, 100, 230, 231, 400, 500], dtype=torch.int32).cuda()
    calls.append(lambda word: q8.q8_mx4_linear_grouped(x, offsets, W, dev_status=word))
    word = status_word()
    want = [c(word) for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i in range(120):
        for s, stream in enumerate(streams):
            k = (i + 3 * s) % len(calls)
            with torch.cuda.stream(stream):
                y = calls[k](word)
                if i % 10 == 9:
                    got.append((k, y))
    torch.cuda.synchronize()
    assert word.item() == 0
    assert len(got) == 24 and all(torch.equal(y, want[k]) for k, y in got)


def test_first_call_of_a_process_is_captured():
    """What a call sets up once (function attributes, the status word's address) may be set up while a stream is captured."""
    code = """
import torch
from paper_1910_06188_b200 import binding as q8
x, w = torch.randn(600, 96, device="cuda"), torch.randn(256, 96, device="cuda")
few, many, offsets = x[:2].clone(), w.reshape(2, 128, 96), torch.tensor([0, 10, 600], dtype=torch.int32, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    W = q8.q8_mx4_quantize(w)
    got = [q8.q8_mx4_linear(x, W), q8.q8_mx4_linear(few, W), q8.q8_mx4_linear_grouped(x, offsets, q8.q8_mx4_quantize(many)),
           q8.q8_mx4_fake_quantize(x), q8.q8_mx4_ste_backward(x)]
graph.replay()
torch.cuda.synchronize()
W = q8.q8_mx4_quantize(w)
want = [q8.q8_mx4_linear(x, W), q8.q8_mx4_linear(few, W), q8.q8_mx4_linear_grouped(x, offsets, q8.q8_mx4_quantize(many)),
        q8.q8_mx4_fake_quantize(x), x]
assert all(torch.equal(a, b) for a, b in zip(got, want))
assert q8.q8_mx4_status() == (0, 0)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
