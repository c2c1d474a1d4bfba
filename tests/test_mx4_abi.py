"""Host-only checks of the MXFP4 entry points: sizes, refusals before anything touches the device, and what the reference itself does."""
import numpy as np
import pytest
import torch

from paper_1910_06188_b200 import binding as q8
from paper_1910_06188_b200 import build
from tests import mx4_reference as ref

FAKE = 0x10000  # never dereferenced
FAR = 0x10000000
MANY = 1 << 60


@pytest.fixture(scope="module")
def lib():
    build.build()
    return q8.load()


def test_sizes(lib):
    assert [q8.q8_mx4_bytes(1, r, K) // 17408 for r, K in ((1, 1), (128, 256), (129, 256), (128, 257), (0, 5))] == [1, 1, 2, 2, 0]
    assert q8.q8_mx4_bytes(3, 130, 600) == 3 * 2 * 3 * 17408
    assert q8.q8_mx4_bytes(1, -1, 4) == q8.q8_mx4_bytes(1, 4, 0) == q8.q8_mx4_bytes(1 << 30, 4, 4) == 0
    assert q8.q8_mx4_linear_workspace_bytes(3, 64) == 0 and q8.q8_mx4_linear_workspace_bytes(130, 300) == 2 * 2 * 17408
    assert q8.q8_mx4_linear_grouped_workspace_bytes(300, 7, 64) == (2 + 7) * 17408
    assert q8.q8_mx4_linear_grouped_workspace_bytes(4, 1000, 64) == 4 * 17408
    assert q8.q8_mx4_linear_grouped_workspace_bytes(4, 1025, 64) == 0


def linear(lib, X=FAKE, xt=0, ldx=64, Wq=FAKE, bias=None, act=0, Y=FAR, yt=0, ldy=8, M=4, N=8, K=64, ws=FAKE, size=MANY, word=None):
    return lib.q8_mx4_linear(X, xt, ldx, Wq, bias, act, Y, yt, ldy, M, N, K, ws, size, word, None)


def linear_q(lib, Xq=FAKE, Wq=FAKE, bias=None, act=0, Y=FAKE, yt=0, ldy=8, M=4, N=8, K=64, word=None):
    return lib.q8_mx4_linear_q(Xq, Wq, bias, act, Y, yt, ldy, M, N, K, word, None)


def grouped(lib, X=FAKE, xt=0, ldx=64, x_rows=4, rows=None, offsets=FAKE, E=3, Wq=FAKE, bias=None, act=0, Y=FAR, yt=0, ldy=8, T=4, N=8, K=64,
            ws=FAKE, size=MANY, word=None):
    return lib.q8_mx4_linear_grouped(X, xt, ldx, x_rows, rows, offsets, E, Wq, bias, act, Y, yt, ldy, T, N, K, ws, size, word, None)


def quantize(lib, X=FAKE, t=0, G=1, R=4, K=64, ld=64, out=FAKE, word=None):
    return lib.q8_mx4_quantize(X, t, G, R, K, ld, out, word, None)


def dequantize(lib, T=FAKE, G=1, R=4, K=64, Y=FAKE, t=0, ld=64):
    return lib.q8_mx4_dequantize(T, G, R, K, Y, t, ld, None)


def fake(lib, X=FAKE, t=0, R=4, K=64, ld=64, out=FAR, ldo=64, word=None):
    return lib.q8_mx4_fake_quantize(X, t, R, K, ld, out, ldo, word, None)


@pytest.mark.parametrize("call,arguments,status", [
    *[(linear, {k: None, "M": 130}, q8.Q8_ERR_NULL) for k in ("X", "Wq", "Y", "ws")],
    *[(linear_q, {k: None}, q8.Q8_ERR_NULL) for k in ("Xq", "Wq", "Y")],
    *[(grouped, {k: None}, q8.Q8_ERR_NULL) for k in ("X", "offsets", "Wq", "Y", "ws")],
    *[(quantize, {k: None}, q8.Q8_ERR_NULL) for k in ("X", "out")],
    *[(dequantize, {k: None}, q8.Q8_ERR_NULL) for k in ("Y", "T")],
    *[(fake, {k: None}, q8.Q8_ERR_NULL) for k in ("X", "out")],
    *[(call, {k: 3}, q8.Q8_ERR_ARG) for call in (linear, grouped) for k in ("xt", "yt", "act")],
    *[(call, {"t": 7}, q8.Q8_ERR_ARG) for call in (quantize, dequantize, fake)],
    (linear_q, {"act": -1}, q8.Q8_ERR_ARG), (linear_q, {"yt": 3}, q8.Q8_ERR_ARG),
    # outputs that overlap an input: in place with another pitch, one row or one value into it, as the input's columns, of another pitch
    (fake, {"out": FAKE, "ldo": 65}, q8.Q8_ERR_ARG), (fake, {"out": FAKE + 256}, q8.Q8_ERR_ARG), (fake, {"out": FAKE + 4}, q8.Q8_ERR_ARG),
    (fake, {"ld": 100, "ldo": 100, "out": FAKE + 4 * 40}, q8.Q8_ERR_ARG), (fake, {"ld": 100, "ldo": 100, "out": FAKE - 4 * 20}, q8.Q8_ERR_ARG),
    (linear, {"Y": FAKE}, q8.Q8_ERR_ARG), (linear, {"Y": FAKE + 4 * 255, "ldy": 64}, q8.Q8_ERR_ARG), (linear, {"Y": FAKE - 4 * 25}, q8.Q8_ERR_ARG),
    (linear, {"M": 130, "Y": FAKE + 4 * 64 * 129}, q8.Q8_ERR_ARG), (linear, {"ldx": 72, "ldy": 72, "Y": FAKE + 4 * 60}, q8.Q8_ERR_ARG),
    (grouped, {"Y": FAKE + 8}, q8.Q8_ERR_ARG), (grouped, {"rows": FAKE, "x_rows": 100, "Y": FAKE + 4 * 64 * 99}, q8.Q8_ERR_ARG),
    *[(call, bad, q8.Q8_ERR_SHAPE) for call in (linear, linear_q) for bad in (
        {"M": -1}, {"N": -1}, {"K": 0}, {"K": -5}, {"K": (1 << 24) + 1, "ldx": 1 << 30} if call is linear else {"K": (1 << 24) + 1}, {"ldy": 7},
        {"M": 1 << 31}, {"N": 1 << 31, "ldy": 1 << 32}, {"M": 1 << 30, "N": 1 << 30, "ldy": 1 << 30})],
    (linear, {"ldx": 63}, q8.Q8_ERR_SHAPE),
    *[(grouped, bad, q8.Q8_ERR_SHAPE) for bad in (
        {"T": -1}, {"T": 5}, {"E": -1}, {"E": 1025}, {"x_rows": -1}, {"x_rows": 3}, {"K": 0}, {"ldx": 1}, {"ldy": 7}, {"N": 1 << 30, "ldy": 1 << 30})],
    *[(quantize, bad, q8.Q8_ERR_SHAPE) for bad in ({"G": -1}, {"R": -1}, {"K": 0}, {"ld": 63}, {"G": 1 << 20, "R": 1 << 20})],
    (dequantize, {"ld": 1}, q8.Q8_ERR_SHAPE), (fake, {"ld": 1}, q8.Q8_ERR_SHAPE), (fake, {"ldo": 1}, q8.Q8_ERR_SHAPE),
    *[(linear, {k: (FAR if k == "Y" else FAKE) + o}, q8.Q8_ERR_ALIGN) for k, o in (("X", 2), ("Wq", 8), ("bias", 2), ("Y", 2), ("ws", 128), ("word", 2))],
    *[(linear_q, {k: FAKE + o}, q8.Q8_ERR_ALIGN) for k, o in (("Xq", 8), ("Wq", 8), ("bias", 2), ("Y", 2), ("word", 2))],
    *[(grouped, {k: (FAR if k == "Y" else FAKE) + o}, q8.Q8_ERR_ALIGN) for k, o in (("X", 2), ("rows", 2), ("offsets", 2), ("Wq", 8), ("bias", 2), ("Y", 2), ("ws", 128))],
    (linear, {"xt": 1, "X": FAKE + 1}, q8.Q8_ERR_ALIGN), (quantize, {"X": FAKE + 2}, q8.Q8_ERR_ALIGN), (quantize, {"out": FAKE + 4}, q8.Q8_ERR_ALIGN),
    (dequantize, {"T": FAKE + 4}, q8.Q8_ERR_ALIGN), (fake, {"out": FAR + 1}, q8.Q8_ERR_ALIGN),
    (linear, {"M": 130, "size": 2 * 17408 - 1}, q8.Q8_ERR_WORKSPACE), (grouped, {"size": 3 * 17408 - 1}, q8.Q8_ERR_WORKSPACE),
    # nothing to do: never reaches the device
    *[(call, {k: 0}, q8.Q8_OK) for call in (linear, linear_q) for k in ("M", "N")], *[(grouped, {k: 0}, q8.Q8_OK) for k in ("T", "N", "E")],
    *[(quantize, {k: 0, "X": None}, q8.Q8_OK) for k in ("G", "R")], (dequantize, {"R": 0}, q8.Q8_OK), (fake, {"R": 0, "X": None}, q8.Q8_OK)])
def test_refusals(lib, call, arguments, status):
    assert call(lib, **arguments) == status



TILE = 17408


@pytest.mark.parametrize("call,arguments", [
    # values on their own tiles; an output on tiles or on the workspace, at the first byte and the last; an input on the workspace
    (quantize, {"out": FAKE}), (quantize, {"out": FAKE + 1008}), (quantize, {"X": FAKE + TILE - 4}), (dequantize, {}), (dequantize, {"Y": FAKE + TILE - 4}),
    (dequantize, {"Y": FAKE - 1020}),
    (linear_q, {"Xq": FAR, "Wq": FAKE}), (linear_q, {"Xq": FAKE, "Wq": FAR}), (linear_q, {"Xq": FAR, "Y": FAKE + TILE - 4}),
    (linear, {"Y": FAR, "Wq": FAR}), (linear, {"Y": FAR + TILE - 4, "Wq": FAR}),
    (linear, {"M": 130, "Y": FAR, "ws": FAR}), (linear, {"M": 130, "Y": FAR + 2 * TILE - 4, "ws": FAR}), (linear, {"M": 130, "X": FAKE, "ws": FAKE}),
    (grouped, {"Wq": FAR}), (grouped, {"Y": FAR + 3 * TILE - 4, "Wq": FAR}), (grouped, {"ws": FAR}), (grouped, {"ws": FAKE}),
    (grouped, {"x_rows": 1000, "rows": FAR, "X": FAKE, "ws": FAKE + 256 * 900})])
def test_memory_used_twice_is_refused(lib, call, arguments):
    assert call(lib, **arguments) == q8.Q8_ERR_ARG


# every pointer at a place of its own
APART = dict(X=1 << 32, Wq=2 << 32, Y=3 << 32, ws=4 << 32)
GROUPED = dict(APART, offsets=5 << 32, rows=6 << 32, bias=7 << 32)


@pytest.mark.parametrize("call,arguments", [
    # Y [4, 8] fp32 over the bias, its first value and its last, and the other way round; in rows 100 values apart on one row, or with a bias longer than that
    *[(linear, dict(APART, **more)) for more in (
        {"bias": APART["Y"]}, {"bias": APART["Y"] + 4 * 31}, {"bias": APART["Y"] - 4 * 7}, {"ldy": 100, "bias": APART["Y"] + 4 * 307},
        {"ldy": 100, "bias": APART["Y"] + 4 * 93}, {"ldy": 100, "N": 60, "bias": APART["Y"] + 4 * 41})],
    *[(linear_q, dict(Xq=1 << 32, Wq=2 << 32, Y=3 << 32, bias=(3 << 32) + o)) for o in (0, 4 * 31, -4 * 7)],
    # a workspace over weights and bias
    *[(linear, dict(APART, M=130, **more)) for more in (
        {"ws": APART["Wq"]}, {"ws": APART["Wq"] + 256 * ((TILE - 1) // 256)}, {"ws": APART["Wq"] - 2 * TILE + 256}, {"bias": APART["ws"]},
        {"bias": APART["ws"] + 2 * TILE - 4}, {"bias": APART["ws"] - 4 * 7})],
    # the grouped layer: Y, and the workspace (3 tiles), over weights, bias [3, 8], offsets [4] and rows [4]
    *[(grouped, dict(GROUPED, **{k: GROUPED["Y"] + o})) for k, n in (("bias", 24), ("offsets", 4), ("rows", 4)) for o in (0, 4 * 31, -4 * (n - 1))],
    *[(grouped, dict(GROUPED, **{k: GROUPED["ws"] + o})) for k, n in (("bias", 24), ("offsets", 4), ("rows", 4)) for o in (0, 3 * TILE - 4, -4 * (n - 1))],
    (grouped, dict(GROUPED, ws=GROUPED["Wq"])), (grouped, dict(GROUPED, ws=GROUPED["Wq"] + 256)), (grouped, dict(GROUPED, ws=GROUPED["Wq"] - 3 * TILE + 256))])
def test_outputs_and_workspaces_over_every_input_are_refused(lib, call, arguments):
    assert call(lib, **arguments) == q8.Q8_ERR_ARG


@pytest.mark.parametrize("call,arguments", [
    (quantize, {"ld": 1 << 55}), (quantize, {"G": 1 << 10, "R": 1 << 10, "ld": 1 << 37}), (dequantize, {"ld": 1 << 62}), (fake, {"ldo": 1 << 55}),
    (linear, {"ldx": 1 << 55}), (linear, {"ldy": 1 << 55}), (linear_q, {"ldy": (1 << 63) - 1}), (grouped, {"ldx": 1 << 55}), (grouped, {"ldy": 1 << 55})])
def test_rows_too_far_apart_are_refused(lib, call, arguments):
    assert call(lib, **arguments) == q8.Q8_ERR_SHAPE


def test_status_word_needs_a_place(lib):
    assert lib.q8_mx4_status_word(None) == q8.Q8_ERR_NULL


def test_tensors_of_the_host_are_refused(lib):
    W = q8.Mx4(torch.zeros(17408, dtype=torch.uint8), (8, 64))
    with pytest.raises(TypeError, match="X must be a CUDA tensor"):
        q8.q8_mx4_quantize(torch.zeros(4, 64))
    with pytest.raises(TypeError, match="CUDA tensor"):
        q8.q8_mx4_linear(torch.zeros(4, 64), W)
    with pytest.raises(TypeError, match="CUDA tensor"):
        q8.q8_mx4_dequantize(W)
    with pytest.raises(TypeError, match="CUDA tensor"):
        q8.q8_mx4_fake_quantize(torch.zeros(4, 64))
    with pytest.raises(ValueError, match="2 or 3 dimensions"):
        q8.q8_mx4_quantize(torch.zeros(64))


# ---------------------------------------------------------------- the reference
def test_reference_rounds_to_the_nearest_of_all_values():
    r = np.random.RandomState(0)
    x = r.standard_normal((200, 64)) * np.exp(r.standard_normal((200, 1)) * 20)
    code, E = ref.quantize(x)
    got = ref.values(code, E, 64).reshape(200, 2, 32)
    every = np.concatenate([ref.GRID, -ref.GRID])[None, None, None, :] * 2.0 ** (E - 127.0)[..., None, None]
    off = np.abs(x.reshape(200, 2, 32)[..., None] - every).min(-1)
    assert np.array_equal(np.abs(x.reshape(200, 2, 32) - got), off)
    top = np.abs(x).reshape(200, 2, 32).max(-1) / 2.0 ** (E - 127.0)
    assert ((top >= 4) & (top < 8)).all()


def test_reference_on_an_example_by_hand():
    """max 5 -> s = 2^(2 - 2) = 1; 0.25, 2.5, 5 are ties and go to 0, 2, 4; 0.75 goes to 1, -3.5 to -4."""
    x = np.zeros((1, 32))
    x[0, :8] = [5, 0.25, 2.5, 0.75, -3.5, 0.3, -0.2, 1.6]
    code, E = ref.quantize(x)
    assert E.tolist() == [[127]]
    assert ref.values(code, E, 8).tolist() == [[4, 0, 2, 1, -4, 0.5, 0, 1.5]]
    assert code[0, :8].tolist() == [6, 0, 4, 2, 14, 1, 8, 3]
    assert ref.values(*ref.quantize(x * 2.0 ** -30), 8).tolist() == (ref.values(code, E, 8) * 2.0 ** -30).tolist()


@pytest.mark.parametrize("grad_out,dtype,numel,grad_in,status", [
    (None, 2, 8, FAR, q8.Q8_ERR_NULL), (FAKE, 2, 8, None, q8.Q8_ERR_NULL), (FAKE, 3, 8, FAR, q8.Q8_ERR_ARG), (FAKE, -1, 8, FAR, q8.Q8_ERR_ARG),
    (FAKE, 0, -1, FAR, q8.Q8_ERR_SHAPE), (FAKE, 0, 1 << 57, FAR, q8.Q8_ERR_SHAPE), (FAKE + 2, 0, 8, FAR, q8.Q8_ERR_ALIGN), (FAKE, 1, 8, FAR + 1, q8.Q8_ERR_ALIGN),
    (FAKE, 2, 8, FAKE + 14, q8.Q8_ERR_ARG), (FAKE, 0, 8, FAKE - 28, q8.Q8_ERR_ARG), (FAKE, 2, 0, None, q8.Q8_OK), (FAKE, 2, 8, FAKE, q8.Q8_OK)])
def test_gradient_refusals(lib, grad_out, dtype, numel, grad_in, status):
    assert lib.q8_mx4_ste_backward(grad_out, dtype, numel, grad_in, None) == status
