"""The 8-bit operators of a transformer's inference pass: quantisation, dense layer, rotary positions, paged cache and its attention.

CPU: the structures' layout, the refusals, the host-side table of rotary phases.  GPU: every operator against its definition in 64 bits (written
here, apart from the kernels), with tolerances that count the roundings: half a step of the output type, 2^-23 of the sum of magnitudes
for each addition in 32 bits (rounded either way), 2^-11 for the probabilities.
"""
import ctypes as C
import math
import os
import subprocess
from decimal import Decimal, getcontext
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2201_05587_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
ADD = 2.0 ** -23
E4M3 = torch.float8_e4m3fn
gpu = pytest.mark.gpu


# ---- definitions in 64 bits -------------------------------------------------------------------------------------------
def ref_scale(most):
    """Smallest power of two s >= 2^-126 with most <= 448 s."""
    e = -126
    while most > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def ref_e4m3(v):
    """float64 -> nearest e4m3 value (ties to even); infinities and NaN -> NaN."""
    v = np.asarray(v, np.float64)
    with np.errstate(invalid="ignore"):
        _, e = np.frexp(np.where(np.isfinite(v), v, 0.0))
        step = np.ldexp(1.0, np.maximum(e - 4, -9))
        return np.where(np.isfinite(v), np.round(v / step) * step, np.nan)


def f8_values(t):
    return t.view(torch.uint8).cpu().view(E4M3).double().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


# ---- host side ----------------------------------------------------------------------------------------------------------
STRUCTS = ["tt_quantize_args", "tt_dense_quantized_args", "tt_rotary_args", "tt_cache", "tt_cache_append_args", "tt_cache_attention_args"]


def test_structures_have_the_layout_of_the_header(tmp_path):
    src = tmp_path / "s.c"
    lines = []
    for n in STRUCTS:
        lines.append(f'printf("{n} %zu", sizeof({n}));')
        lines += [f'printf(" %zu", offsetof({n}, {f}));' for f, _ in getattr(B, n)._fields_]
        lines.append('printf("\\n");')
    src.write_text('#include <stdio.h>\n#include "tt.h"\nint main(void) { %s return 0; }\n' % "\n".join(lines))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "s"), str(src)])
    for line in subprocess.check_output([str(tmp_path / "s")], text=True).splitlines():
        name, size, *offsets = line.split()
        t = getattr(B, name)
        assert C.sizeof(t) == int(size), name
        assert [getattr(t, f).offset for f, _ in t._fields_] == [int(o) for o in offsets], name


P = 1 << 20          # an address that a refused call never looks at


def quantize_args(**kw):
    a = dict(x=P, q=P, scales=P, x_row=256, q_row=256, s_row=1, s_block=4, x_type=B.TT_TYPE_BF16, m=4, kk=256, block_rows=1)
    a.update(kw)
    return B.tt_quantize_args(**a)


def dense_args(**kw):
    a = dict(x=P, w=P, x_scale=P, w_scale=P, bias=None, y=P, status=P, x_row=256, w_row=256, y_row=128, xs_row=1, xs_block=4, ws_row=2, ws_block=1,
             y_type=B.TT_TYPE_F32, m=4, nn=128, kk=256, act=B.TT_ACT_NONE)
    a.update(kw)
    return B.tt_dense_quantized_args(**a)


def rotary_args(**kw):
    a = dict(positions=P, turns=P, type=B.TT_TYPE_F16, position_bits=32, tokens=3, d=64, rot=64, interleaved=0, inverse=0, factor=1.0)
    arrays = dict(x=(P, P), y=(P, P), heads=(4, 2), x_token=(256, 128), x_head=(64, 64), y_token=(256, 128), y_head=(64, 64))
    for k, v in kw.items():
        (arrays if k in arrays else a)[k] = v
    r = B.tt_rotary_args(**a)
    for k, v in arrays.items():
        getattr(r, k)[0], getattr(r, k)[1] = v
    return r


def cache_struct(**kw):
    a = dict(table=P, table_row=8, pages=16, heads=2, block=64, d=128, batch=2, max_pages=8)
    arrays = dict(data=(P, P), scale=(P, P), page=(16384, 16384), head=(8192, 8192), token=(128, 128), s_page=(2, 2), s_head=(1, 1))
    for k, v in kw.items():
        (arrays if k in arrays else a)[k] = v
    r = B.tt_cache(**a)
    for k, v in arrays.items():
        getattr(r, k)[0], getattr(r, k)[1] = v
    return r


def append_args(cache=None, **kw):
    a = dict(cache=cache or cache_struct(), starts=P, lengths=P, status=P, type=B.TT_TYPE_BF16, tokens=6)
    x = kw.pop("x", (P, P))
    a.update(kw)
    r = B.tt_cache_append_args(**a)
    for i in range(2):
        r.x[i], r.x_token[i], r.x_head[i] = x[i], 256, 128
    return r


def attention_args(cache=None, **kw):
    a = dict(cache=cache or cache_struct(), q=P, y=P, q_token=512, q_head=128, y_token=512, y_head=128, starts=P, lengths=P, status=P, workspace=P,
             workspace_bytes=1 << 30, type=B.TT_TYPE_BF16, tokens=2, heads_q=4, causal=1, window=0, max_count=1, max_length=0, scale=0.1)
    a.update(kw)
    return B.tt_cache_attention_args(**a)


BAD, NOT = B.TT_ERR_INVALID_ARG, B.TT_ERR_NOT_IMPLEMENTED
REFUSED = [
    ("tt_quantize", quantize_args, [dict(x=None), dict(q=None), dict(scales=None), dict(x_row=255), dict(q_row=100), dict(m=-1), dict(kk=-1), dict(block_rows=64),
                                    dict(x_type=3), dict(x=P + 1), dict(scales=P + 2), dict(s_row=-1)], BAD),
    ("tt_dense_quantized", dense_args, [dict(x=None), dict(w=None), dict(x_scale=None), dict(w_scale=None), dict(y=None), dict(status=None), dict(x=P + 8), dict(w=P + 4),
                                        dict(x_row=264), dict(w_row=257), dict(x_row=128), dict(y_row=127), dict(m=-1), dict(nn=-1), dict(kk=0), dict(act=9), dict(act=-1),
                                        dict(y_type=3), dict(bias=P + 1), dict(y=P + 2), dict(xs_row=-1), dict(ws_block=-1)], BAD),
    ("tt_rotary", rotary_args, [dict(x=(None, P)), dict(y=(P, None)), dict(positions=None), dict(turns=None), dict(turns=P + 4), dict(position_bits=16), dict(rot=63), dict(rot=66),
                                dict(rot=-2), dict(tokens=-1), dict(type=7), dict(heads=(-1, 2)), dict(x=(P + 1, P)), dict(x_head=(-64, 64)), dict(positions=P + 2)], BAD),
    ("tt_cache_append", append_args, [dict(x=(None, P)), dict(starts=None), dict(lengths=None), dict(status=None), dict(tokens=-1), dict(type=5), dict(x=(P + 1, P))], BAD),
    ("tt_cache_append", lambda **kw: append_args(cache_struct(**kw)),
     [dict(data=(None, P)), dict(data=(P, P + 8)), dict(scale=(P, None)), dict(page=(16392, 16384)), dict(token=(120, 128)), dict(head=(8192, -16)), dict(table=None),
      dict(table_row=7), dict(pages=-1), dict(batch=-1), dict(max_pages=1 << 30, table_row=1 << 30)], BAD),
    ("tt_cache_append", lambda **kw: append_args(cache_struct(**kw)), [dict(block=8), dict(block=48), dict(block=256), dict(d=48), dict(d=288), dict(d=0)], NOT),
    ("tt_cache_attention", attention_args, [dict(q=None), dict(y=None), dict(starts=None), dict(lengths=None), dict(status=None), dict(type=B.TT_TYPE_F32), dict(heads_q=5), dict(tokens=-1),
                                            dict(window=-1), dict(window=4, causal=0), dict(max_count=-1), dict(max_length=-1), dict(scale=float("nan")), dict(q=P + 1), dict(q_token=-1)], BAD),
    ("tt_cache_attention", lambda **kw: attention_args(cache_struct(**kw)), [dict(data=(None, P)), dict(scale=(P + 1, P)), dict(head=(8, 8192)), dict(table_row=7)], BAD),
    ("tt_cache_attention", lambda **kw: attention_args(cache_struct(**kw)), [dict(block=24), dict(d=100), dict(d=512)], NOT),
]


@pytest.mark.parametrize("fn,make,cases,want", REFUSED, ids=[f"{i}-{r[0]}" for i, r in enumerate(REFUSED)])
def test_refusals(fn, make, cases, want):
    call = getattr(B.lib(), fn)
    assert call(None, None) == BAD
    for kw in cases:
        assert call(C.byref(make(**kw)), None) == want, kw


def test_sizes_and_strides_beyond_what_the_kernels_count():
    most, far = (1 << 31) - 1, 1 << 40
    for fn, make, cases in (("tt_quantize", quantize_args, [dict(m=most), dict(kk=most, x_row=most, q_row=most), dict(m=most, block_rows=128)]),
                            ("tt_dense_quantized", dense_args, [dict(m=most), dict(nn=most, y_row=most), dict(kk=most, x_row=1 << 31, w_row=1 << 31), dict(x_row=far), dict(w_row=far), dict(y_row=far)]),
                            ("tt_cache_append", lambda **kw: append_args(cache_struct(**kw)), [dict(page=(far, 16384)), dict(head=(8192, far)), dict(token=(far, 128))]),
                            ("tt_cache_attention", lambda **kw: attention_args(cache_struct(**kw)), [dict(page=(16384, far)), dict(head=(far, 8192)), dict(token=(128, far))])):
        for kw in cases:
            assert getattr(B.lib(), fn)(C.byref(make(**kw)), None) == BAD, (fn, kw)


def test_a_split_attention_needs_its_workspace():
    long = cache_struct(max_pages=2048, table_row=2048)
    n = C.c_int64()
    assert B.lib().tt_cache_attention_workspace(C.byref(attention_args(long)), C.byref(n)) == B.TT_OK and n.value > 0
    for kw in (dict(workspace=None), dict(workspace=P + 4), dict(workspace_bytes=n.value - 1)):
        assert B.lib().tt_cache_attention(C.byref(attention_args(long, **kw)), None) == BAD, kw
    assert B.lib().tt_cache_attention_workspace(C.byref(attention_args(long, max_length=100)), C.byref(n)) == B.TT_OK and n.value == 0
    assert B.lib().tt_cache_attention_workspace(None, C.byref(n)) == BAD
    assert B.lib().tt_cache_attention_workspace(C.byref(attention_args(long)), None) == BAD


def test_nothing_to_do_is_ok_and_without_a_gpu_the_rest_is_an_error():
    lib = B.lib()
    for fn, a in (("tt_quantize", quantize_args(m=0)), ("tt_quantize", quantize_args(kk=0)), ("tt_dense_quantized", dense_args(m=0)), ("tt_dense_quantized", dense_args(nn=0)),
                  ("tt_rotary", rotary_args(tokens=0)), ("tt_rotary", rotary_args(heads=(0, 0))), ("tt_cache_append", append_args(tokens=0)),
                  ("tt_cache_append", append_args(cache_struct(batch=0))), ("tt_cache_attention", attention_args(tokens=0)), ("tt_cache_attention", attention_args(heads_q=0))):
        assert getattr(lib, fn)(C.byref(a), None) == B.TT_OK, fn
    if not torch.cuda.is_available():
        for fn, a in (("tt_quantize", quantize_args()), ("tt_dense_quantized", dense_args()), ("tt_rotary", rotary_args()), ("tt_cache_append", append_args()), ("tt_cache_attention", attention_args())):
            assert getattr(lib, fn)(C.byref(a), None) == B.TT_ERR_CUDA, fn


def test_the_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    with pytest.raises(B.TTError):
        B.quantize(x, torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(2, 4))              # not on a GPU
    with pytest.raises(B.TTError):
        B.quantize(x, torch.zeros(4, 255, dtype=torch.uint8), torch.zeros(2, 4))
    with pytest.raises(B.TTError):
        B.dense_quantized(x, torch.zeros(2, 4), x, torch.zeros(1, 2), torch.zeros(4, 4))
    with pytest.raises(B.TTError):
        B.rotary(x, torch.zeros(4, dtype=torch.int32), torch.zeros(8, dtype=torch.int64))


def test_rotary_turns_are_exact_to_the_last_of_64_bits():
    getcontext().prec = 60
    pi = Fraction(Decimal("3.14159265358979323846264338327950288419716939937510582097494"))
    f = B.rotary_frequencies(128) + [0.0, 1.0, math.pi, 2 * math.pi, -0.3, 1e-9, 1234.5, 2.0 ** -80]
    got = [v % (1 << 64) for v in B.rotary_table(f, device="cpu").tolist()]
    for v, t in zip(f, got):
        want = Fraction(v) / (2 * pi) % 1 * (1 << 64)
        far = abs(want - t)
        # the quotient and its fraction in an extended mantissa of 64 bits: half a unit each of what lies above the point, and the rounding
        assert min(far, (1 << 64) - far) <= 1 + abs(Fraction(v)) / (2 * pi) * 2, v
    for bad in (math.inf, math.nan):
        with pytest.raises(B.TTError):
            B.rotary_table([1.0, bad], device="cpu")


def test_rotary_frequencies_are_scaled_as_stated():
    f = B.rotary_frequencies(64)
    assert f == [10000.0 ** (-2.0 * i / 64) for i in range(32)]
    assert B.rotary_frequencies(64, scaling="linear", factor=4.0) == [v / 4.0 for v in f]
    g = B.rotary_frequencies(64, scaling="base", factor=4.0)
    assert g[0] == 1.0 and abs(g[-1] * 4.0 / f[-1] - 1) < 1e-12
    g = B.rotary_frequencies(64, scaling="by_parts", factor=4.0, context=4096)
    assert g[0] == f[0] and abs(g[-1] * 4.0 / f[-1] - 1) < 1e-12 and all(v / 4 * (1 - 1e-12) <= u <= v for u, v in zip(g, f))
    with pytest.raises(B.TTError):
        B.rotary_frequencies(63)
    with pytest.raises(B.TTError):
        B.rotary_frequencies(64, scaling="other")


# ---- GPU: quantisation --------------------------------------------------------------------------------------------------
def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def f8_matrix(rows, cols, fill=0):
    """e4m3 [rows, cols] whose rows start on 16-byte boundaries, and the whole buffer with its padding."""
    whole = torch.full((rows, -(-max(cols, 1) // 16) * 16 + 16), fill, dtype=torch.uint8, device="cuda")
    return whole.view(E4M3)[:, :cols], whole


def run_quantize(x, rows):
    m, k = x.shape
    q, whole = f8_matrix(m, k, 0x55)
    kb, mb = -(-k // 128), -(-m // rows)
    scales = torch.full((kb + 1, mb + 1), -7.0, device="cuda")
    B.quantize(x, q, scales[:kb, :mb], block_rows=rows).run()
    torch.cuda.synchronize()
    assert (whole[:, k:] == 0x55).all() and (scales[kb] == -7).all() and (scales[:, mb] == -7).all()      # nothing beside the outputs
    return f8_values(q), scales[:kb, :mb].cpu().double().numpy()


def check_quantize(x, rows):
    m, k = x.shape
    q, scales = run_quantize(x, rows)
    v = x.double().cpu().numpy()
    for i in range(scales.shape[1]):
        for b in range(scales.shape[0]):
            at = np.s_[i * rows:(i + 1) * rows, b * 128:(b + 1) * 128]
            fine = np.abs(v[at][np.isfinite(v[at])])
            s = ref_scale(fine.max() if fine.size else 0.0)
            assert scales[b, i] == s, (b, i)
            assert same(q[at], ref_e4m3(v[at] / s)), (b, i)


@gpu
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("m,k", [(1, 1), (1, 128), (3, 130), (7, 1000), (129, 257), (2, 4096), (200, 1031)])
def test_quantize(kind, rows, m, k):
    x = (torch.randn(m, k, generator=gen(m * k), device="cuda") * torch.exp(2 * torch.randn(k, generator=gen(k), device="cuda"))).to(TYPES[kind])
    check_quantize(x, rows)


@gpu
def test_quantize_many_rows_and_strided_ones():
    x = torch.randn(1030, 2200, generator=gen(1), device="cuda").to(torch.bfloat16)      # (the form with four loads under way)
    check_quantize(x[:, :2049], 1)
    check_quantize(x[::2, 8:1008], 1)              # rows on 16-byte boundaries
    check_quantize(x[:77, 3:700], 1)               # ... and on none
    check_quantize(x[:140, 5:260], 128)


@gpu
@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_values_at_the_borders(rows):
    x = torch.zeros(9, 256, device="cuda")
    x[1, :4] = torch.tensor([448.0, -448.0, 1.0, 2.0 ** -9], device="cuda")
    x[2, :4] = torch.tensor([math.nextafter(448.0, 500.0) + 2.0 ** -15, 1.0, 17.0, 19.0], device="cuda")      # just over a border; ties
    x[3, :4] = torch.tensor([3.4028234e38, -1.0, 1e30, 2.0 ** -149], device="cuda")
    x[4, :4] = torch.tensor([2.0 ** -149, 2.0 ** -140, 0.0, -2.0 ** -149], device="cuda")
    x[5, :4] = torch.tensor([math.inf, -math.inf, math.nan, 5.0], device="cuda")
    x[6, :4] = torch.tensor([math.nan, 0.0, 0.0, 0.0], device="cuda")
    x[7, :4] = torch.tensor([2.0 ** -118, 448 * 2.0 ** -126, 0.0, 1e-39], device="cuda")
    check_quantize(x, rows)
    if rows == 1:
        for i in range(9):
            check_quantize(x[i:i + 1, :4], 1)


# ---- GPU: dense layer -----------------------------------------------------------------------------------------------------
def random_f8(rows, cols, seed, spread=1.0):
    q, whole = f8_matrix(rows, cols, 0x7f)                     # (what lies between the rows is NaN)
    q.view(torch.uint8).copy_((torch.randn(rows, cols, generator=gen(seed), device="cuda") * spread * 30).clamp(-448, 448).to(E4M3).view(torch.uint8))
    return q


def act64(v, act):
    if act == B.TT_ACT_RELU:
        return np.maximum(v, 0)
    if act == B.TT_ACT_RELU6:
        return np.clip(v, 0, 6)
    if act == B.TT_ACT_GELU_ERF:
        return 0.5 * v * (1 + np.vectorize(math.erf)(v / math.sqrt(2)))
    return v


def dense_case(m, n, k, seed=0):
    x, w = random_f8(m, k, seed + 1), random_f8(n, k, seed + 2)
    kb, nb = -(-k // 128), -(-n // 128)
    xs = torch.exp(torch.randn(kb, m, generator=gen(seed + 3), device="cuda")) * 2.0 ** -5
    ws = torch.exp(torch.randn(nb, kb, generator=gen(seed + 4), device="cuda")) * 2.0 ** -7
    return x, xs, w, ws


def dense_reference(x, xs, w, ws, bias):
    n, k = w.shape
    a = f8_values(x) * np.repeat(xs.cpu().double().numpy(), 128, axis=0)[:k].T
    b = f8_values(w) * np.repeat(np.repeat(ws.cpu().double().numpy(), 128, axis=0)[:n], 128, axis=1)[:, :k]
    y, most = a @ b.T, np.abs(a) @ np.abs(b).T
    if bias is not None:
        y, most = y + bias.cpu().double().numpy(), most + np.abs(bias.cpu().double().numpy())
    return y, most


def check_dense(m, n, k, kind="f32", act=B.TT_ACT_NONE, bias=True, seed=0, pad=3):
    x, xs, w, ws = dense_case(m, n, k, seed)
    b = torch.randn(n, generator=gen(seed + 5), device="cuda") if bias else None
    whole = torch.full((m + 2, n + pad), -77.0, dtype=TYPES[kind], device="cuda")
    y = whole[1:m + 1, :n]
    call = B.dense_quantized(x, xs, w, ws, y, bias=b, act=act)
    call.run()
    assert call.status() == B.TT_OK
    first = y.clone()
    call.run()
    torch.cuda.synchronize()
    assert torch.equal(first, y)
    assert (whole[0] == -77).all() and (whole[-1] == -77).all() and (whole[:, n:] == -77).all()
    ref, most = dense_reference(x, xs, w, ws, b)
    got = y.double().cpu().numpy()
    # every product, scale and addition in 32 bits; GELU has a slope of at most 1.13 and an absolute error of 1.5e-7 |v| of its own
    off = most * ADD * (128 + 3 * (k // 128 + 1) + 8) * 1.13 + (np.abs(ref) * 2e-7 if act == B.TT_ACT_GELU_ERF else 0)
    ref = act64(ref, act)
    assert (np.abs(got - ref) <= off + HALF_STEP[TYPES[kind]] * (np.abs(ref) + off) + 2.0 ** -25).all(), np.max(np.abs(got - ref) / (off + 1e-30))


@gpu
@pytest.mark.parametrize("m", [1, 7, 16, 17, 33, 64, 65, 129, 300])
@pytest.mark.parametrize("n,k", [(1, 1), (64, 128), (130, 300), (1000, 1031), (257, 2048)])
def test_dense(m, n, k):
    check_dense(m, n, k, bias=(m + n) % 2 == 0)


@gpu
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("act", [B.TT_ACT_NONE, B.TT_ACT_RELU, B.TT_ACT_RELU6, B.TT_ACT_GELU_ERF])
@pytest.mark.parametrize("m,pad", [(5, 8), (200, 8), (200, 3)])
def test_dense_types_and_activations(kind, act, m, pad):
    check_dense(m, 264, 640, kind=kind, act=act, pad=pad)


@gpu
@pytest.mark.parametrize("m,n,k", [(8, 4096, 4096), (1, 128, 8192), (128, 128, 8192), (600, 2304, 768), (1500, 1300, 500), (200, 2000, 1000), (4000, 128, 1000), (2000, 300, 2000), (130, 4096, 1024), (64, 900, 3000), (30, 300, 8000)])
def test_dense_larger(m, n, k):
    check_dense(m, n, k)


@gpu
def test_dense_scales_of_any_strides_and_extremes():
    m, n, k = 40, 300, 500
    x, xs, w, ws = dense_case(m, n, k, 9)
    xs = xs.t().contiguous().t()                    # a token's scales side by side
    ws = ws.t().contiguous().t()
    xs[0, 3], xs[1, 4], ws[1, 2] = 2.0 ** 100, 2.0 ** -126, 0.0
    y = torch.empty(m, n, device="cuda")
    B.dense_quantized(x, xs, w, ws, y).run()
    ref, most = dense_reference(x, xs, w, ws, None)
    assert (np.abs(y.double().cpu().numpy() - ref) <= most * ADD * 160).all()
    x.view(torch.uint8)[5, 7] = 0x7f                # a NaN reaches its row and no other
    B.dense_quantized(x, xs, w, ws, y).run()
    nan = torch.isnan(y).cpu().numpy()
    assert nan[5].all() and nan.sum() == n


@gpu
@pytest.mark.parametrize("m,n,k", [(1000, 3000, 640), (2500, 700, 1000), (257, 20000, 256), (5000, 129, 384)])
@pytest.mark.parametrize("kind,act,pad", [("f32", B.TT_ACT_NONE, 8), ("bf16", B.TT_ACT_GELU_ERF, 8), ("f16", B.TT_ACT_RELU6, 8), ("bf16", B.TT_ACT_RELU, 3)])
def test_dense_by_pairs(m, n, k, kind, act, pad):
    check_dense(m, n, k, kind=kind, act=act, pad=pad + (-n) % 8 if pad == 8 else pad)


@gpu
@pytest.mark.parametrize("m", [5, 100, 2000])
@pytest.mark.parametrize("act", [B.TT_ACT_NONE, B.TT_ACT_RELU, B.TT_ACT_RELU6, B.TT_ACT_GELU_ERF])
def test_dense_nan_stays_nan(m, act):
    x, xs, w, ws = dense_case(m, 2000, 300, 9)
    x.view(torch.uint8)[m - 1, 299] = 0x7f
    y = torch.empty(m, 2000, device="cuda")
    B.dense_quantized(x, xs, w, ws, y, act=act).run()
    nan = torch.isnan(y)
    assert nan[m - 1].all() and not nan[:m - 1].any()


@gpu
def test_dense_one_row_without_a_pitch():
    x, xs, w, ws = dense_case(1, 200, 100, 3)
    tight = torch.empty(112, dtype=torch.uint8, device="cuda")[:100].view(1, 100).view(E4M3)
    tight.view(torch.uint8).copy_(x.view(torch.uint8))
    y = torch.empty(1, 200, device="cuda")
    B.dense_quantized(tight, xs, w, ws, y).run()
    ref, most = dense_reference(x, xs, w, ws, None)
    assert (np.abs(y.double().cpu().numpy() - ref) <= most * ADD * 160).all()


# ---- GPU: rotary positions ------------------------------------------------------------------------------------------------
def rotary_reference(x, positions, freq, interleaved, factor, inverse):
    y = x.double().cpu().numpy().copy()
    half = len(freq)
    angle = np.array(positions, dtype=np.longdouble)[:, None] * np.array(freq, dtype=np.longdouble)[None, :]
    if inverse:
        angle = -angle
    angle = np.remainder(angle, 2 * np.longdouble("3.14159265358979323846264338327950288"))
    c, s = (np.cos(angle) * factor).astype(np.float64)[:, None], (np.sin(angle) * factor).astype(np.float64)[:, None]
    ia, ib = (np.s_[..., 0:2 * half:2], np.s_[..., 1:2 * half:2]) if interleaved else (np.s_[..., :half], np.s_[..., half:2 * half])
    a, b = y[ia].copy(), y[ib].copy()
    most = np.abs(y)
    most[ia] = most[ib] = np.abs(a) + np.abs(b)
    y[ia], y[ib] = a * c - b * s, b * c + a * s
    return y, most * abs(factor)


def check_rotary(xs, ys, positions, freq, interleaved, factor=1.0, inverse=False):
    want = [rotary_reference(x, positions.tolist(), freq, interleaved, factor, inverse) for x in xs]
    kept = [x.clone() for x in xs]
    B.rotary(xs, positions, B.rotary_table(freq), ys, interleaved=interleaved, factor=factor, inverse=inverse).run()
    for x, y, old, (ref, most) in zip(xs, ys or xs, kept, want):
        if ys is not None:
            assert torch.equal(x, old)
        got, rot = y.double().cpu().numpy(), 2 * len(freq)
        # the angle to 2^-25 half turns, sine and cosine to two steps, two products and a sum
        off = most * (math.pi * 2.0 ** -25 + 5 * 2.0 ** -23)
        assert (np.abs(got - ref) <= off + HALF_STEP[x.dtype] * (np.abs(ref) + off) + 2.0 ** -25)[..., :rot].all()
        assert np.array_equal(got[..., rot:], ref[..., rot:])


@gpu
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot", [(1, 1, 1, 2, 2), (5, 4, 2, 64, 64), (3, 8, 1, 128, 32), (130, 3, 3, 80, 40), (2, 4, 4, 96, 12), (17, 12, 12, 256, 256)])
def test_rotary(kind, interleaved, tokens, hq, hk, d, rot):
    xs = [torch.randn(tokens, h, d, generator=gen(h + d), device="cuda").to(TYPES[kind]) for h in (hq, hk)]
    ys = [torch.empty_like(x) for x in xs]
    positions = torch.randint(0, 1 << 20, (tokens,), generator=gen(5), device="cuda", dtype=torch.int32)
    check_rotary(xs, ys, positions, B.rotary_frequencies(rot, scaling="by_parts", factor=8.0) if rot > 2 else [1.0], interleaved, factor=1.2)


@gpu
def test_rotary_far_and_negative_positions_in_place_and_strided():
    freq = B.rotary_frequencies(64)
    for dtype, far in ((torch.int32, [0, 1, (1 << 31) - 1, -(1 << 31), -5]), (torch.int64, [0, 1 << 36, -(1 << 36), 7, 1 << 31])):
        positions = torch.tensor(far, dtype=dtype, device="cuda")
        packed = torch.randn(5, 6, 3, 64, generator=gen(1), device="cuda")          # queries, keys and values of a token side by side
        check_rotary([packed[:, :4, 0], packed[:, 4:, 1]], None, positions, freq, False)
        check_rotary([packed[:, :, 2]], None, positions, freq, True, inverse=True)
        off = torch.randn(5, 2, 67, generator=gen(2), device="cuda").to(torch.float16)
        check_rotary([off[..., 1:66]], [torch.empty(5, 2, 65, dtype=torch.float16, device="cuda")], positions, B.rotary_frequencies(64), False)


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_inverse_is_the_gradient(interleaved):
    freq, factor = B.rotary_frequencies(48), 1.3
    x, g = (torch.randn(9, 3, 64, generator=gen(i), device="cuda") for i in (1, 2))
    positions = torch.randint(0, 5000, (9,), generator=gen(3), device="cuda")
    table = B.rotary_table(freq)
    y, back, moved = torch.empty_like(x), torch.empty_like(g), torch.empty_like(x)
    B.rotary(x, positions, table, y, interleaved=interleaved, factor=factor).run()
    B.rotary(g, positions, table, back, interleaved=interleaved, factor=factor, inverse=True).run()
    # <R x, g> = <x, R^T g>, and the difference along any direction of the linear map
    size = float(x.abs().double().sum())
    assert abs(float((y.double() * g.double()).sum() - (x.double() * back.double()).sum())) <= size * 20 * 2.0 ** -22
    step = torch.randn(9, 3, 64, generator=gen(4), device="cuda")
    B.rotary(x + step, positions, table, moved, interleaved=interleaved, factor=factor).run()
    assert abs(float(((moved.double() - y.double()) * g.double()).sum() - (step.double() * back.double()).sum())) <= size * 60 * 2.0 ** -22


# ---- GPU: the cache -------------------------------------------------------------------------------------------------------
class Pages:
    """A cache for sequences of given lengths, filled with a pattern, its pages in random order."""

    def __init__(self, lengths, heads, d, block, seed=0, spare=3, by_token=False, random_values=True):
        g = gen(seed)
        need = [-(-n // block) for n in lengths]
        pages, most = sum(need) + spare, max(need + [1]) + 1
        shape = (pages, block, heads, d) if by_token else (pages, heads, block, d)
        self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
        if by_token:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.ks, self.vs = (torch.zeros(pages, heads, device="cuda") for _ in range(2))
        order = torch.randperm(pages, generator=g, device="cuda").tolist()
        self.table_cpu = [[order.pop() for _ in range(n)] for n in need]
        self.free = order
        table = torch.full((len(lengths), most), 1 << 30, dtype=torch.int32)           # (behind the last page: no page)
        for b, row in enumerate(self.table_cpu):
            table[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
        self.table, self.block, self.heads, self.d, self.lengths = table.cuda(), block, heads, d, list(lengths)
        if random_values:
            # values in the slots that are in use, 0x7f (NaN) in all others
            for b, row in enumerate(self.table_cpu):
                for j, p in enumerate(row):
                    n = min(block, lengths[b] - j * block)
                    for data, scale in ((self.k, self.ks), (self.v, self.vs)):
                        x = torch.randn(heads, n, d, generator=g, device="cuda") * torch.exp(torch.randn(heads, 1, 1, generator=g, device="cuda"))
                        data.view(torch.uint8)[p, :, :n] = (x * 60).clamp(-448, 448).to(E4M3).view(torch.uint8)
                        scale[p] = 2.0 ** torch.randint(-9, -4, (heads,), generator=g, device="cuda").float()

    def cache(self):
        return B.Cache(self.k, self.v, self.ks, self.vs, self.table)

    def values(self, b, which):
        """Keys (0) or values (1) of sequence b in 64 bits, [heads, length, d]."""
        data, scale = ((self.k, self.ks), (self.v, self.vs))[which]
        n = self.lengths[b]
        if n == 0:
            return np.zeros((self.heads, 0, self.d))
        rows = [data.view(torch.uint8)[p].contiguous().view(E4M3).double() * scale[p].double()[:, None, None] for p in self.table_cpu[b]]
        return torch.cat(rows, dim=1)[:, :n].cpu().numpy()


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def reference_append(p, counts, xs):
    """(bytes as values, scales) of keys and values after the append, in 64 bits."""
    out = []
    for x, data, scale in ((xs[0], p.k, p.ks), (xs[1], p.v, p.vs)):
        vals, sc = f8_values(data.contiguous()).reshape(data.shape), scale.double().cpu().numpy().copy()
        x, at = x.double().cpu().numpy(), 0
        for b, (count, length) in enumerate(zip(counts, p.lengths)):
            first = length - count
            for j in range(first // p.block, -(-length // p.block) if count else 0):
                lo, hi = max(first, j * p.block), min(length, (j + 1) * p.block)
                if lo >= hi:
                    continue
                page, held = p.table_cpu[b][j], lo - j * p.block
                for h in range(p.heads):
                    new = x[at + lo - first:at + hi - first, h]
                    fine = np.abs(new[np.isfinite(new)])
                    s = ref_scale(fine.max() if fine.size else 0.0)
                    if held:
                        s = max(s, sc[page, h])
                        if s != sc[page, h]:
                            vals[page, h, :held] = ref_e4m3(vals[page, h, :held] * (sc[page, h] / s))
                    sc[page, h] = s
                    vals[page, h, held:held + hi - lo] = ref_e4m3(new / s)
            at += count
        out.append((vals, sc))
    return out


def check_append(p, counts, xs, behind=0):
    want = reference_append(p, counts, xs)
    starts = int32([0] + list(np.cumsum(counts)))
    call = B.cache_append(p.cache(), xs[0], xs[1], starts, int32(p.lengths))
    call.run()
    assert call.status() == B.TT_OK
    for (vals, sc), data, scale in zip(want, (p.k, p.v), (p.ks, p.vs)):
        assert same(f8_values(data.contiguous()).reshape(data.shape), vals)
        assert np.array_equal(scale.double().cpu().numpy(), sc)


@gpu
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("heads,d,block", [(1, 32, 16), (2, 64, 32), (3, 96, 64), (2, 256, 128)])
def test_append(kind, heads, d, block):
    lengths, counts = [1, 5, 200, 17, 64, 130, 0, 33], [1, 5, 200, 1, 64, 3, 0, 32]
    p = Pages(lengths, heads, d, block, seed=d)
    extra = 4                                                   # tokens of a padded batch, which go nowhere
    xs = [(torch.randn(sum(counts) + extra, heads, d, generator=gen(7 + i), device="cuda") * torch.exp(2 * torch.randn(heads, 1, generator=gen(3), device="cuda"))).to(TYPES[kind]) for i in (0, 1)]
    check_append(p, counts, xs)


@gpu
def test_append_token_by_token_raises_the_scale():
    p = Pages([0], 2, 64, 32, spare=4, random_values=False)
    p.table_cpu = [[p.free.pop(), p.free.pop()]]
    p.table = int32([p.table_cpu[0]])
    for n in range(1, 41):
        p.lengths = [n]
        x = torch.randn(1, 2, 64, generator=gen(n), device="cuda") * 1.3 ** n
        check_append(p, [1], [x, -x / 3 ** n])


@gpu
def test_append_strided_tokens_and_pages_that_are_ordered_by_token():
    p = Pages([70, 40], 3, 64, 32, seed=2, by_token=True)
    packed = torch.randn(33, 5, 3, 65, generator=gen(1), device="cuda").to(torch.bfloat16)
    check_append(p, [30, 3], [packed[:, 0, :, :64], packed[:, 1, :, 1:]])
    p = Pages([70, 40], 3, 64, 32, seed=2)
    packed = torch.randn(33, 5, 3, 64, generator=gen(1), device="cuda").to(torch.float16)
    check_append(p, [30, 3], [packed[:, 0], packed[:, 3]])


@gpu
def test_append_of_what_is_not_finite_and_of_zeros():
    p = Pages([40, 20], 2, 32, 16, seed=4)
    x = torch.randn(23, 2, 32, generator=gen(1), device="cuda")
    x[3, 0, 5], x[4, 1, 2], x[5] = math.inf, math.nan, -math.inf
    check_append(p, [22, 1], [x, torch.zeros_like(x)])
    p = Pages([40, 20], 2, 32, 16, seed=4)
    p.ks.mul_(1.37)                                             # scales of another origin, which are no powers of two
    check_append(p, [2, 1], [x[:3] * 100, x[:3] * 1e-3])


@gpu
def test_append_reports_what_only_the_device_sees():
    for table, lengths, starts in (([[0, 1 << 30]], [20], [0, 10]), ([[-1, 1]], [10], [0, 10]), ([[0, 1]], [33], [0, 10]), ([[0, 1]], [5], [0, 10]), ([[0, 1]], [20], [0, 11]), ([[0, 1]], [20], [3, 1])):
        p = Pages([32], 1, 32, 16, seed=1)
        p.table = int32(table)
        x = torch.randn(10, 1, 32, generator=gen(1), device="cuda")
        call = B.cache_append(p.cache(), x, x, int32(starts), int32(lengths))
        call.run()
        assert call.status() == B.TT_ERR_INVALID_ARG, (table, lengths, starts)
        assert call.status() == B.TT_OK                         # (the look clears it)


@gpu
def test_append_reports_starts_that_do_not_rise_from_0():
    p = Pages([80, 80], 1, 32, 16, seed=1)
    before = p.k.view(torch.uint8).clone(), p.ks.clone()
    x = torch.randn(200, 1, 32, generator=gen(1), device="cuda")
    for starts in ([100, 110, 120], [100, 90, 120], [-40, -20, 0]):
        call = B.cache_append(p.cache(), x, x, int32(starts), int32([0, 0]))
        call.run()
        assert call.status() == B.TT_ERR_INVALID_ARG, starts
    assert torch.equal(before[0], p.k.view(torch.uint8)) and torch.equal(before[1], p.ks)


# ---- GPU: attention ---------------------------------------------------------------------------------------------------------
def reference_attention(p, counts, q, scale, causal, window):
    """Outputs and bounds of their errors in 64 bits, [tokens, heads_q, d]."""
    q = q.double().cpu().numpy()
    out, off, at, group = np.zeros_like(q), np.zeros_like(q), 0, q.shape[1] // p.heads
    for b, count in enumerate(counts):
        k, v, n = p.values(b, 0), p.values(b, 1), p.lengths[b]
        for i in range(count):
            pos = n - count + i
            hi = min(n, pos + 1) if causal else n
            lo = max(0, pos + 1 - window) if window else 0
            if hi <= lo:
                continue
            for h in range(q.shape[1]):
                kk, vv = k[h // group, lo:hi], v[h // group, lo:hi]
                s = kk @ q[at + i, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[at + i, h] = w @ vv
                # 2^-11 of each probability, its score's additions and products, its exponential, the sums
                score = (np.abs(kk) @ np.abs(q[at + i, h])).max() * abs(scale) * (p.d + 8) * ADD
                off[at + i, h] = (2.0 ** -11 + 2 * score + (np.abs(s - s.max()).max() + 16) * 2.0 ** -22 + (hi - lo) ** 0.5 * ADD) * (w @ np.abs(vv))
        at += count
    return out, off


def check_attention(p, counts, heads_q, kind="bf16", causal=True, window=0, seed=0, q=None, scale=None, want_call=False, max_count=0, max_length=0):
    tokens = sum(counts)
    if q is None:
        q = (torch.randn(tokens + 2, heads_q, p.d, generator=gen(seed + 50), device="cuda") * 2).to(TYPES[kind])
    scale = 1 / math.sqrt(p.d) if scale is None else scale
    y = torch.full_like(q, -77.0)
    starts = int32([0] + list(np.cumsum(counts)))
    call = B.cache_attention(p.cache(), q, y, starts, int32(p.lengths), scale, causal=causal, window=window, max_count=max_count, max_length=max_length)
    call.run()
    assert call.status() == B.TT_OK
    first = y.clone()
    y.fill_(-77.0)
    call.run()                                                  # (the workspace is ready again, and the order of sums the same)
    torch.cuda.synchronize()
    assert torch.equal(first, y)
    assert (y[tokens:] == -77).all()
    ref, off = reference_attention(p, counts, q[:tokens], scale, causal, window)
    got = y[:tokens].double().cpu().numpy()
    bad = np.abs(got - ref) > off + HALF_STEP[q.dtype] * (np.abs(ref) + off) + 2.0 ** -25
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])
    return (call, q, y, starts) if want_call else y


@gpu
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("block", [16, 64])
def test_attention_of_single_tokens(kind, d, block):
    p = Pages([1, 7, 16, 65, 200, 0, 300], 2, d, block, seed=d + block)
    check_attention(p, [1, 1, 1, 1, 1, 0, 1], 4, kind)


@gpu
@pytest.mark.parametrize("heads,heads_q", [(1, 1), (2, 14), (1, 8), (3, 48), (1, 40)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 37)])
def test_attention_of_several_tokens(heads, heads_q, causal, window):
    p = Pages([9, 50, 300, 64], heads, 64, 32, seed=heads)
    check_attention(p, [9, 3, 20, 1], heads_q, causal=causal, window=window)


@gpu
@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("window", [0, 100, 1000])
def test_attention_of_prompts(d, window):
    p = Pages([150, 333, 1000], 1, d, 128, seed=3)
    check_attention(p, [150, 130, 1], 2, "f16", window=window)


@gpu
@pytest.mark.parametrize("d", [32, 96])
@pytest.mark.parametrize("block", [16, 128])
@pytest.mark.parametrize("window", [0, 1000])
def test_attention_of_prompts_with_short_heads(d, block, window):
    p = Pages([700, 64, 1500, 20], 2, d, block, seed=d)
    check_attention(p, [300, 64, 40, 3], 6, window=window)
    p = Pages([6000], 1, d, block, seed=d + 1)
    check_attention(p, [70], 2, kind="f16", window=window)
    check_attention(p, [70], 2, causal=False)


@gpu
@pytest.mark.parametrize("length,window", [(5000, 0), (9001, 0), (9001, 4000)])
def test_attention_splits_a_long_sequence(length, window):
    p = Pages([length, 3, 2049], 2, 64, 64, seed=length)
    check_attention(p, [1, 1, 2], 8, window=window)
    check_attention(p, [1, 1, 2], 8, window=window, max_count=2, max_length=length)


@gpu
@pytest.mark.parametrize("batch", [33, 70, 1100])
@pytest.mark.parametrize("count,max_count", [(1, 1), (1, 0), (3, 3), (3, 0)])
def test_attention_of_large_batches(batch, count, max_count):
    lengths = [(17 * b) % 60 for b in range(batch)]
    counts = [min(n, 1 + b % count) if b % 7 else 0 for b, n in enumerate(lengths)]
    p = Pages(lengths, 1, 32, 16, seed=batch)
    check_attention(p, counts, 4, max_count=max_count)
    x = torch.randn(sum(counts), 1, 32, generator=gen(1), device="cuda")
    check_append(p, counts, [x, -x])


@gpu
def test_attention_rows_that_see_nothing_are_zeros():
    p = Pages([0, 3, 0], 1, 64, 16, seed=1)
    y = check_attention(p, [2, 5, 0], 2)                          # the first two queries of the second sequence stand in front of its tokens
    assert (y[:4] == 0).all() and (y[4:7] != 0).any()


@gpu
def test_attention_over_no_pages_at_all():
    for pages, columns in ((0, 3), (4, 0)):
        k = torch.zeros(pages, 2, 16, 64, dtype=torch.uint8, device="cuda").view(E4M3)
        s = torch.zeros(pages, 2, device="cuda")
        q = torch.randn(3, 4, 64, generator=gen(1), device="cuda").to(torch.bfloat16)
        y = torch.full_like(q, 5.0)
        call = B.cache_attention(B.Cache(k, k, s, s, torch.zeros(2, columns, dtype=torch.int32, device="cuda")), q, y, int32([0, 1, 3]), int32([0, 0]), 0.1)
        call.run()
        assert call.status() == B.TT_OK and (y == 0).all()


@gpu
def test_attention_by_token_layout_strided_queries_and_shared_pages():
    p = Pages([200, 180], 3, 64, 32, seed=5, by_token=True)
    p.table_cpu[1][:5] = p.table_cpu[0][:5]                      # a common beginning
    p.table[1, :5] = p.table[0, :5]
    packed = torch.randn(9, 12, 3, 64, generator=gen(1), device="cuda").to(torch.float16)
    check_attention(p, [4, 3], 6, q=packed[:, :6, 1])
    check_attention(p, [4, 3], 6, q=packed.transpose(0, 1).contiguous().transpose(0, 1)[:, 3:9, 0])
    odd = torch.randn(9, 6, 67, generator=gen(2), device="cuda").to(torch.bfloat16)
    check_attention(p, [4, 3], 6, q=odd[..., 3:])


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("offset", [0, 1, 4])                    # of 16 bytes, of 2, of 8
@pytest.mark.parametrize("heads,heads_q", [(2, 2), (1, 3), (2, 16)])
@pytest.mark.parametrize("counts,lengths", [([90, 150], [300, 150]), ([40], [5000])])
def test_attention_of_prompts_at_any_alignment(d, offset, heads, heads_q, counts, lengths):
    p, tokens = Pages(lengths, heads, d, 16, seed=d + offset), sum(counts)
    wide = (torch.randn(tokens, heads_q, d + 8, generator=gen(5), device="cuda") * 2).to(torch.float16)
    into = torch.full((tokens + 1, heads_q, d + 8), -77.0, dtype=torch.float16, device="cuda")
    q, y = wide[..., offset:offset + d], into[:tokens, :, offset:offset + d]
    call = B.cache_attention(p.cache(), q, y, int32([0] + list(np.cumsum(counts))), int32(lengths), 1 / math.sqrt(d))
    call.run()
    assert call.status() == B.TT_OK
    ref, off = reference_attention(p, counts, q, 1 / math.sqrt(d), True, 0)
    got = y.double().cpu().numpy()
    assert (np.abs(got - ref) <= off + HALF_STEP[torch.float16] * (np.abs(ref) + off) + 2.0 ** -25).all()
    y.fill_(-77.0)
    assert (into == -77.0).all()


@gpu
@pytest.mark.parametrize("n", [1348, 1349, 1351])
@pytest.mark.parametrize("kind", list(TYPES))
def test_dense_rows_that_begin_anywhere(n, kind):
    m, k = 3001, 200                                            # (pairs of CTAs: 3001 x 1348 tiles of 256)
    (x, xs, w, ws), bias = dense_case(m, n, k, seed=n), torch.randn(n, generator=gen(9), device="cuda")
    ref, most = dense_reference(x, xs, w, ws, bias)
    off = most * ADD * (k + 32)
    into = torch.full((m + 1, n + 5), -77.0, dtype=TYPES[kind], device="cuda")
    for first in (0, 1, 3):
        y = into[:m, first:first + n]
        call = B.dense_quantized(x, xs, w, ws, y, bias=bias)
        call.run()
        assert call.status() == B.TT_OK
        assert (np.abs(y.double().cpu().numpy() - ref) <= off + HALF_STEP[TYPES[kind]] * (np.abs(ref) + off) + 2.0 ** -25).all()
        y.fill_(-77.0)
        assert (into == -77.0).all()


@gpu
def test_attention_scales_that_differ_by_much():
    p = Pages([256], 1, 64, 16, seed=6)
    e = torch.linspace(-30, 8, p.ks.numel(), device="cuda").round().view_as(p.ks)
    p.vs = (2.0 ** e[torch.randperm(e.numel(), generator=gen(1), device="cuda")]).contiguous()
    # a page counts as much as its scale: the bound is on the sum of magnitudes, of which the largest pages have the most
    check_attention(p, [3], 2, "f16")
    p.vs.fill_(2.0 ** -126)
    p.vs[p.table_cpu[0][3]] = 1.0                                # (the scale of a page of zeros)
    check_attention(p, [3], 2, "f16")
    p.vs = (p.vs * 0 + 0.37).contiguous()
    p.ks = (p.ks * 1.7).contiguous()                             # no powers of two
    check_attention(p, [3], 2, "f16")


@gpu
def test_attention_of_large_and_small_queries():
    p = Pages([100], 1, 64, 16, seed=7)
    for size in (2.0 ** -100, 2.0 ** 90):
        q = (torch.randn(3, 2, 64, generator=gen(1), device="cuda") * size).to(torch.bfloat16)
        check_attention(p, [1], 2, q=q, scale=0.2 / size)
    q = (torch.randn(3, 2, 64, generator=gen(1), device="cuda") * 2.0 ** -18).to(torch.float16)
    check_attention(p, [1], 2, q=q, scale=2.0 ** 15)
    q = torch.zeros(3, 2, 64, dtype=torch.float16, device="cuda")
    check_attention(p, [1], 2, q=q)


@gpu
@pytest.mark.parametrize("d", [64, 128])
def test_attention_nan_reaches_the_rows_that_see_it(d):
    p = Pages([80], 1, d, 16, seed=8)
    counts = [40]
    for data, col in ((p.k, 3), (p.v, 5)):
        q = (torch.randn(40, 2, d, generator=gen(1), device="cuda")).to(torch.float16)
        clean = check_attention(p, counts, 2, q=q).clone()
        at = 61                                                   # seen by the queries 21 .. 39
        page, slot = p.table_cpu[0][at // 16], at % 16
        keep = data.view(torch.uint8)[page, 0, slot, col].clone()
        data.view(torch.uint8)[page, 0, slot, col] = 0xff
        y = torch.empty_like(q)
        B.cache_attention(p.cache(), q, y, int32([0, 40]), int32([80]), 1 / math.sqrt(d)).run()
        nan = torch.isnan(y)
        assert not nan[:21].any() and torch.equal(y[:21], clean[:21])
        if data is p.k:
            assert nan[21:].all()
        else:
            assert nan[21:, :, 5].all() and nan.sum() == 19 * 2
            assert torch.allclose(y[21:, :, 6:].float(), clean[21:, :, 6:].float(), atol=0, rtol=0)
        data.view(torch.uint8)[page, 0, slot, col] = keep


@gpu
def test_attention_offsets_beyond_32_bits():
    heads, d, block = 1, 64, 16
    pages = (1 << 32) // (block * d * 4) + 40                     # pages four times as far apart as they are large
    whole = torch.empty(pages * block * d * 4, dtype=torch.uint8, device="cuda")
    p = Pages([40, 1], heads, d, block, seed=9)
    for name in ("k", "v"):
        far = torch.as_strided(whole, (pages, heads, block, d), (block * d * 4, block * d, d, 1), block * d * (0 if name == "k" else 1))
        near = getattr(p, name).view(torch.uint8)
        far[-near.shape[0]:] = near
        setattr(p, name, far.view(E4M3))
        s = torch.zeros(pages, heads, device="cuda")
        s[-near.shape[0]:] = getattr(p, name + "s")
        setattr(p, name + "s", s)
    shift = pages - near.shape[0]
    p.table_cpu = [[i + shift for i in row] for row in p.table_cpu]
    for b, row in enumerate(p.table_cpu):
        p.table[b, :len(row)] = int32(row)
    check_attention(p, [3, 1], 2)
    x = torch.randn(4, heads, d, generator=gen(1), device="cuda")
    starts = int32([0, 3, 4])
    B.cache_append(p.cache(), x, x, starts, int32(p.lengths)).run()
    check_attention(p, [3, 1], 2)


@gpu
def test_attention_reports_what_only_the_device_sees():
    for table, lengths, starts in (([[0, 1 << 30]], [20], [0, 2]), ([[-1, 1]], [10], [0, 2]), ([[0, 1]], [33], [0, 2]), ([[0, 1]], [-1], [0, 2]), ([[0, 1]], [20], [0, 3]), ([[0, 1]], [20], [2, 1])):
        p = Pages([32], 1, 32, 16, seed=1)
        p.table = int32(table)
        q = torch.randn(2, 1, 32, generator=gen(1), device="cuda").to(torch.float16)
        call = B.cache_attention(p.cache(), q, torch.empty_like(q), int32(starts), int32(lengths), 0.1)
        call.run()
        assert call.status() == B.TT_ERR_INVALID_ARG, (table, lengths, starts)
    for bound in (dict(max_length=16), dict(max_count=1)):
        call = B.cache_attention(p.cache(), q, torch.empty_like(q), int32([0, 2]), int32([20]), 0.1, **bound)
        call.run()
        assert call.status() == B.TT_ERR_INVALID_ARG, bound


@gpu
@pytest.mark.parametrize("heads_q,max_count", [(8, 0), (8, 2), (64, 0)])
def test_attention_reports_starts_that_do_not_rise_from_0(heads_q, max_count):
    p = Pages([80, 80], 1, 64, 16, seed=1)
    q = torch.randn(200, heads_q, 64, generator=gen(1), device="cuda").to(torch.float16)
    for starts in ([100, 102, 104], [100, 90, 104], [-40, -20, 0]):
        y = torch.full_like(q, 7.0)
        call = B.cache_attention(p.cache(), q, y, int32(starts), int32(p.lengths), 0.1, max_count=max_count)
        call.run()
        if max_count == 0 or starts[0] < 0 or starts[1] < starts[0]:
            assert call.status() == B.TT_ERR_INVALID_ARG, starts
        assert (y[:max(0, min(starts))] == 7.0).all()          # (a sequence whose own starts rise has its rows)


@gpu
def test_one_workspace_serves_calls_of_all_sizes():
    # (batch, heads, query heads, new tokens, length): most of them split, by either kernel, each over what the ones before have left
    sizes = [(1, 8, 8, 1, 5000), (8, 8, 8, 1, 2500), (32, 2, 8, 1, 1100), (1, 1, 4, 70, 6000), (3, 1, 8, 2, 4000), (1, 8, 8, 1, 5000), (2, 1, 2, 40, 5000), (9, 8, 8, 1, 2600)]
    workspace = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
    for i, (batch, heads, heads_q, count, length) in enumerate(sizes):
        p = Pages([length - 7 * b for b in range(batch)], heads, 64, 64, seed=i)
        counts = [count] * batch
        q = (torch.randn(batch * count, heads_q, 64, generator=gen(i), device="cuda") * 2).to(torch.float16)
        y = torch.full_like(q, -77.0)
        call = B.cache_attention(p.cache(), q, y, int32([count * b for b in range(batch + 1)]), int32(p.lengths), 0.125, max_count=count)
        assert call.args.workspace_bytes <= workspace.numel()
        call.args.workspace, call.args.workspace_bytes = workspace.data_ptr(), workspace.numel()
        for _ in range(2):
            call.run()
            assert call.status() == B.TT_OK
            ref, off = reference_attention(p, counts, q, 0.125, True, 0)
            assert (np.abs(y.double().cpu().numpy() - ref) <= off + HALF_STEP[torch.float16] * (np.abs(ref) + off) + 2.0 ** -25).all(), i
            y.fill_(-77.0)


@gpu
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("length,count,heads_q,window", [(300, 1, 4, 20), (300, 3, 4, 37), (745, 5, 2, 301), (5000, 2, 8, 2100), (1500, 40, 2, 1000), (6000, 40, 2, 4000), (400, 40, 2, 30)])
def test_attention_needs_no_page_in_front_of_the_window(block, length, count, heads_q, window):
    given_back = (length - count + 1 - window) // block            # pages that no query sees
    for entry in (-1, None):
        p = Pages([length], 1, 64, block, seed=window)
        p.ks[p.free[:1]], p.vs[p.free[:1]] = math.nan, math.nan
        p.ks[p.free[1:2]], p.vs[p.free[1:2]] = math.inf, math.inf
        for j in range(given_back):                                # none, or one of another's with scales of anything
            p.table[0, j] = entry if entry is not None else p.free[j % 2]
        check_attention(p, [count], heads_q, window=window)


@gpu
@pytest.mark.parametrize("heads_q", [1, 8])
def test_attention_with_a_window_as_long_as_a_number_can_be(heads_q):
    for lengths, counts in (([3, 50], [8, 20]), ([100], [120])):      # (queries in front of the tokens see none)
        p = Pages(lengths, 1, 64, 16, seed=2)
        y = check_attention(p, counts, heads_q, window=(1 << 31) - 1)
        assert torch.equal(y, check_attention(p, counts, heads_q))
        check_attention(p, counts, heads_q, window=max(lengths))      # (another form may take it: the same within the roundings)


def check_scales_apart(p, count, heads_q, window=0):
    """check_attention for one sequence whose pages' scales of values differ by more than the bits of a number."""
    length, d = p.lengths[0], p.d
    q = (torch.randn(count, heads_q, d, generator=gen(50), device="cuda") * 2).to(torch.bfloat16)
    y = torch.full_like(q, -77.0)
    call = B.cache_attention(p.cache(), q, y, int32([0, count]), int32([length]), 1 / math.sqrt(d), window=window)
    call.run()
    assert call.status() == B.TT_OK
    ref, off = reference_attention(p, [count], q, 1 / math.sqrt(d), True, window)
    # A probability times its page's scale is a 16-bit number in units of 2^-7 (of 2^-15) of the largest probability times the largest scale that the row
    # sees, or times one up to 2^5 larger.  Normal ones are in `off`; those below 2^-14 are off by half a step of 2^-24, so each key by 2^-27 of that,
    # times its byte, 448 at most.
    scales = p.vs[p.table_cpu[0]].amax(dim=1).repeat_interleave(p.block).cpu().double().numpy()
    for i in range(count):
        pos = length - count + i
        lo = max(0, pos + 1 - window) if window else 0
        off[i] += 2.0 ** -27 * 448 * (pos + 1 - lo) * scales[lo:pos + 1].max()
    got = y.double().cpu().numpy()
    bad = np.abs(got - ref) > off + 2.0 ** -8 * (np.abs(ref) + off) + 2.0 ** -125
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("count,heads_q", [(20, 1), (10, 3), (90, 1), (60, 6)])
def test_attention_of_queries_that_see_only_pages_of_small_scales(d, block, count, heads_q):
    # pages that one query of a tile sees are 2^24 and 2^48 times as large as those of another
    for exponents in ([-48, -24, 0, 24], [0, -48, -24, 0], [24, 0, -24, -48]):
        p = Pages([4 * block - 3], 1, d, block, seed=d)
        for j, e in enumerate(exponents):
            p.vs[p.table_cpu[0][j]] = 2.0 ** (e - 8)
        for first in (0, block):                                      # rows whose last token is in the first page, in the second
            n = min(count, 3 * block - 3)
            p.lengths = [first + n]
            check_scales_apart(p, n, heads_q)
            check_scales_apart(p, n, heads_q, window=3)


@gpu
@pytest.mark.parametrize("count,heads_q", [(7, 2), (200, 2)])
def test_attention_behind_a_window_of_large_scales(count, heads_q):
    # what the first queries see and the last ones do not is 2^30 times as large
    length, window = 3000, 700
    p = Pages([length], 1, 64, 16, seed=count)
    lo, edge = length - count + 1 - window, length - window
    for j, page in enumerate(p.table_cpu[0]):
        p.vs[page] = 2.0 ** (22 if 16 * j <= max(lo, edge - 24) else -8)
    check_scales_apart(p, count, heads_q, window=window)


@gpu
@pytest.mark.parametrize("exponent", [-126, -100, -60, 0, 60, 100])
@pytest.mark.parametrize("count,heads_q", [(1, 4), (20, 1), (100, 1)])
def test_attention_of_values_of_any_size(exponent, count, heads_q):
    p = Pages([300], 1, 64, 16, seed=4)
    p.vs.fill_(2.0 ** -7)
    q = (torch.randn(count, heads_q, 64, generator=gen(1), device="cuda") * 2).to(torch.bfloat16)
    want = check_attention(p, [count], heads_q, q=q).clone()
    p.vs.fill_(2.0 ** exponent)
    y = torch.empty_like(q)
    B.cache_attention(p.cache(), q, y, int32([0, count]), int32([300]), 0.125).run()
    want = want.double() * 2.0 ** (exponent + 7)
    # the same bits but for another power of two, unless a result is no normal number of the type
    normal = want.abs() >= 2.0 ** -126
    assert torch.equal(y.double()[normal], want[normal]) and (y.double() - want).abs()[~normal].le(2.0 ** -133).all()


@gpu
@pytest.mark.parametrize("which,scale", [("ks", math.nan), ("vs", math.nan), ("vs", math.inf)])
@pytest.mark.parametrize("count,heads_q,d", [(4, 2, 64), (20, 1, 256), (100, 2, 64), (100, 1, 128)])
@pytest.mark.parametrize("at", [0, 20, -1])                          # the page: the first, one in the middle, the last
def test_attention_nan_scales_reach_the_rows_that_see_their_page(which, scale, count, heads_q, d, at):
    p = Pages([450], 1, d, 16, seed=8)
    q = torch.randn(count, heads_q, d, generator=gen(1), device="cuda").to(torch.float16)
    for window in (0, 390):
        clean = check_attention(p, [count], heads_q, q=q, window=window).clone()
        page = p.table_cpu[0][at]
        keep = getattr(p, which)[page].clone()
        getattr(p, which)[page] = scale
        y = torch.empty_like(q)
        B.cache_attention(p.cache(), q, y, int32([0, count]), int32([450]), 1 / math.sqrt(d), window=window).run()
        j = at % len(p.table_cpu[0])
        pos = torch.arange(450 - count, 450, device="cuda")
        sees = (16 * j <= pos) & ((16 * j + 16 > pos + 1 - window) if window else True)
        assert torch.isnan(y[sees]).all()
        assert torch.equal(y[~sees], clean[~sees])
        getattr(p, which)[page] = keep


@gpu
@pytest.mark.parametrize("m,n,k", [(5, 300, 1300), (40, 700, 300), (200, 300, 900), (300, 1000, 260), (3000, 2000, 300)])
@pytest.mark.parametrize("xe,we", [(-126, -17), (-17, -126), (-149, 10), (-126, 0), (-126, 120), (100, 1)])
def test_dense_scales_of_the_smallest_and_largest_products(m, n, k, xe, we):
    x, _, w, _ = dense_case(m, n, k, 9)
    kb, nb = -(-k // 128), -(-n // 128)
    xs = ((1 + torch.rand(kb, m, generator=gen(3), device="cuda").double()) * 2.0 ** xe).float()
    ws = ((1 + torch.rand(nb, kb, generator=gen(4), device="cuda").double()) * 2.0 ** we).float()
    y = torch.empty(m, n, device="cuda")
    call = B.dense_quantized(x, xs, w, ws, y)
    call.run()
    assert call.status() == B.TT_OK
    ref, most = dense_reference(x, xs, w, ws, None)
    # the products, the two scales and the additions in 32 bits; a product of scales below 2^-126 is off by 2^-150 at most, and a block's sum is 2^25 at most
    off = most * ADD * (128 + 3 * (kb + 1)) + (kb * 2.0 ** -125 if xe + we < -126 else 0)
    assert (np.abs(y.double().cpu().numpy() - ref) <= off).all()


@gpu
def test_words_of_a_call_stay_until_its_runs_on_other_streams_are_done():
    p = Pages([6000], 1, 64, 64, seed=1)
    q = torch.randn(1, 4, 64, generator=gen(1), device="cuda").to(torch.float16)
    y, starts, lengths = torch.empty_like(q), int32([0, 1]), int32([6000])
    want = check_attention(p, [1], 4, q=q, scale=0.1)
    call = B.cache_attention(p.cache(), q, y, starts, lengths, 0.1)
    held, n = call.args.workspace, call.args.workspace_bytes
    word = call.args.status
    assert n > 0
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1 << 28)
        call.run()
        done = torch.cuda.Event()
        done.record()
    del call
    while_it_runs = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(4)] + [torch.empty(4, dtype=torch.uint8, device="cuda") for _ in range(64)]
    assert not done.query()                                           # (the run is still to come)
    assert held not in [t.data_ptr() for t in while_it_runs] and word not in [t.data_ptr() for t in while_it_runs]
    side.synchronize()
    assert torch.equal(y, want)


@gpu
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("count,heads_q,d,length,window", [
    (12, 2, 64, 80, 0), (30, 1, 128, 200, 0), (14, 2, 160, 100, 0), (9, 3, 256, 90, 0), (40, 2, 256, 90, 0),                    # few rows of a tile, long heads
    (12, 2, 64, 200, 50), (30, 1, 128, 200, 70), (9, 3, 256, 300, 33), (60, 2, 32, 200, 40),                                    # ... behind a window
    (4, 2, 64, 5000, 0), (4, 2, 64, 5000, 3000), (90, 2, 64, 900, 600), (90, 2, 96, 900, 600), (100, 1, 128, 1200, 700),        # splits; prompts behind a window
    (70, 2, 64, 6000, 0), (70, 2, 128, 6000, 0), (70, 2, 64, 6000, 3000), (33, 1, 32, 4000, 2500)])                             # prompts in splits
def test_attention_nan_reaches_the_rows_that_see_it_in_every_form(which, count, heads_q, d, length, window):
    p = Pages([length], 1, d, 16, seed=8)
    data, col = (p.k, 3) if which == "k" else (p.v, d - 5)
    q = torch.randn(count, heads_q, d, generator=gen(1), device="cuda").to(torch.float16)
    clean = check_attention(p, [count], heads_q, q=q, window=window).clone()
    pos = torch.arange(length - count, length, device="cuda")
    # seen from the middle of the queries on, by the last alone, by all; behind a window by the first, by the first ones; by none
    places = [length - count // 2, length - 1, (length - count) // 2] + ([length - count + 1 - window, length - window - count // 2, length - count - window] if window else [])
    for at in places:
        page, slot = p.table_cpu[0][at // 16], at % 16
        keep = data.view(torch.uint8)[page, 0, slot, col].clone()
        data.view(torch.uint8)[page, 0, slot, col] = 0xff
        y = torch.full_like(q, -77.0)
        call = B.cache_attention(p.cache(), q, y, int32([0, count]), int32([length]), 1 / math.sqrt(d), window=window)
        call.run()
        assert call.status() == B.TT_OK
        sees = (at <= pos) & ((at > pos - window) if window else True)
        nan = torch.isnan(y)
        want = torch.zeros_like(nan)
        if which == "k":
            want[sees] = True
        else:
            want[sees, :, col] = True
        assert torch.equal(nan, want), at
        assert torch.equal(y[~want], clean[~want]), at
        data.view(torch.uint8)[page, 0, slot, col] = keep


@gpu
def test_dense_beside_a_layer_that_takes_all_tensor_memory():
    # Clusters of two kernels on two streams, of which an SM has room for a CTA of each but not for their tensor memory: neither waits for a peer that waits
    # for what it holds.
    from paper_2201_05587_b200 import workloads as W
    spec = W._dense(512, 256, 512, act=B.TT_ACT_NONE, name="beside")
    wl = spec.workload()
    info = wl.apply(B.make_record(B.TT_FAMILY_GEMM_TC, tile_n=64, tile_k=32, stages=2, split_k=4, mma_m_axis=1, acc_split=8))
    assert info.tmem_cols == 512 and info.legal.split_k == 4
    t, tensors = W.device_tensors(spec, W.make_inputs(spec, 1))
    x, xs, w, ws = dense_case(8, 4096, 4096)
    y = torch.empty(8, 4096, device="cuda")
    call = B.dense_quantized(x, xs, w, ws, y)
    call.run()
    wl.run(tensors)
    torch.cuda.synchronize()
    want = y.clone(), t["y"].clone()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        y.zero_()
        t["y"].zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            with torch.cuda.stream(streams[0]):
                call.run()
            with torch.cuda.stream(streams[1]):
                wl.run(tensors)
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(t["y"], want[1])
    assert call.status() == B.TT_OK and wl.status() == B.TT_OK
    wl.close()


# ---- GPU: together, as a program uses them ------------------------------------------------------------------------------
class Layer:
    """One attention block of a decoder whose weights and cache are in e4m3: quantise, project, turn, append, attend, quantise, project."""

    def __init__(self, tokens, width, hq, hk, d, p, starts, lengths, seed=0):
        self.hidden = torch.randn(tokens, width, generator=gen(seed), device="cuda").to(torch.bfloat16)
        out = (hq + 2 * hk) * d
        self.x, _ = f8_matrix(tokens, width)
        self.xs = torch.empty(-(-width // 128), tokens, device="cuda")
        self.packed = torch.empty(tokens, out, dtype=torch.bfloat16, device="cuda")
        heads = self.packed.view(tokens, hq + 2 * hk, d)
        self.q, self.k, self.v = heads[:, :hq], heads[:, hq:hq + hk], heads[:, hq + hk:]
        self.o = torch.empty(tokens, hq, d, dtype=torch.bfloat16, device="cuda")
        self.o8, _ = f8_matrix(tokens, hq * d)
        self.os = torch.empty(-(-hq * d // 128), tokens, device="cuda")
        self.y = torch.empty(tokens, width, dtype=torch.bfloat16, device="cuda")
        self.positions = torch.zeros(tokens, dtype=torch.int32, device="cuda")
        self.weights = []
        for i, (n, k) in enumerate(((out, width), (width, hq * d))):
            w = torch.randn(n, k, generator=gen(70 + i), device="cuda") / math.sqrt(k)
            q, _ = f8_matrix(n, k)
            s = torch.empty(-(-n // 128), -(-k // 128), device="cuda")
            B.quantize(w, q, s.t(), block_rows=128).run()
            self.weights.append((q, s))
        self.scale, cache = 1 / math.sqrt(d), p.cache()
        self.calls = [B.quantize(self.hidden, self.x, self.xs), B.dense_quantized(self.x, self.xs, *self.weights[0], self.packed),
                      B.rotary([self.q, self.k], self.positions, B.rotary_table(B.rotary_frequencies(d))),
                      B.cache_append(cache, self.k, self.v, starts, lengths), B.cache_attention(cache, self.q, self.o, starts, lengths, self.scale),
                      B.quantize(self.o.view(tokens, hq * d), self.o8, self.os), B.dense_quantized(self.o8, self.os, *self.weights[1], self.y)]

    def run(self):
        for c in self.calls:
            c.run()


@gpu
def test_a_decoder_step_over_the_cache():
    width, hq, hk, d, block = 256, 4, 2, 64, 16
    p = Pages([90, 40], hk, d, block, seed=11, random_values=False)
    # two prompts, then single tokens, a step at a time; the steps' arguments live on the device
    prompt = Layer(20 + 33, width, hq, hk, d, p, int32([0, 20, 53]), int32([20, 33]), seed=1)
    prompt.positions.copy_(int32(list(range(20)) + list(range(33))))
    prompt.run()
    p.lengths = [20, 33]
    ref, off = reference_attention(p, [20, 33], prompt.q, prompt.scale, True, 0)
    assert (np.abs(prompt.o.double().cpu().numpy() - ref) <= off + 2.0 ** -8 * (np.abs(ref) + off) + 2.0 ** -25).all()
    lengths = int32([21, 34])
    step = Layer(2, width, hq, hk, d, p, int32([0, 1, 2]), lengths, seed=2)
    for i in range(6):
        step.hidden.copy_(torch.randn(2, width, generator=gen(100 + i), device="cuda"))
        p.lengths = [21 + i, 34 + i]
        lengths.copy_(int32(p.lengths))
        step.positions.copy_(lengths - 1)
        step.run()
        ref, off = reference_attention(p, [1, 1], step.q, step.scale, True, 0)
        assert (np.abs(step.o.double().cpu().numpy() - ref) <= off + 2.0 ** -8 * (np.abs(ref) + off) + 2.0 ** -25).all()
    assert all(c.status() == B.TT_OK for c in prompt.calls + step.calls)
    # the projections, from the operands that the calls have left
    for x, xs, w, y in ((step.x, step.xs, step.weights[0], None), (step.o8, step.os, step.weights[1], step.y)):
        ref, most = dense_reference(x, xs, *w, None)
        if y is not None:
            assert (np.abs(y.double().cpu().numpy() - ref) <= most * ADD * 160 + 2.0 ** -8 * np.abs(ref)).all()


@gpu
def test_a_captured_step_gives_the_bits_of_an_eager_one():
    def fresh():
        p = Pages([3000, 40], 2, 64, 16, seed=12)
        return p, Layer(2, 256, 4, 2, 64, p, int32([0, 1, 2]), int32([3000, 40]), seed=3)
    p, eager = fresh()
    eager.run()
    torch.cuda.synchronize()
    p2, layer = fresh()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                                # another stream than the one that made the calls
        layer.run()
    side.synchronize()
    assert torch.equal(eager.y, layer.y)
    p3, layer = fresh()
    graph = torch.cuda.CUDAGraph()
    layer.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        layer.run()
    layer.y.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(eager.y, layer.y)
    for a, b in ((p.k, p3.k), (p.v, p3.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    cache, starts, lengths = p3.cache(), int32([0, 1, 2]), int32([3000, 40])
    with pytest.raises(B.TTError):                               # device words are made before a capture
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            B.cache_append(cache, layer.k, layer.v, starts, lengths)
