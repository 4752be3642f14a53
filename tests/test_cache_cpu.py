"""Rotary frequencies against formulas written out, and what the entry points of the growing cache refuse, without a GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2504_00970_amd as skv
from paper_2504_00970_amd import binding


def close(got, want):
    assert len(got) == len(want)
    for g, w in zip(got, want):
        assert abs(g - w) <= 2.0 ** -46 * abs(w), (g, w)       # a few roundings of 2^-53; a power amplifies its exponent's by ln base < 20


@pytest.mark.parametrize("rot", [2, 6, 64, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies_follow_their_formulas(rot, base):
    n = rot // 2
    plain = [base ** (-2.0 * i / rot) for i in range(n)]
    f, m = skv.rotary_freqs(rot, base)
    close(f.tolist(), plain)
    assert m == 1.0 and f.dtype == torch.float64
    f, m = skv.rotary_freqs(rot, base, skv.SKV_ROPE_LINEAR, 4.0)
    close(f.tolist(), [x / 4.0 for x in plain])
    assert m == 1.0
    if rot >= 4:
        f, m = skv.rotary_freqs(rot, base, skv.SKV_ROPE_NTK, 8.0)
        close(f.tolist(), [(base * 8.0 ** (rot / (rot - 2))) ** (-2.0 * i / rot) for i in range(n)])
        assert f[0] == 1.0 and abs(f[-1] * 8.0 / plain[-1] - 1) < 1e-12 and m == 1.0
    f, m = skv.rotary_freqs(rot, base, skv.SKV_ROPE_TURNS, 8.0, 1.0, 4.0, 8192.0)
    for x, p in zip(f.tolist(), plain):
        r = 8192.0 * p / (2 * math.pi)
        g = min(1.0, max(0.0, (r - 1.0) / 3.0))
        # the blend's weight carries the rounding of r, up to 2^-40 of itself beside 1
        assert abs(x - ((1 - g) * p / 8.0 + g * p)) <= 2.0 ** -36 * p
    assert m == 1.0
    f, m = skv.rotary_freqs(rot, base, skv.SKV_ROPE_YARN, 16.0, 1.0, 32.0, 4096.0)
    where = lambda r: rot * math.log(4096.0 / (2 * math.pi * r)) / (2 * math.log(base))      # noqa: E731
    a, z = max(math.floor(where(32.0)), 0), min(math.ceil(where(1.0)), rot - 1)
    for i, (x, p) in enumerate(zip(f.tolist(), plain)):
        u = min(1.0, max(0.0, (i - a) / (z - a))) if z > a else float(i > a)
        assert abs(x - (p / 16.0 * u + p * (1 - u))) <= 2.0 ** -40 * p
    assert abs(m - (0.1 * math.log(16.0) + 1.0)) <= 2.0 ** -23


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=3), dict(rot=130), dict(rot=-2), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                                dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("inf")), dict(scaling=2, factor=2.0, rot=2),
                                dict(scaling=3, factor=2.0), dict(scaling=3, factor=2.0, low=4.0, high=1.0, original=8.0), dict(scaling=4, factor=2.0, low=0.0, original=8.0),
                                dict(scaling=4, factor=float("nan"), original=8.0), dict(scaling=4, factor=2.0, original=float("inf"))])
def test_frequencies_refuse(kw):
    a = dict(rot=64, base=10000.0, scaling=skv.SKV_ROPE_PLAIN)
    a.update(kw)
    with pytest.raises(skv.SkvError) as e:
        skv.rotary_freqs(**a)
    assert e.value.status == skv.SKV_EINVAL
    assert binding._lib().skv_rotary_freqs(64, 10000.0, 0, 1.0, 1.0, 32.0, 0.0, None, None) == skv.SKV_EINVAL


def test_reference_codes_round_to_the_nearest_value():
    v = R.e4m3_value(np.arange(0x7f))
    assert np.array_equal(R.e4m3_code(v), np.arange(0x7f)) and np.array_equal(R.e4m3_code(-v[1:]), np.arange(1, 0x7f) | 0x80)
    x = np.random.RandomState(0).standard_normal(20000) * np.exp2(np.random.RandomState(1).randint(-12, 8, 20000))
    x = np.clip(x, -448, 448).astype(np.float32)
    x = np.concatenate([x, (v[1:] + v[:-1]).astype(np.float32) / 2])                                     # ties too
    assert np.array_equal(R.e4m3_code(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


# ---- refusals: a context that holds nothing but its descriptor (a context begins with it), so that a call that passes its checks ends where it asks for the device --------------

DESC = dict(n_layers=2, n_q_heads=8, n_kv_heads=4, head_dim=128, kv_dtype=skv.SKV_BF16, max_tokens=1000, max_sentences=8, max_budget=16, max_batch=3,
            semvec_dtype=skv.SKV_F32)


class _Fake(ctypes.Structure):
    _fields_ = [("d", binding._Desc), ("stream", ctypes.c_void_p), ("device", ctypes.c_int), ("n_cu", ctypes.c_int), ("G", ctypes.c_int), ("rest", ctypes.c_char * 4096)]


BUF = (ctypes.c_char * 64)()
P = (ctypes.addressof(BUF) + 15) // 16 * 16             # an aligned address that nothing reads
OTHER = P + 16

GOOD = {
    "skv_rotary": dict(n=5, q=P, k=P, pos=P, inv_freq=P, rot=64, interleaved=0, mscale=1.0, q_out=P, k_out=P),
    "skv_cache_append": dict(layer=1, B=2, k=P, v=P, n_new=3, cu_new=P, max_new=3, cu_tok=P, n_tok=P, K=P, V=P, k_scale=P, v_scale=P, T_total=100, block=32, acc=P),
    "skv_cache_attend": dict(layer=1, B=2, q=P, K=P, V=P, k_scale=P, v_scale=P, T_total=100, block=32, cu_tok=P, n_tok=P, tok_idx=None, max_n=50, out=P, lse=P, acc=P,
                             acc_out=P, decay=0.5, work=P, work_bytes=1 << 30),
    "skv_cache_evict": dict(B=2, acc=P, T_total=100, cu_tok=P, n_tok=P, max_n=50, keep=20, sink=4, recent=5, keep_idx=P, n_keep=OTHER),
    "skv_cache_compact": dict(B=2, K=P, V=P, k_scale=P, v_scale=P, acc=P, T_total=100, block=32, cu_tok=P, keep_idx=P, keep=20, n_keep=P, K_out=P, V_out=P, k_scale_out=P,
                              v_scale_out=P, acc_out=P),
}
INVALID, CAPACITY, PASSES = skv.SKV_EINVAL, skv.SKV_ECAPACITY, None
NAN = float("nan")
CASES = [(name, {}, PASSES) for name in GOOD]
for _name, _good in GOOD.items():
    for _arg in _good:
        if _good[_arg] in (P, OTHER):
            optional = (_name, _arg) in (("skv_cache_append", "acc"), ("skv_cache_attend", "lse"), ("skv_cache_attend", "acc"))
            CASES.append((_name, {_arg: None}, PASSES if optional else INVALID))
            if _arg not in ("n_tok", "k_scale", "v_scale", "acc", "k_scale_out", "v_scale_out", "acc_out"):
                CASES.append((_name, {_arg: P + 8}, INVALID))
            else:
                together = {x: P + 4 for x in (_arg, _arg.removesuffix("_out"), _arg + "_out") if x in _good and _name == "skv_cache_compact"} or {_arg: P + 4}
                CASES += [(_name, together, PASSES), (_name, {_arg: P + 2}, INVALID)]
CASES += [("skv_rotary", kw, want) for kw, want in [
    (dict(n=-1), INVALID), (dict(n=1001), CAPACITY), (dict(rot=0), INVALID), (dict(rot=63), INVALID), (dict(rot=130), INVALID), (dict(interleaved=2), INVALID),
    (dict(mscale=NAN), INVALID), (dict(mscale=math.inf), INVALID), (dict(q=None, q_out=None), PASSES), (dict(k=None, k_out=None), PASSES),
    (dict(q=None, q_out=None, k=None, k_out=None), INVALID), (dict(rot=2), PASSES), (dict(rot=128), PASSES)]]
CASES += [("skv_cache_append", kw, want) for kw, want in [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(B=0), INVALID), (dict(B=4), CAPACITY), (dict(n_new=-1), INVALID), (dict(n_new=1001), CAPACITY),
    (dict(max_new=-1), INVALID), (dict(T_total=0), INVALID), (dict(T_total=1001), CAPACITY), (dict(block=8), INVALID), (dict(block=48), INVALID), (dict(block=256), INVALID),
    (dict(block=0), INVALID), (dict(n_new=0, k=None, v=None), PASSES)]]
CASES += [("skv_cache_attend", kw, want) for kw, want in [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(B=0), INVALID), (dict(B=4), CAPACITY), (dict(max_n=-1), INVALID), (dict(max_n=1001), CAPACITY),
    (dict(T_total=0), INVALID), (dict(T_total=1001), CAPACITY), (dict(block=17), INVALID), (dict(decay=-0.1), INVALID), (dict(decay=1.1), INVALID), (dict(decay=NAN), INVALID),
    (dict(tok_idx=P), INVALID), (dict(tok_idx=P, acc=None, acc_out=None), PASSES), (dict(tok_idx=P + 4, acc=None, acc_out=None), INVALID), (dict(acc=None, acc_out=None), PASSES),
    (dict(work_bytes=100), INVALID), (dict(work_bytes=-1), INVALID)]]
CASES += [("skv_cache_evict", kw, want) for kw, want in [
    (dict(B=0), INVALID), (dict(B=4), CAPACITY), (dict(T_total=0), INVALID), (dict(T_total=1001), CAPACITY), (dict(max_n=-1), INVALID), (dict(max_n=1001), CAPACITY),
    (dict(keep=-1, sink=0, recent=0), INVALID), (dict(sink=-1), INVALID), (dict(recent=-1), INVALID), (dict(sink=10, recent=11), INVALID), (dict(sink=10, recent=10), PASSES),
    (dict(n_keep=P), INVALID), (dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1, keep=2 ** 31 - 1), INVALID)]]
CASES += [("skv_cache_compact", kw, want) for kw, want in [
    (dict(B=0), INVALID), (dict(B=4), CAPACITY), (dict(T_total=0), INVALID), (dict(T_total=1001), CAPACITY), (dict(block=31), INVALID), (dict(keep=-1), INVALID),
    (dict(acc=None, acc_out=None), PASSES), (dict(K_out=OTHER), INVALID), (dict(acc_out=OTHER), INVALID),
    (dict(K_out=OTHER, V_out=OTHER, k_scale_out=OTHER, v_scale_out=OTHER), INVALID),
    (dict(K_out=OTHER, V_out=OTHER, k_scale_out=OTHER, v_scale_out=OTHER, acc_out=OTHER), PASSES)]]


def _call(name, ctx, kw):
    args = dict(GOOD[name])
    args.update(kw)
    return getattr(binding._lib(), name)(ctx, *args.values())


def _fake():
    f = _Fake()
    f.d, f.device, f.n_cu, f.G = binding._Desc(*DESC.values()), 0, 256, 2
    return f


@pytest.mark.parametrize("name,kw,want", CASES)
def test_refusals(name, kw, want):
    if want is PASSES and torch.cuda.is_available():
        pytest.skip("a call that passes its checks is for a machine without a GPU")
    f = _fake()
    assert _call(name, ctypes.addressof(f), kw) == (skv.SKV_EHIP if want is PASSES else want)


def test_null_contexts_and_work_sizes():
    lib, f = binding._lib(), _fake()
    for name in GOOD:
        assert _call(name, None, {}) == skv.SKV_EINVAL
    size = lambda *a: lib.skv_cache_attend_work_bytes(ctypes.addressof(f), *a)      # noqa: E731
    assert lib.skv_cache_attend_work_bytes(None, 1, 1, 0) == -1
    for bad in ((0, 5, 0), (4, 5, 0), (1, -1, 0), (1, 1001, 0), (1, 5, 2)):
        assert size(*bad) == -1
    assert size(3, 1000, 0) > 0 and size(3, 1000, 1) >= size(3, 1000, 0) + 3 * 8 * 1000 * 4
    assert _call("skv_cache_attend", ctypes.addressof(f), dict(work_bytes=size(2, 50, 1) - 1)) == skv.SKV_EINVAL


@pytest.mark.parametrize("heads,group,dtype", [(1, 1, skv.SKV_BF16), (8, 4, skv.SKV_BF16), (8, 8, skv.SKV_F32), (15, 2, skv.SKV_F32)])
def test_work_for_a_large_call_does_for_smaller_ones(heads, group, dtype):
    """The bytes never fall as sequences, rows or weights are added, and the call takes a buffer of a larger one's size."""
    f = _fake()
    f.d.n_kv_heads, f.d.n_q_heads, f.d.kv_dtype, f.d.max_tokens, f.d.max_batch, f.G = heads, heads * group, dtype, 1 << 20, 4096, group
    size = lambda *a: binding._lib().skv_cache_attend_work_bytes(ctypes.addressof(f), *a)      # noqa: E731
    rows = sorted({max(0, int(x)) for p in range(21) for x in (2 ** p - 1, 2 ** p, 2 ** p + 1, 1.3 * 2 ** p)} | set(range(3500, 5500, 20)) | {(1 << 20)})
    rows = [n for n in rows if n <= 1 << 20]
    before = None
    for B in (1, 2, 3, 16, 17, 64, 128, 129, 512, 513, 1024, 1025, 4096):
        now = [[size(B, n, w) for n in rows] for w in (0, 1)]
        for by_rows in now:
            assert all(a <= b for a, b in zip(by_rows, by_rows[1:]))
        assert all(a <= b for a, b in zip(*now))
        assert before is None or all(a <= b for x, y in zip(before, now) for a, b in zip(x, y))
        before = now
    if not torch.cuda.is_available():                       # a call that passes its checks
        for n in (0, 1, 129, 4000, 4159):
            kw = dict(layer=0, B=1, T_total=5000, max_n=n, work_bytes=size(1, 4160, 1))
            assert _call("skv_cache_attend", ctypes.addressof(f), kw) == skv.SKV_EHIP
            assert _call("skv_cache_attend", ctypes.addressof(f), dict(kw, work_bytes=size(1, n, 1) - 1)) == skv.SKV_EINVAL


@pytest.mark.parametrize("through", ["native", "ctypes"])
@pytest.mark.parametrize("name", sorted(GOOD))
def test_python_calls_refuse_arguments_in_each_others_place(name, through):
    lib = binding._lib()
    call, kinds = getattr(binding._CALLS if through == "native" else binding._CtypesCalls(lib), name), binding._SIGNATURES[name][1]
    args = [None if k is ctypes.c_void_p else 1 for k in kinds]
    assert call(*args) == skv.SKV_EINVAL                   # the context is null
    for i, k in enumerate(kinds):
        bad = list(args)
        bad[i] = torch.zeros(1) if k is not ctypes.c_void_p or i == 0 else 4096
        with pytest.raises(TypeError):
            call(*bad)
        if k is ctypes.c_float:
            bad[i] = 0.25
            assert call(*bad) == skv.SKV_EINVAL
        elif k is ctypes.c_void_p and i:
            bad[i] = torch.zeros(4, 4).t()
            with pytest.raises(AssertionError):
                call(*bad)
    with pytest.raises(TypeError):
        call(*args[:-1])
