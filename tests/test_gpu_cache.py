"""Rotary positions and the growing 8-bit cache on the GPU, against the 64-bit definitions of cache_ref.  Codes, scales, lists and counts have to be equal; for
computed numbers the bound is derived where it is used."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2504_00970_amd as skv

pytestmark = pytest.mark.gpu

DEV, D = "cuda:0", 128
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 2.0 ** -24                                           # half a step of fp32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"


def context(L=1, H=2, G=2, dtype="bf16", tokens=1 << 20, batch=8):
    return skv.Context(skv.Desc(n_layers=L, n_q_heads=H * G, n_kv_heads=H, kv_dtype=skv.dtype_code(TYPES[dtype]), max_tokens=tokens, max_batch=batch))


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def f64(t):
    return t.detach().cpu().double().numpy()


# ---- rotary ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [2, 6, 16, 40, 64, 96, 126, 128])
@pytest.mark.parametrize("n,H,G,mscale", [(1, 1, 1, 1.0), (3, 2, 4, 1.25), (67, 5, 8, 0.75)])
def test_rotary(dtype, interleaved, rot, n, H, G, mscale):
    ctx = context(H=H, G=G, dtype=dtype)
    g = torch.Generator().manual_seed(rot * 131 + n)
    q, k = (torch.randn(n, h, D, generator=g).to(TYPES[dtype]) for h in (H * G, H))
    pos = torch.randint(-3, 1 << 20, (n,), generator=g, dtype=torch.int32)
    pos[0], pos[-1] = (0, -77) if n > 1 else ((1 << 31) - 1,) * 2
    freq, _ = skv.rotary_freqs(rot, 10000.0)
    qd, kd, pd, fd = q.to(DEV), k.to(DEV), pos.to(DEV), freq.to(DEV)
    qo, ko = torch.full_like(qd, 7.0), torch.full_like(kd, 7.0)
    ctx.rotary(n, qd, kd, pd, fd, rot, interleaved, mscale, qo, ko)
    for x, got in ((q, qo), (k, ko)):
        x, got = x.double().numpy(), f64(got)
        want = R.rotary(x, pos.numpy(), freq.numpy(), rot, interleaved, mscale)
        size = np.abs(x[..., :rot]).max(axis=-1, keepdims=True) * 2 * mscale
        # The angle: position times frequency is off by 2^-53 of up to 2^31, and so is its product by 1 / 2 pi: 2^-20 at the largest positions, 2^-31 at 2^20.  The
        # fraction of a turn in fp32: 2^-26 turns = 2^-23.3.  sin and cos: within 2 units of the last place, 2^-22; mscale, two products, one sum: 4 half steps.
        far = float(np.abs(pos.numpy().astype(np.int64)).max())
        bound = size * (2 * math.pi * far * 2.0 ** -51 + 2.0 ** -23.3 + 2.0 ** -22 + 4 * EPS)
        if dtype == "bf16":
            bound = bound + np.abs(want) * 2.0 ** -8
        assert np.all(np.abs(got - want)[..., :rot] <= np.broadcast_to(bound, want.shape)[..., :rot])
        assert np.array_equal(got[..., rot:], x[..., rot:])
    a, b = qd.clone(), kd.clone()
    ctx.rotary(n, a, b, pd, fd, rot, interleaved, mscale, a, b)                    # where they lie
    assert torch.equal(a, qo) and torch.equal(b, ko)
    a.fill_(5.0)
    b.fill_(5.0)
    ctx.rotary(n, qd, None, pd, fd, rot, interleaved, mscale, a, None)             # one of them
    ctx.rotary(n, None, kd, pd, fd, rot, interleaved, mscale, None, b)
    assert torch.equal(a, qo) and torch.equal(b, ko)


def test_rotary_back_and_its_transpose():
    ctx = context(H=2, G=2, dtype="f32")
    g = torch.Generator().manual_seed(4)
    x, y = (torch.randn(33, 4, D, generator=g).to(DEV) for _ in range(2))
    pos = torch.randint(0, 1 << 20, (33,), generator=g, dtype=torch.int32).to(DEV)
    freq = skv.rotary_freqs(128, 500000.0, skv.SKV_ROPE_YARN, 8.0, 1.0, 32.0, 8192.0)[0].to(DEV)
    fwd, back, grad = (torch.empty_like(x) for _ in range(3))
    ctx.rotary(33, x, None, pos, freq, 128, False, 1.0, fwd, None)
    ctx.rotary(33, fwd, None, -pos, freq, 128, False, 1.0, back, None)
    # two turns of pairs of size up to 2 max |x|, each within the bound of test_rotary at 2^20
    assert float((back - x).abs().max()) <= 2 * 2 * float(x.abs().max()) * (2.0 ** -23.3 + 2.0 ** -22 + 5 * EPS)
    ctx.rotary(33, x, None, pos, freq, 128, False, 1.5, fwd, None)
    ctx.rotary(33, y, None, -pos, freq, 128, False, 1.5, grad, None)
    a, b = float((fwd.double() * y.double()).sum()), float((x.double() * grad.double()).sum())         # <R x, y> = <x, R' y>
    assert abs(a - b) <= 2 * 1.5 * 2 * float((x.abs().double() * y.abs().double()).sum() + x.double().norm() * y.double().norm()) * (2.0 ** -23.3 + 2.0 ** -22 + 5 * EPS)


def test_rotary_of_many_tokens_takes_each_once():
    n, H = 5003, 3
    ctx = context(H=H, G=1)
    x = torch.randn(n, H, D, device=DEV).bfloat16()
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    freq = skv.rotary_freqs(64, 10000.0)[0].to(DEV)
    out = torch.zeros(n + 8, H, D, device=DEV, dtype=torch.bfloat16)
    ctx.rotary(n, x, None, pos, freq, 64, False, 1.0, out, None)
    one = torch.empty(1, H, D, device=DEV, dtype=torch.bfloat16)
    for t in (0, 1, 2500, n - 1):
        ctx.rotary(1, x[t:t + 1].clone(), None, pos[t:t + 1].clone(), freq, 64, False, 1.0, one, None)
        assert torch.equal(out[t], one[0])
    assert float(out[n:].abs().max()) == 0.0
    ctx.rotary(0, x, None, pos, freq, 64, False, 1.0, out, None)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [40, 64, 126, 128])
def test_rotary_sines_near_half_a_turn(interleaved, rot):
    """Angles next to odd multiples of pi, where the sine is small beside the angle: a fraction of a turn that was rounded to 32 bits would lose up to 9e-8 of it.  Rows of (1, 0) show
    cosine and sine themselves.  Sines and cosines are within 2 units of the last place (4 half steps), the rest of the angle is added with one rounding; the 64-bit angle is
    off by less than 2^-50 of 7 pi, below 2^-24 of the smallest sine."""
    half = rot // 2
    freq = math.pi * (1.0 + np.exp2(-np.linspace(4.0, 18.0, half)) * np.where(np.arange(half) % 2, -1.0, 1.0))
    pos = np.array([1, -1, 3, 7, -5], np.int32)
    x = torch.zeros(5, 2, D)
    a = np.arange(half) * 2 if interleaved else np.arange(half)
    b = a + (1 if interleaved else half)
    x[:, :, a] = 1.0
    ctx, out = context(H=1, G=2, dtype="f32"), torch.zeros(5, 2, D, device=DEV)
    ctx.rotary(5, x.to(DEV), None, i32(pos), torch.from_numpy(freq).to(DEV), rot, interleaved, 1.0, out, None)
    angle = pos[:, None].astype(np.float64) * freq[None]
    for at, want in ((a, np.cos(angle)), (b, np.sin(angle))):
        got = f64(out)[:, :, at]
        assert np.all(np.abs(got - want[:, None]) <= 6 * EPS * np.abs(want[:, None])), (np.abs(got / want[:, None] - 1)).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [126, 128])
@pytest.mark.parametrize("n", [4099, 8209])
def test_rotary_of_prompts_whose_waves_take_several_groups_of_heads(n, rot, interleaved, dtype):
    """45 heads: two waves a token take 24 and 21 of them, or one takes all, in groups of 4 or 8 with the next group on its way."""
    H, G = 5, 8
    ctx = context(H=H, G=G, dtype=dtype)
    g = torch.Generator(device=DEV).manual_seed(rot + n)
    q, k = (torch.randn(n, h, D, device=DEV, generator=g).to(TYPES[dtype]) for h in (H * G, H))
    pos = torch.randint(0, 1 << 20, (n,), device=DEV, generator=g, dtype=torch.int32)
    freq = skv.rotary_freqs(rot, 500000.0)[0].to(DEV)
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    ctx.rotary(n, q, k, pos, freq, rot, interleaved, 1.25, qo, ko)
    angle = pos.double()[:, None] * freq
    c, s = 1.25 * torch.cos(angle)[:, None], 1.25 * torch.sin(angle)[:, None]
    at = torch.arange(rot // 2, device=DEV)
    a, b = (2 * at, 2 * at + 1) if interleaved else (at, at + rot // 2)
    for x, got in ((q, qo), (k, ko)):
        x = x.double()
        want = x.clone()
        want[..., a], want[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        # the bound of test_rotary at 2^20
        bound = x[..., :rot].abs().amax(-1, keepdim=True) * 2 * 1.25 * (2 * math.pi * 2.0 ** -31 + 2.0 ** -23.3 + 2.0 ** -22 + 4 * EPS) + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0.0)
        assert bool(((got.double() - want).abs() <= bound)[..., :rot].all()) and torch.equal(got[..., rot:].double(), x[..., rot:])
    ctx.rotary(n, q, k, pos, freq, rot, interleaved, 1.25, q, k)                   # where they lie
    assert torch.equal(q, qo) and torch.equal(k, ko)


@pytest.mark.parametrize("rot", [126, 128])
def test_rotary_of_more_tokens_than_a_grid_has_waves(rot):
    """2^22 blocks of four waves are a token each; behind them waves take a second one, with the angles of its own position."""
    n = (1 << 24) + 4099
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    ctx = skv.Context(skv.Desc(n_layers=1, n_q_heads=1, n_kv_heads=1, kv_dtype=skv.SKV_BF16, max_tokens=n, max_sentences=1, max_budget=1, max_batch=1))
    x = torch.empty(n, 1, D, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(rot))
    pos, freq = torch.arange(n, dtype=torch.int32, device=DEV) % 100003, skv.rotary_freqs(rot, 10000.0)[0].to(DEV)
    out = torch.full_like(x, 7.0)
    ctx.rotary(n, x, None, pos, freq, rot, False, 1.0, out, None)
    step = 1 << 20
    part = torch.empty(step, 1, D, dtype=torch.bfloat16, device=DEV)
    for at in (0, 5 * step + 3, n - step):                     # a call of these tokens alone, whose waves take one each
        ctx.rotary(step, x[at: at + step], None, pos[at: at + step].clone(), freq, rot, False, 1.0, part, None)
        assert torch.equal(out[at: at + step], part)


# ---- append ---------------------------------------------------------------------------------------------------------------

def device_cache(ref):
    return {"K": torch.as_tensor(ref.codes[0]).to(DEV), "V": torch.as_tensor(ref.codes[1]).to(DEV), "ks": torch.as_tensor(ref.scale[0]).float().to(DEV),
            "vs": torch.as_tensor(ref.scale[1]).float().to(DEV), "acc": torch.as_tensor(ref.acc).float().to(DEV), "cu": i32(ref.cu)}


def same_codes(got, want):
    nan = (want & 0x7f) == 0x7f
    return np.array_equal(got[~nan], want[~nan]) and np.all((got[nan] & 0x7f) == 0x7f)


def check_cache(dev, ref):
    assert same_codes(dev["K"].cpu().numpy(), ref.codes[0]) and same_codes(dev["V"].cpu().numpy(), ref.codes[1])
    assert np.array_equal(f64(dev["ks"]), ref.scale[0]) and np.array_equal(f64(dev["vs"]), ref.scale[1])
    assert np.array_equal(dev["acc"].cpu().numpy(), ref.acc.astype(np.float32))


def random_rows(rng, m, dtype, spread=1.5):
    x = torch.from_numpy(rng.standard_normal((m, D)) * np.exp(spread * rng.standard_normal((m, 1)))).to(TYPES[dtype])
    return x


def filled(cu, L, H, block, rng):
    """A cache with something in every place, used or not."""
    ref = R.Cache(cu, L, H, block)
    ref.codes[...] = rng.randint(0, 0x7f, ref.codes.shape) | (rng.randint(0, 2, ref.codes.shape) << 7)
    ref.scale[...] = np.exp2(rng.randint(-9, 3, ref.scale.shape))
    ref.acc[...] = rng.rand(*ref.acc.shape).astype(np.float32)
    return ref


def run_append(ref, dev, ctx, layer, held, new, k, v, n_tok, T, with_acc=True, max_new=None, cu_new=None):
    """k, v [n][H][D] torch on the CPU."""
    cu_new = np.concatenate([[0], np.cumsum(new)]) if cu_new is None else cu_new
    ctx.cache_append(layer, ref.B, k.to(DEV), v.to(DEV), len(k), i32(cu_new), int(max(new)) if max_new is None else max_new, dev["cu"], n_tok, dev["K"], dev["V"],
                     dev["ks"], dev["vs"], T, ref.block, dev["acc"] if with_acc else None)
    keep = ref.acc.copy()
    for b in range(ref.B):
        for h in range(ref.H):
            part = slice(int(cu_new[b]), int(cu_new[b]) + int(new[b]))
            ref.append(layer, b, h, int(held[b][h]), k[part, h].double().numpy(), v[part, h].double().numpy())
    if not with_acc:
        ref.acc[...] = keep


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("new,held", [((1,), (0,)), ((1, 1, 1), (63, 64, 5)), ((300, 0, 17), (3, 40, 127)), ((129, 255), (0, 128)), ((1, 16, 15), (15, 16, 1))])
def test_append(dtype, block, new, held):
    rng = np.random.RandomState(block + len(new))
    L, H, B = 2, 3, len(new)
    cu = np.concatenate([[0], np.cumsum(np.array(new) + np.array(held) + rng.randint(0, 40, B))])
    ref = filled(cu, L, H, block, rng)
    dev, T = device_cache(ref), ref.T
    ctx = context(L=L, H=H, dtype=dtype)
    heldh = np.array([[x, max(0, x - 1), max(0, x - 20)] for x in held])           # heads may hold unlike numbers
    n = sum(new)
    k, v = (torch.stack([random_rows(rng, n, dtype) for _ in range(H)], 1) for _ in range(2))
    k[0, 0, 5], v[0, 1, 7], v[0, 1, 9] = math.nan, math.inf, -math.inf
    k[n // 2, 1] = 0.0
    for with_acc in (True, False):
        run_append(ref, dev, ctx, 1, heldh, new, k, v, i32(heldh), T, with_acc)
        check_cache(dev, ref)
    run_append(ref, dev, ctx, 0, heldh, new, 300 * v, k, i32(heldh), T)            # larger rows: scales grow
    check_cache(dev, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_rounds_every_value_to_its_nearest_code(dtype):
    """All 2^16 bf16 values (fp32: with neighbours), in blocks of like size and of unlike sizes, subnormal and non-finite ones among them."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    rows = bits.view(-1, D)
    if dtype == "f32":
        rows = (rows.float().view(torch.int32) + torch.arange(-1, 2, dtype=torch.int32).repeat(43)[:128] * 3).view(torch.float32)
    n = len(rows)
    for order in (np.arange(n), np.random.RandomState(3).permutation(n)):
        ref = R.Cache([0, n + 5], 1, 1, 16)
        dev = device_cache(ref)
        k = rows[torch.from_numpy(order)][:, None]
        run_append(ref, dev, context(H=1, dtype=dtype), 0, [[0]], [n], k, k.flip(0), i32([[0]]), ref.T)
        check_cache(dev, ref)


def test_append_token_by_token_and_what_does_not_fit():
    rng = np.random.RandomState(8)
    H, block = 2, 32
    ref = filled([0, 70, 75, 200], 1, H, block, rng)
    dev, ctx = device_cache(ref), context(H=H)
    n_tok = torch.zeros(3, H, dtype=torch.int32, device=DEV)
    for step in range(80):                                  # the second sequence has 5 rows, the first 70
        k, v = (torch.stack([random_rows(rng, 3, "bf16") for _ in range(H)], 1) for _ in range(2))
        run_append(ref, dev, ctx, 0, [[min(step, c)] * H for c in (70, 5, 125)], [1, 1, 1], k, v, n_tok, ref.T)
        n_tok += 1
    check_cache(dev, ref)
    # counts and offsets that say more than there is: cut, nothing outside touched.  (Of the first call's, head 0 of the last sequence fits: 6 tokens behind 70 of 125 rows.)
    k = torch.stack([random_rows(rng, 9, "bf16") for _ in range(H)], 1)
    kept = ref.acc.copy()
    ref.append(0, 2, 0, 70, *[k[3:, 0].double().numpy()] * 2)
    ref.acc[...] = kept
    ctx.cache_append(0, 3, k.to(DEV), k.to(DEV), 9, i32([0, 3, 3, 9]), 9, i32([0, 70, 75, 4000]), i32([[70, 1 << 30]] * 3), dev["K"], dev["V"], dev["ks"], dev["vs"], 200, block)
    ctx.cache_append(0, 3, k.to(DEV), k.to(DEV), 9, i32([5, 5, 2, -4]), 9, dev["cu"], i32([[0, 0]] * 3), dev["K"], dev["V"], dev["ks"], dev["vs"], 200, block)
    ctx.cache_append(0, 3, k.to(DEV), k.to(DEV), 9, i32([0, 3, 6, 9]), 9, i32([300, -5, 250, 200]), i32([[0, 0]] * 3), dev["K"], dev["V"], dev["ks"], dev["vs"], 200, block)
    ctx.cache_append(0, 3, k.to(DEV), k.to(DEV), 0, i32([0, 3, 6, 9]), 9, dev["cu"], i32([[0, 0]] * 3), dev["K"], dev["V"], dev["ks"], dev["vs"], 200, block)
    check_cache(dev, ref)
    # more tokens than max_new: the first ones
    run_append(ref, dev, ctx, 0, [[0, 0]] * 3, [2, 2, 2], k, k, i32([[0, 0]] * 3), 200, max_new=2, cu_new=[0, 3, 6, 9])
    check_cache(dev, ref)


@pytest.mark.parametrize("block", [16, 64])
def test_append_of_more_blocks_than_a_grid_has(block):
    """65535 launch blocks of 32 rows (or of one scale block of 64) take 2.1 (4.2) million rows of a head: the first ones take rows again behind them."""
    n, held = 65535 * max(block, 32) + 5003, 5
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    T = n + held
    ctx = skv.Context(skv.Desc(n_layers=1, n_q_heads=1, n_kv_heads=1, kv_dtype=skv.SKV_BF16, max_tokens=T, max_batch=1))
    g = torch.Generator(device=DEV).manual_seed(block)
    k, v = (torch.randn(n, 1, D, device=DEV, generator=g).mul_(torch.exp(torch.randn(n, 1, 1, device=DEV, generator=g))).bfloat16() for _ in range(2))
    K, V = (torch.zeros(1, 1, T, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.full((1, 1, T // block + 1), 2.0 ** -9, device=DEV) for _ in range(2))
    acc = torch.ones(1, 1, T, device=DEV)
    ctx.cache_append(0, 1, k, v, n, i32([0, n]), n, i32([0, T]), i32([[held]]), K, V, ks, vs, T, block, acc)
    blocks = -(-T // block)
    for x, codes, scale in ((k, K, ks), (v, V, vs)):
        rows = torch.zeros(blocks * block, D, dtype=torch.bfloat16, device=DEV)
        rows[held: T] = x[:, 0]
        most = rows.view(blocks, -1).abs().amax(1).double()
        e = torch.ceil(torch.log2(most / 448.0)).clamp(min=-9.0)                   # (no quotient of bf16 numbers by 448 is near enough to a power of two to be rounded across it but for the powers)
        want = torch.exp2(e)
        assert bool((most <= 448.0 * want).all()) and bool(((most > 224.0 * want) | (want == 2.0 ** -9)).all())
        assert torch.equal(scale[0, 0, :blocks].double()[1:], want[1:]) and float(scale[0, 0, 0]) == max(2.0 ** -9, float(want[0]))
        lost = (rows.view(blocks, block, D).float() / want[:, None, None].float()).to(torch.float8_e4m3fn).view(torch.uint8).view(-1, D)
        assert torch.equal(codes[0, 0, held:], lost[held: T]) and int(codes[0, 0, :held].max()) == 0
        del rows, lost
    assert bool((acc[0, 0, held:] == 0).all()) and bool((acc[0, 0, :held] == 1).all())


# ---- attend ---------------------------------------------------------------------------------------------------------------

def run_attend(ref, dev, ctx, layer, q, n_tok, max_n, idx=None, acc=None, acc_out=None, decay=1.0, lse=True):
    B, Hq = q.shape[:2]
    out, l = torch.full((B, Hq, D), 9.0, device=DEV), torch.full((B, Hq), 9.0, device=DEV)
    work = torch.full((ctx.cache_attend_work_bytes(B, max_n, acc_out is not None),), 0xAB, dtype=torch.uint8, device=DEV)
    ctx.cache_attend(layer, B, q, dev["K"], dev["V"], dev["ks"], dev["vs"], ref.T, ref.block, dev["cu"], n_tok, idx, max_n, out, l if lse else None, acc, acc_out, decay, work)
    return f64(out), f64(l)


def check_attend(ref, layer, q, n, out, lse, idx=None, acc=None, decay=1.0, acc_out=None):
    B, Hq = q.shape[:2]
    H, G = ref.H, Hq // ref.H
    q = f64(q)
    want_acc = None if acc_out is None else acc_out[0].copy()
    slack = None if acc_out is None else np.zeros_like(want_acc)
    for b in range(B):
        for h in range(H):
            m = int(n[b][h])
            rows = np.arange(m) if idx is None else np.asarray(idx[b][h][:m])
            rows = rows[(rows >= 0) & (rows < ref.cu[b + 1] - ref.cu[b])]
            K, V = (ref.rows(kv, layer, h, b, rows) for kv in range(2))
            want, wl, p, l1 = R.attend(q[b, h * G:(h + 1) * G], K, V)
            # A logit: 128 products and their fp32 sum (fp32 queries: three pieces, 384), scale and 1 / sqrt(D): (384 + 4) half steps of the sum of |products|.  A weight:
            # twice that (numerator and normaliser), the exponent's own rounding and exp2; sums over the rows of a wave and over waves and blocks.
            logit = 388 * EPS * l1
            weight = 2 * logit + 2 * (abs(wl).max() if len(rows) else 0.0) * 4 * EPS + 8 * EPS + (len(rows) / 32 + 300) * EPS
            size = np.stack([(p[g][:, None] * np.abs(V)).sum(0) for g in range(G)]) if len(rows) else 0.0
            got, gl = out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G]
            assert np.all(np.abs(got - want) <= 2 * weight * size + 1e-30), (b, h, np.abs(got - want).max())
            if len(rows):
                assert np.all(np.abs(gl - wl) <= logit + weight + 4 * EPS * np.abs(wl)), (b, h)
            else:
                assert np.all(np.isneginf(gl)) and np.all(got == 0.0)
            if acc_out is not None:
                at = ref.cu[b] + np.arange(m)
                want_acc[layer, h, at] = (0.0 if acc is None else decay * acc[layer, h, at]) + p.sum(0)
                slack[layer, h, at] = p.sum(0) * 2 * weight + 4 * EPS * want_acc[layer, h, at]
    if acc_out is not None:
        assert np.all(np.abs(acc_out[1] - want_acc) <= slack)


def attend_case(seed, lengths, H, G, dtype, block, L=2):
    rng = np.random.RandomState(seed)
    cu = np.concatenate([[0], np.cumsum(np.array(lengths) + rng.randint(0, 30, len(lengths)))])
    ref = filled(cu, L, H, block, rng)
    ref.scale[0] = np.exp2(rng.randint(-10, -5, ref.scale[0].shape))
    q = torch.from_numpy(rng.standard_normal((len(lengths), H * G, D))).to(TYPES[dtype]).to(DEV)
    return rng, ref, device_cache(ref), context(L=L, H=H, G=G, dtype=dtype), q


LENGTHS = [(1,), (0,), (15, 16, 17, 0), (31, 32, 33), (127, 128, 129, 1), (700, 5), (3001,)]


@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("H,G,dtype,block", [(1, 1, "bf16", 16), (2, 2, "f32", 32), (3, 4, "bf16", 128), (1, 8, "f32", 64), (2, 8, "bf16", 64)])
def test_attend_rows_in_use(lengths, H, G, dtype, block):
    rng, ref, dev, ctx, q = attend_case(sum(lengths) + G, lengths, H, G, dtype, block)
    n = np.array([[x, max(0, x - 1), max(0, x - 9)][:H] for x in lengths])
    max_n = int(n.max())
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n), max_n)
    check_attend(ref, 1, q, n, out, lse)
    again = run_attend(ref, dev, ctx, 1, q, i32(n), max_n)
    assert np.array_equal(out, again[0]) and np.array_equal(lse, again[1])
    out2, _ = run_attend(ref, dev, ctx, 1, q, i32(n), max_n, lse=False)
    assert np.array_equal(out, out2)
    # a bound on the lengths that is far too high changes how the work is cut, not what comes out
    out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), max_n + 5000)
    check_attend(ref, 0, q, n, out, lse)


@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("H,G,dtype,block", [(1, 1, "f32", 16), (2, 8, "bf16", 32), (3, 4, "bf16", 64)])
def test_attend_gathers_the_weights(lengths, H, G, dtype, block):
    rng, ref, dev, ctx, q = attend_case(sum(lengths) + 3 * G, lengths, H, G, dtype, block)
    n = np.array([[x, max(0, x - 1), max(0, x - 9)][:H] for x in lengths])
    for acc, decay in ((None, 1.0), (dev["acc"], 0.875)):
        acc_out = torch.rand(ref.acc.shape, device=DEV)
        before = f64(acc_out)
        out, lse = run_attend(ref, dev, ctx, 1, q, i32(n), int(n.max()), acc=acc, acc_out=acc_out, decay=decay)
        check_attend(ref, 1, q, n, out, lse, acc=None if acc is None else ref.acc, decay=decay, acc_out=(before, f64(acc_out)))
    inplace = dev["acc"].clone()
    run_attend(ref, dev, ctx, 1, q, i32(n), int(n.max()), acc=inplace, acc_out=inplace, decay=0.875)
    used = torch.zeros_like(acc_out, dtype=torch.bool)
    for b in range(len(lengths)):
        for h in range(H):
            used[1, h, ref.cu[b]: ref.cu[b] + int(n[b][h])] = True
    assert torch.equal(inplace[used], acc_out[used]) and torch.equal(inplace[~used], dev["acc"][~used])


@pytest.mark.parametrize("lengths", [(1, 0, 700, 33), (0, 0, 0), (0, 5000, 1, 0, 129), (128, 128, 128), (4097, 300)])
@pytest.mark.parametrize("H,G,dtype,block", [(1, 1, "bf16", 16), (2, 8, "bf16", 32), (3, 4, "f32", 64)])
@pytest.mark.parametrize("weights", [False, True])
def test_attend_deals_long_batches_in_equal_shares(lengths, H, G, dtype, block, weights):
    """The bound on the lengths says that a batch is long: blocks then take equal shares of all rows, whatever the lengths are (some more blocks than rows)."""
    rng, ref, dev, ctx, q = attend_case(sum(lengths) + 7 * G, lengths, H, G, dtype, block)
    n = np.array([[x, max(0, x - 1), max(0, x - 9)][:H] for x in lengths])
    acc_out = torch.rand(ref.acc.shape, device=DEV) if weights else None
    before = f64(acc_out) if weights else None
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n), 400000, acc=dev["acc"] if weights else None, acc_out=acc_out, decay=0.5)
    check_attend(ref, 1, q, n, out, lse, acc=ref.acc, decay=0.5, acc_out=(before, f64(acc_out)) if weights else None)
    again = run_attend(ref, dev, ctx, 1, q, i32(n), 400000)
    if not weights:
        assert np.array_equal(out, again[0]) and np.array_equal(lse, again[1])


@pytest.mark.parametrize("B", [512, 513, 600])
def test_attend_as_many_pairs_as_equal_shares_are_dealt_for_and_more(B):
    lengths = tuple(int(x) for x in np.random.RandomState(0).randint(0, 200, B))
    rng, ref, dev, _, q = attend_case(1, lengths, 2, 1, "bf16", 32, L=1)
    ctx = context(H=2, G=1, batch=B)
    n = np.array([[x, x // 2] for x in lengths])
    for max_n in (200, 3000):
        acc_out = torch.rand(ref.acc.shape, device=DEV)
        before = f64(acc_out)
        out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), max_n, acc=dev["acc"], acc_out=acc_out)
        check_attend(ref, 0, q, n, out, lse, acc=ref.acc, acc_out=(before, f64(acc_out)))


@pytest.mark.parametrize("B,most,long", [(600, 900, 0), (600, 40, 20000), (2048, 20, 9000), (2049, 20, 9000)])
def test_attend_of_more_pairs_alike_and_with_a_long_one_among_them(B, most, long):
    """More pairs than those of long batches that always take shares: chunks of their own, or shares where one sequence has most of the rows, up to 4096 pairs."""
    lengths = [int(x) for x in np.random.RandomState(1).randint(0, most, B)]
    lengths[B - 2] = long or lengths[B - 2]
    rng, ref, dev, _, q = attend_case(1, tuple(lengths), 2, 1, "bf16", 32, L=1)
    ctx = context(H=2, G=1, batch=B)
    n = np.array([[x, x // 2] for x in lengths])
    acc_out = torch.rand(ref.acc.shape, device=DEV)
    before = f64(acc_out)
    out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), max(lengths), acc=dev["acc"], acc_out=acc_out)
    check_attend(ref, 0, q, n, out, lse, acc=ref.acc, acc_out=(before, f64(acc_out)))
    two, lse2 = run_attend(ref, dev, ctx, 0, q, i32(n), max(lengths))
    check_attend(ref, 0, q, n, two, lse2)


def test_attend_of_many_rows_of_one_sequence():
    """More parts than the attention launch joins itself, and scores of more tiles than a wave keeps."""
    rng, ref, dev, ctx, q = attend_case(3, (70001,), 1, 2, "bf16", 128, L=1)
    acc_out = torch.rand(ref.acc.shape, device=DEV)
    before = f64(acc_out)
    n = np.array([[70001]])
    out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), 70001, acc=dev["acc"], acc_out=acc_out, decay=0.25)
    check_attend(ref, 0, q, n, out, lse, acc=ref.acc, decay=0.25, acc_out=(before, f64(acc_out)))
    two, _ = run_attend(ref, dev, ctx, 0, q, i32(n), 70001)
    check_attend(ref, 0, q, n, two, lse)


@pytest.mark.parametrize("length,listed", [(40, 1), (40, 40), (900, 129), (5000, 2048), (5000, 1027)])
@pytest.mark.parametrize("H,G,dtype,block", [(1, 1, "bf16", 16), (2, 4, "f32", 32), (3, 8, "bf16", 64)])
def test_attend_listed_rows(length, listed, H, G, dtype, block):
    rng, ref, dev, ctx, q = attend_case(length + listed, (length, length // 2 + 1), H, G, dtype, block)
    idx = np.full((2, H, listed), -5, np.int32)
    n = np.zeros((2, H), np.int32)
    for b, m in enumerate((length, length // 2 + 1)):
        for h in range(H):
            n[b, h] = min(listed, m) - (h if listed > 8 else 0)
            idx[b, h, : n[b, h]] = np.sort(rng.permutation(m)[: n[b, h]])
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n), listed, idx=i32(idx))
    check_attend(ref, 1, q, n, out, lse, idx)
    # entries that are no rows are skipped, the same row twice counts twice, any order
    for b in range(2):
        for h in range(H):
            rng.shuffle(idx[b, h, : n[b, h]])
            some = rng.rand(n[b, h]) < 0.2
            idx[b, h, : n[b, h]][some] = rng.choice([-1, -2 ** 31, 2 ** 31 - 1, ref.T, 0, 0], some.sum())
    idx[1, H - 1] = -1                                      # nothing is left of this one
    out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), listed, idx=i32(idx))
    check_attend(ref, 0, q, n, out, lse, idx)


def test_attend_leaves_out_what_is_not_in_use():
    """NaN codes in every row behind the ones in use, in other sequences and in skipped entries' place: no trace in the results."""
    rng, ref, dev, ctx, q = attend_case(5, (37, 100), 2, 4, "bf16", 32)
    n = np.array([[37, 20], [0, 99]])
    for h in range(2):
        for b in range(2):
            a = ref.cu[b]
            for kv in range(2):
                ref.codes[kv, :, h, a + n[b, h]: ref.cu[b + 1]] = 0x7f
    dev = device_cache(ref)
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n), 100)
    check_attend(ref, 1, q, n, out, lse)
    idx = np.full((2, 2, 50), 99, np.int32)                 # rows 99: in sequence 1 NaN, in sequence 0 none
    idx[:, :, 1::2] = np.arange(25)
    idx[:, :, ::2] = -1
    n2 = np.array([[30, 30], [0, 50]])
    ref.codes[1, :, :, ref.cu[0]] = 0x7f                    # row 0, which a skipped entry might read
    idx[:, :, 1] = 2
    dev = device_cache(ref)
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n2), 50, idx=i32(idx))
    check_attend(ref, 1, q, n2, out, lse, idx)


def test_attend_scales_of_blocks_not_in_use_leave_no_trace():
    """NaN in the scales of every block without rows in use (memory that nothing was written to): lists of entries that are no rows, empty sequences, empty lists."""
    rng, ref, dev, ctx, q = attend_case(8, (64, 100, 5), 2, 4, "bf16", 32)
    n = np.array([[33, 0], [99, 64], [0, 0]])
    for b in range(3):
        for h in range(2):
            used = -(-int(n[b, h]) // 32)
            ref.scale[:, :, h, ref.slot(b, 0) + used: ref.slot(b + 1, 0) if b < 2 else ref.ns] = np.nan
    dev = device_cache(ref)
    acc_out = torch.zeros(ref.acc.shape, device=DEV)
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n), 100, acc_out=acc_out)
    check_attend(ref, 1, q, n, out, lse, acc_out=(np.zeros(ref.acc.shape), f64(acc_out)))
    idx = np.full((3, 2, 40), -1, np.int32)
    idx[0, 0, :20], idx[1, :, 5:15] = np.arange(20), np.arange(10)
    n2 = np.array([[40, 40], [30, 40], [40, 0]])
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n2), 40, idx=i32(idx))
    check_attend(ref, 1, q, n2, out, lse, idx)
    assert np.all(out[2] == 0.0) and np.all(np.isneginf(lse[2])) and np.all(out[0, 4:] == 0.0)
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n2), 0, idx=i32(idx))
    assert np.all(out == 0.0) and np.all(np.isneginf(lse))


def test_attend_counts_and_offsets_are_cut_to_the_pool():
    rng, ref, dev, ctx, q = attend_case(6, (37, 100), 2, 4, "bf16", 32)
    full = np.array([[ref.cu[b + 1] - ref.cu[b]] * 2 for b in range(2)])
    want = run_attend(ref, dev, ctx, 1, q, i32(full), 200)
    got = run_attend(ref, dev, ctx, 1, q, i32([[1 << 30, 1 << 30]] * 2), 200)
    assert np.array_equal(want[0], got[0]) and np.array_equal(want[1], got[1])
    got = run_attend(ref, dev, ctx, 1, q, i32(full), 30)                            # no more than max_n
    check_attend(ref, 1, q, np.minimum(full, 30), *got)
    dev["cu"] = i32([-4, 1 << 30, 3])
    got = run_attend(ref, dev, ctx, 1, q, i32([[-5, 3]] * 2), 200)
    assert np.all(got[0] == 0.0) and np.all(np.isneginf(got[1]))
    acc_out = torch.rand(ref.acc.shape, device=DEV)
    before = acc_out.clone()
    run_attend(ref, dev, ctx, 1, q, i32([[5, 3]] * 2), 0, acc_out=acc_out)
    assert torch.equal(before, acc_out)


def test_scales_weights_and_counts_may_begin_at_any_word():
    rng, ref, dev, ctx, q = attend_case(21, (300, 77), 3, 2, "bf16", 32)
    n = np.array([[300, 299, 3], [77, 0, 1]])

    def moved(x):
        y = torch.zeros(x.numel() + 5, dtype=x.dtype, device=DEV)
        y[5:] = x.flatten()
        return y[5:].view(x.shape)

    want = run_attend(ref, dev, ctx, 1, q, i32(n), 300, acc=dev["acc"], acc_out=(a := torch.zeros_like(dev["acc"])))
    m = dict(dev, ks=moved(dev["ks"]), vs=moved(dev["vs"]))
    got = run_attend(ref, m, ctx, 1, q, moved(i32(n)), 300, acc=moved(dev["acc"]), acc_out=(b := moved(torch.zeros_like(a))))
    assert np.array_equal(want[0], got[0]) and np.array_equal(want[1], got[1]) and torch.equal(a, b)
    m["acc"] = moved(dev["acc"])
    k = torch.randn(5, 3, D).bfloat16()
    run_append(ref, m, ctx, 1, n, [3, 2], k, 4 * k, moved(i32(n)), ref.T)
    check_cache(m, ref)
    idx, n_keep = torch.zeros(2, 2, 3, 9, dtype=torch.int32, device=DEV), torch.zeros(2, 2, 3, dtype=torch.int32, device=DEV)
    ctx.cache_evict(2, m["acc"], ref.T, m["cu"], moved(i32([n, n])), 300, 9, 2, 3, idx, n_keep)
    for l in range(2):
        for b in range(2):
            for h in range(3):
                at = R.evict(ref.acc[l, h, ref.cu[b]: ref.cu[b] + n[b, h]].astype(np.float32), 9, 2, 3)
                assert np.array_equal(idx[l, b, h, : len(at)].cpu().numpy(), at)
                ref.compact(l, b, h, at)
    ctx.cache_compact(2, m["K"], m["V"], m["ks"], m["vs"], m["acc"], ref.T, 32, m["cu"], idx, 9, n_keep, m["K"], m["V"], m["ks"], m["vs"], m["acc"])
    check_cache(m, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_special_logits(dtype):
    rng, ref, dev, ctx, q = attend_case(9, (200,), 2, 2, dtype, 64)
    ref.codes[0, 1, 0, 77, 3] = 0x7f                        # a NaN key in head 0, a NaN value in head 1
    ref.codes[1, 1, 1, 12, 5] = 0xff
    dev = device_cache(ref)
    out, lse = run_attend(ref, dev, ctx, 1, q, i32([[200, 200]]), 200)
    assert np.all(np.isnan(out[0, :2])) and np.all(np.isnan(lse[0, :2]))
    assert np.all(np.isnan(out[0, 2:, 5])) and np.all(np.isfinite(out[0, 2:, :5])) and np.all(np.isfinite(lse[0, 2:]))
    # infinite and NaN queries: NaN for their heads, nothing else
    rng, ref, dev, ctx, q = attend_case(10, (200,), 2, 2, dtype, 64)
    q[0, 1, 4], q[0, 2, 9] = math.inf, math.nan
    out, lse = run_attend(ref, dev, ctx, 1, q, i32([[200, 200]]), 200)
    assert np.all(np.isnan(out[0, 1:3])) and np.all(np.isfinite(out[0, [0, 3]])) and np.all(np.isfinite(lse[0, [0, 3]]))


@pytest.mark.parametrize("shift", [-60, 40])
def test_attend_large_and_small_magnitudes(shift):
    """Logits of up to thousands, scales far from one: the running reference moves, weights vanish."""
    rng, ref, dev, ctx, q = attend_case(11, (900, 333), 2, 4, "f32", 16)
    ref.scale[0] *= 64.0
    ref.scale[1] = np.exp2(rng.randint(shift - 3, shift, ref.scale[1].shape))
    dev = device_cache(ref)
    n = np.array([[900, 800], [333, 1]])
    acc_out = torch.rand(ref.acc.shape, device=DEV)
    before = f64(acc_out)
    out, lse = run_attend(ref, dev, ctx, 1, q, i32(n), 900, acc_out=acc_out)
    # a logit of thousands is off by more than a weight may be for the plain bound: what is checked is the same, with its larger logit error
    for b in range(2):
        for h in range(2):
            K, V = (ref.rows(kv, 1, h, b, np.arange(n[b, h])) for kv in range(2))
            want, wl, p, l1 = R.attend(f64(q)[b, h * 4:(h + 1) * 4], K, V)
            d = math.expm1(2 * 388 * EPS * l1 + 8 * EPS * l1) + 400 * EPS
            size = np.stack([(p[g][:, None] * np.abs(V)).sum(0) for g in range(4)])
            # and numbers below 2^-126, the smallest normal one, may count as zero: a weight times its scale, which meets codes of up to 448, in every row
            gone = 448 * 2.0 ** -126 * n[b, h]
            assert np.all(np.abs(out[b, h * 4:(h + 1) * 4] - want) <= 2 * d * size + gone)
            assert np.all(np.abs(lse[b, h * 4:(h + 1) * 4] - wl) <= d + 400 * EPS * l1)


def weight_bound(l1, lse, rows):
    """A weight's relative error, as in check_attend."""
    return 2 * 388 * EPS * l1 + 8 * EPS * float(np.abs(lse).max()) + 8 * EPS + (rows / 32 + 300) * EPS


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [(40, 7), (900, 300)])
def test_attend_logits_of_minus_infinity_weigh_nothing(dtype, lengths):
    """A query with an infinite element over keys that are positive there: all of its logits are -inf (nothing is weighed, as without rows) or +inf (NaN); the other
    queries are what they are without it.  NaN queries stay NaN wherever their bits are."""
    rng, ref, dev, ctx, q = attend_case(12, lengths, 2, 4, dtype, 64)
    ref.codes[0, 1, :, :, 4] = rng.randint(1, 0x7f, ref.codes[0, 1, :, :, 4].shape)
    dev, n = device_cache(ref), np.array([[x, x - 1] for x in lengths])
    plain = q.clone()
    q[:, 1, 4], q[:, 6, 4], q[:, 5, 4] = -math.inf, math.inf, math.nan
    if dtype == "f32":
        q.view(torch.int32)[:, 5, 4] = 0x7f800001              # NaN by its last bit
    acc_out = torch.rand(ref.acc.shape, device=DEV)
    want_out, want_lse = run_attend(ref, dev, ctx, 1, plain, i32(n), max(lengths))
    idx = np.broadcast_to(np.arange(max(lengths)), (2, 2, max(lengths))).copy()
    listed = run_attend(ref, dev, ctx, 1, q, i32(n), max(lengths), idx=i32(idx))
    shares = run_attend(ref, dev, ctx, 1, q, i32(n), 400000)
    weighed = run_attend(ref, dev, ctx, 1, q, i32(n), max(lengths), acc=dev["acc"], acc_out=acc_out, decay=0.5)
    for out, lse in (run_attend(ref, dev, ctx, 1, q, i32(n), max(lengths)), listed, shares, weighed):
        assert np.all(out[:, 1] == 0.0) and np.all(np.isneginf(lse[:, 1]))
        assert np.all(np.isnan(out[:, 5:7])) and np.all(np.isnan(lse[:, 5:7]))
        for i in (0, 2, 3, 4, 7):
            assert np.all(np.abs(lse[:, i] - want_lse[:, i]) <= 1e-5 * np.abs(want_lse[:, i]) + 1e-5)
            assert np.all(np.isfinite(out[:, i]))
    for b in range(2):
        at = ref.cu[b] + np.arange(n[b, 0])
        finite = f64(plain)[b, [0, 2, 3]]
        K, V = (ref.rows(kv, 1, 0, b, np.arange(n[b, 0])) for kv in range(2))
        want, wl, p, l1 = R.attend(finite, K, V)
        w = weight_bound(l1, wl, n[b, 0])
        size = np.stack([(p[g][:, None] * np.abs(V)).sum(0) for g in range(3)])
        for out, _ in (listed, shares, weighed):
            assert np.all(np.abs(out[b, [0, 2, 3]] - want) <= 2 * w * size + 1e-30)
        got, sure = f64(acc_out)[1, 0, at], 0.5 * ref.acc[1, 0, at] + p.sum(0)
        assert np.all(np.abs(got - sure) <= p.sum(0) * 2 * w + 4 * EPS * sure)
        assert np.all(np.isnan(f64(acc_out)[1, 1, ref.cu[b] + np.arange(n[b, 1])]))


@pytest.mark.parametrize("size", [16.0, 64.0, 256.0])
@pytest.mark.parametrize("lengths,max_n", [((5,), 5), ((700,), 700), ((70001,), 70001), ((5, 3001), 400000)])
@pytest.mark.parametrize("G,dtype", [(1, "bf16"), (8, "f32")])
def test_gathered_weights_of_equal_rows_are_equal_parts_whatever_their_logits(size, lengths, max_n, G, dtype):
    """Rows alike have one logit, of 260 to 4200 in powers of two.  Every weight's power is then 1 and the normaliser the number of rows, exactly: a weight is off by
    the rounding of one quotient and of the product with it, the sum of G of them by G - 1 more.  In one block, in parts that the attention launch joins, in parts joined behind it, in shares."""
    ref = R.Cache(np.concatenate([[0], np.cumsum(lengths)]), 1, 1, 32)
    ref.codes[...] = 0x38                                      # 1
    dev, ctx = device_cache(ref), context(L=1, H=1, G=G, dtype=dtype)
    q = torch.full((len(lengths), G, D), size, dtype=TYPES[dtype], device=DEV)
    acc_out = torch.zeros(ref.acc.shape, device=DEV)
    out, _ = run_attend(ref, dev, ctx, 0, q, i32([[n] for n in lengths]), max_n, acc_out=acc_out)
    assert np.all(np.abs(out - 1.0) <= 4 * EPS)
    got = f64(acc_out)[0, 0]
    for b, n in enumerate(lengths):
        assert np.all(np.abs(got[ref.cu[b]: ref.cu[b + 1]] - G / n) <= (G + 2) * EPS * G / n), (b, n)


@pytest.mark.parametrize("max_n", [900, 400000])
def test_gathered_weights_of_large_logits_add_up(max_n):
    """Logits of up to 10^5: whatever the weights are, those of a query add up to 1, since the normaliser is the sum of the same powers.  Off by the roundings of that sum (a lane's rows, then
    waves and parts), by those of exponents, which are at most 64 half steps where a power counts, and by the products' own."""
    rng, ref, dev, ctx, q = attend_case(13, (900, 333), 2, 4, "f32", 16)
    ref.scale[0] *= 2.0 ** 13
    dev, n = device_cache(ref), np.array([[900, 800], [333, 1]])
    acc_out = torch.zeros(ref.acc.shape, device=DEV)
    run_attend(ref, dev, ctx, 1, q, i32(n), max_n, acc_out=acc_out)
    for b in range(2):
        for h in range(2):
            total = f64(acc_out)[1, h, ref.cu[b]: ref.cu[b] + n[b, h]].sum()
            assert abs(total - 4.0) <= 4.0 * (n[b, h] / 32 + 400) * EPS, (b, h, total)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_at_the_ends_of_its_range(dtype):
    """Elements of a query of 2^112, whose products with codes reach 2^128 nearly; rows times scale of 2^110, with weights of 200 times the reference's before they are divided."""
    ref = R.Cache([0, 1664], 1, 1, 32)
    rng, n = np.random.RandomState(0), np.array([[1664]])
    ref.codes[0] = 0x7e
    ref.codes[0, 0, 0, 1::3] = 0xfe                            # -448: these rows' weights vanish
    ref.scale[0] = 2.0 ** -100
    ref.codes[1] = rng.randint(0, 0x7f, ref.codes[1].shape)
    dev, ctx = device_cache(ref), context(H=1, G=1, dtype=dtype)
    q = torch.full((1, 1, D), 2.0 ** 112, dtype=TYPES[dtype], device=DEV)
    out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), 1664)
    rows = np.setdiff1d(np.arange(1664), np.arange(1, 1664, 3))
    want, logit = ref.rows(1, 0, 0, 0, rows).mean(0), 128 * 448 * 2.0 ** 12 / math.sqrt(D)
    # equal weights, exactly: a sum of them times values, and its quotient; the logit: scale, constant, their products
    assert np.all(np.abs(out[0, 0] - want) <= (1664 / 32 + 300) * EPS * want) and abs(lse[0, 0] - logit - math.log(len(rows))) <= 8 * EPS * logit
    # a wave's first tile sets its reference to 0, the others stay 7.65 above it (powers of two) without moving it
    ref.codes[0] = 0x37                                        # 0.9375
    ref.codes[0, 0, 0, :128] = 0
    ref.scale[0], ref.scale[1], ref.codes[1] = 0.5, 2.0 ** 99, 0x7e
    dev = device_cache(ref)
    q.fill_(1.0)
    for max_n in (400000, 1664):                               # 13 tiles a wave, and one
        out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), max_n)
        assert np.all(np.abs(out / (448 * 2.0 ** 99) - 1.0) <= (1664 / 32 + 300) * EPS)


def attend_on_device(dev, q, n, G, cu, block):
    """One KV head, in 64 bits on the device: out, lse, the sum of the weights of a row's queries, and the largest sum of |products| of a logit, for each sequence."""
    for b, m in enumerate(n):
        rows = torch.arange(m, device=DEV)
        slot = cu[b] // block + b + rows // block
        K, V = ((dev[x][0, 0, cu[b]: cu[b] + m].view(torch.float8_e4m3fn).double() * dev[s][0, 0, slot].double()[:, None]) for x, s in (("K", "ks"), ("V", "vs")))
        x = torch.stack([(q[b, g].double() * K).sum(1) for g in range(G)]) / math.sqrt(D)
        top = x.max(1, keepdim=True).values
        e = torch.exp(x - top)
        z = e.sum(1, keepdim=True)
        p = e / z
        size = torch.stack([(p[g][:, None] * V.abs()).sum(0) for g in range(G)])
        l1 = max(float((q[b, g].double().abs() * K.abs()).sum(1).max()) for g in range(G)) / math.sqrt(D)
        yield torch.stack([(p[g][:, None] * V).sum(0) for g in range(G)]), (top + torch.log(z))[:, 0], p.sum(0), size, l1


@pytest.mark.parametrize("G,dtype", [(1, "bf16"), (8, "bf16"), (2, "f32"), (8, "f32")])
@pytest.mark.parametrize("n,max_n", [((3001,), 400000), ((1664,), 400000), ((420001, 400777), 420001)])
def test_gathered_weights_of_more_tiles_than_a_wave_keeps(n, max_n, G, dtype):
    """A wave keeps the scores of 8 tiles before it writes them: 13 tiles in chunks of 1664 rows (one sequence whose bound is 400000 rows), 8 to 13 in shares of 820000 rows."""
    rng = np.random.RandomState(G)
    cu = np.concatenate([[0], np.cumsum(np.array(n) + 3)])
    T, block = int(cu[-1]), 64
    g = torch.Generator(device=DEV).manual_seed(G)
    dev = {x: torch.randint(0, 0x7f, (1, 1, T, D), device=DEV, generator=g, dtype=torch.uint8) | (torch.randint(0, 2, (1, 1, T, D), device=DEV, generator=g, dtype=torch.uint8) << 7)
           for x in ("K", "V")}
    dev.update({x: torch.exp2(torch.randint(-10, -5, (1, 1, T // block + len(n)), device=DEV, generator=g).float()) for x in ("ks", "vs")}, cu=i32(cu))
    dev["acc"] = torch.rand(1, 1, T, device=DEV, generator=g)
    ctx = context(H=1, G=G, dtype=dtype)
    ref = R.Cache([0, 1], 1, 1, block)
    ref.T = T
    q = torch.from_numpy(rng.standard_normal((len(n), G, D))).to(TYPES[dtype]).to(DEV)
    acc_out = torch.full((1, 1, T), -1.0, device=DEV)
    out, lse = run_attend(ref, dev, ctx, 0, q, i32(np.array(n)[:, None]), max_n, acc=dev["acc"], acc_out=acc_out, decay=0.5)
    for b, (want, wl, p, size, l1) in enumerate(attend_on_device(dev, q, n, G, cu, block)):
        logit = 388 * EPS * l1
        # sums of a wave's rows one by one: 128 rows a step of four waves' 32, at most 820000 / 512 of them in a block's share, or 1664
        w = 2 * logit + 8 * EPS * float(wl.abs().max()) + 8 * EPS + (1700 / 16 + 1200) * EPS
        assert np.all(np.abs(out[b] - f64(want)) <= 2 * w * f64(size) + 1e-30)
        assert np.all(np.abs(lse[b] - f64(wl)) <= logit + w + 4 * EPS * np.abs(f64(wl)))
        at = slice(int(cu[b]), int(cu[b]) + n[b])
        sure = 0.5 * dev["acc"][0, 0, at].double() + p
        # decay * acc, and G weights added to it one by one: G + 1 roundings of numbers up to the sum, half a step each
        assert bool(((acc_out[0, 0, at].double() - sure).abs() <= p * 2 * w + (G + 1) * EPS * sure).all())
        assert bool((acc_out[0, 0, at.stop: int(cu[b + 1])] == -1.0).all())


@pytest.mark.parametrize("lengths,listed", [((60000,), 40000), ((60000, 57000), 50000)])
@pytest.mark.parametrize("G,dtype", [(2, "bf16"), (8, "f32")])
def test_attend_long_lists(lengths, listed, G, dtype):
    """Chunks of 256 entries, and of 1024, the most that a block takes; more parts than the attention launch joins."""
    H = 1 if len(lengths) == 1 else 3
    rng, ref, dev, ctx, q = attend_case(listed + G, lengths, H, G, dtype, 64, L=1)
    B = len(lengths)
    idx, n = np.full((B, H, listed), -5, np.int32), np.zeros((B, H), np.int32)
    for b in range(B):
        for h in range(H):
            n[b, h] = (listed, listed - 1023, 700)[h]
            idx[b, h, : n[b, h]] = rng.permutation(lengths[b])[: n[b, h]]
            idx[b, h, : n[b, h]: 7] = rng.choice([-1, 2 ** 31 - 1, 0, lengths[b] - 1], len(range(0, n[b, h], 7)))
    idx[0, 0, 2048: 4096] = -1                                  # whole blocks of entries that are none
    out, lse = run_attend(ref, dev, ctx, 0, q, i32(n), listed, idx=i32(idx))
    check_attend(ref, 0, q, n, out, lse, idx)
    again = run_attend(ref, dev, ctx, 0, q, i32(n), listed, idx=i32(idx))
    assert np.array_equal(out, again[0]) and np.array_equal(lse, again[1])


# ---- evict and compact ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,keep,sink,recent", [(0, 4, 1, 1), (1, 1, 0, 0), (5, 5, 2, 2), (5, 0, 0, 0), (6, 5, 2, 3), (6, 5, 2, 2), (300, 77, 4, 30), (1024, 1023, 0, 0), (1025, 64, 0, 64),
                                                (1025, 64, 64, 0), (4097, 1000, 3, 500), (20000, 4096, 4, 1000), (70001, 9, 0, 1),
                                                (70001, 40000, 5, 34000), (32769, 32768, 0, 0), (150000, 150, 0, 0)])
@pytest.mark.parametrize("kind", ["spread", "ties", "special", "close"])
def test_evict(n, keep, sink, recent, kind):
    rng = np.random.RandomState(n + keep)
    L, H, B = 2, 2, 2
    cu = np.array([0, n + 3, 2 * n + 10])
    acc = rng.standard_normal((L, H, cu[-1])).astype(np.float32)
    if kind == "ties":
        acc = rng.randint(0, 3, acc.shape).astype(np.float32) * np.where(rng.rand(*acc.shape) < 0.5, -0.0, 1.0).astype(np.float32)
    elif kind == "special":
        for v in (np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-42):
            acc[rng.rand(*acc.shape) < 0.15] = v
    elif kind == "close":
        acc = (np.float32(0.7).view(np.int32) + rng.randint(0, 40, acc.shape).astype(np.int32)).view(np.float32)
    n_tok = np.array([[[n, max(0, n - 1)], [max(0, n - 2), n]]] * L)
    ctx = context(L=L, H=H)
    idx = torch.full((L, B, H, max(keep, 1)), -3, dtype=torch.int32, device=DEV)
    n_keep = torch.full((L, B, H), -3, dtype=torch.int32, device=DEV)
    ctx.cache_evict(B, torch.from_numpy(acc).to(DEV), int(cu[-1]), i32(cu), i32(n_tok), max(n, 1), keep, sink, recent, idx, n_keep)
    for l in range(L):
        for b in range(B):
            for h in range(H):
                m = n_tok[l, b, h]
                want = R.evict(acc[l, h, cu[b]: cu[b] + m], keep, sink, recent)
                got = idx[l, b, h].cpu().numpy()
                assert int(n_keep[l, b, h]) == len(want)
                assert np.array_equal(got[: len(want)], want) and np.all(got[len(want):] == -3), (l, b, h)


@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_evict_of_more_long_heads_than_have_room_at_once(kind):
    """100 heads of up to 40000 rows: their slices are counted in groups of heads; some heads are short, empty or hold less than may stay."""
    rng = np.random.RandomState(5)
    L, H, B, keep, sink, recent = 10, 2, 5, 3000, 2, 100
    n = np.array([40000, 33000, 0, 2500, 9000])
    cu = np.concatenate([[0], np.cumsum(n + 1)])
    acc = rng.standard_normal((L, H, cu[-1])).astype(np.float32)
    if kind == "ties":
        acc = np.round(acc * 2)
    n_tok = np.broadcast_to(n[None, :, None], (L, B, H)).copy()
    n_tok[3, 0, 1] = 39990
    ctx = context(L=L, H=H)
    idx = torch.full((L, B, H, keep), -3, dtype=torch.int32, device=DEV)
    n_keep = torch.full((L, B, H), -3, dtype=torch.int32, device=DEV)
    ctx.cache_evict(B, torch.from_numpy(acc).to(DEV), int(cu[-1]), i32(cu), i32(n_tok), 180000, keep, sink, recent, idx, n_keep)
    idx, n_keep = idx.cpu().numpy(), n_keep.cpu().numpy()
    for l in range(L):
        for b in range(B):
            for h in range(H):
                want = R.evict(acc[l, h, cu[b]: cu[b] + n_tok[l, b, h]], keep, sink, recent)
                assert n_keep[l, b, h] == len(want) and np.array_equal(idx[l, b, h, : len(want)], want) and np.all(idx[l, b, h, len(want):] == -3), (l, b, h)


def test_evict_cuts_counts_to_the_pool():
    ctx = context(H=2)
    acc = torch.rand(1, 2, 100, device=DEV)
    idx, n_keep = torch.full((1, 3, 2, 64), -3, dtype=torch.int32, device=DEV), torch.zeros(1, 3, 2, dtype=torch.int32, device=DEV)
    ctx.cache_evict(3, acc, 100, i32([0, 40, 30, 900]), i32([[[1 << 30, -4]] * 3]), 50, 64, 0, 0, idx, n_keep)
    assert n_keep.cpu().tolist() == [[[40, 0], [0, 0], [50, 0]]]
    assert idx[0, 0, 0, :40].cpu().tolist() == list(range(40)) and idx[0, 2, 0, :50].cpu().tolist() == list(range(50))


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("n,keep", [(1, 1), (40, 17), (128, 127), (129, 128), (300, 300), (1000, 257), (5000, 2500)])
def test_compact(inplace, block, n, keep):
    rng = np.random.RandomState(n + block)
    L, H, B = 2, 2, 2
    ref = filled([0, n + 5, 2 * n + 7], L, H, block, rng)
    ref.codes[:, 0, 0, 3: 9] = 0x7f
    dev, out = device_cache(ref), filled(ref.cu, L, H, block, rng)
    to = dev if inplace else device_cache(out)
    want = ref if inplace else out
    idx, n_keep = np.full((L, B, H, keep), -9, np.int32), np.zeros((L, B, H), np.int32)
    for l in range(L):
        for b in range(B):
            for h in range(H):
                m = max(0, min(keep, n) - (l + b + h if keep > 10 else 0))
                idx[l, b, h, :m], n_keep[l, b, h] = np.sort(rng.permutation(n)[:m]), m
                if l == 1 and h == 1:                       # the first rows stay where they are
                    idx[l, b, h, : m // 2] = np.arange(m // 2)
                    idx[l, b, h, m // 2: m] = np.arange(n - (m - m // 2), n)
                ref.compact(l, b, h, idx[l, b, h, :m], want)
    ctx = context(L=L, H=H)
    ctx.cache_compact(B, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"], ref.T, block, dev["cu"], i32(idx), keep, i32(n_keep), to["K"], to["V"], to["ks"], to["vs"],
                      to["acc"])
    check_cache(to, want)


def test_compact_of_lists_that_do_not_fit_and_without_weights():
    rng = np.random.RandomState(2)
    ref, out = filled([0, 50, 90], 1, 2, 16, rng), filled([0, 50, 90], 1, 2, 16, rng)
    dev, to, ctx = device_cache(ref), device_cache(out), context(H=2)
    idx = rng.randint(0, 40, (1, 2, 2, 30)).astype(np.int32)                        # any order, repeated: fine where the outputs are others
    idx[0, 0, 0, ::3], idx[0, 1, 1, ::2], idx[0, 0, 1] = -1, 40, 2 ** 31 - 1
    keep_acc = out.acc.copy()
    for b in range(2):
        for h in range(2):
            ref.compact(0, b, h, idx[0, b, h], out)
    out.acc[...] = keep_acc
    ctx.cache_compact(2, dev["K"], dev["V"], dev["ks"], dev["vs"], None, 90, 16, dev["cu"], i32(idx), 30, i32([[[1 << 30, 30]] * 2]), to["K"], to["V"], to["ks"], to["vs"], None)
    check_cache(to, out)


def test_evict_and_compact_of_more_heads_than_one_launch_has_threads_for():
    """70 layers, 4096 sequences, 15 heads: 4.3 million heads of 1024 threads are more than the 2^32 threads that a launch may have in a dimension.  Two rows a head, the heavier one stays."""
    L, B, H, block = 70, 4096, 15, 16
    T = 2 * B
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB")
    ctx = skv.Context(skv.Desc(n_layers=L, n_q_heads=H, n_kv_heads=H, kv_dtype=skv.SKV_BF16, max_tokens=T, max_sentences=1, max_budget=1, max_batch=B))
    g = torch.Generator(device=DEV).manual_seed(0)
    acc = torch.randint(0, 3, (L, H, B, 2), device=DEV, generator=g).float()
    which = (acc[..., 1] > acc[..., 0]).int()                                      # [L][H][B]; equal: the lower row
    cu, n_tok = i32(2 * np.arange(B + 1)), torch.full((L, B, H), 2, dtype=torch.int32, device=DEV)
    idx, n_keep = torch.full((L, B, H, 1), -3, dtype=torch.int32, device=DEV), torch.full((L, B, H), -3, dtype=torch.int32, device=DEV)
    ctx.cache_evict(B, acc, T, cu, n_tok, 5000, 1, 0, 0, idx, n_keep)             # (a bound of 5000 rows takes 1024 threads)
    assert torch.equal(idx[..., 0], which.transpose(1, 2)) and bool((n_keep == 1).all())
    K, V = (torch.randint(0, 127, (L, H, B, 2, D), device=DEV, generator=g, dtype=torch.uint8) for _ in range(2))
    ks, vs = (torch.ones(L, H, T // block + B, device=DEV) for _ in range(2))
    pick = which[..., None].bool()
    want = [torch.where(pick, x[..., 1, :], x[..., 0, :]) for x in (K, V)] + [acc.max(-1).values]
    second = K[..., 1, :].clone()
    ctx.cache_compact(B, K, V, ks, vs, acc, T, block, cu, idx, 1, n_keep, K, V, ks, vs, acc)
    assert torch.equal(K[..., 0, :], want[0]) and torch.equal(V[..., 0, :], want[1]) and torch.equal(acc[..., 0], want[2])
    assert torch.equal(K[..., 1, :], second) and bool((ks == 1).all()) and bool((vs == 1).all())


@pytest.mark.parametrize("inplace", [False, True])
def test_compact_of_lists_with_room_for_more_rows_than_there_are(inplace):
    """`keep` is the length of a list, not of a sequence: 2^31 - 1 entries of one head, of which 70 are used."""
    keep = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    rng = np.random.RandomState(4)
    ref, out = filled([0, 200], 1, 1, 32, rng), filled([0, 200], 1, 1, 32, rng)
    dev = device_cache(ref)
    to, want = (dev, ref) if inplace else (device_cache(out), out)
    ctx = context(H=1)
    idx, n_keep = torch.empty(keep, dtype=torch.int32, device=DEV), torch.zeros(1, 1, 1, dtype=torch.int32, device=DEV)
    ctx.cache_evict(1, dev["acc"], 200, dev["cu"], i32([[[70]]]), 200, keep, 4, 10, idx, n_keep)
    assert int(n_keep) == 70 and np.array_equal(idx[:70].cpu().numpy(), np.arange(70))
    rows = np.sort(rng.permutation(200)[:70])
    idx[:70] = i32(rows)
    ref.compact(0, 0, 0, rows, want)
    ctx.cache_compact(1, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"], 200, 32, dev["cu"], idx, keep, n_keep, to["K"], to["V"], to["ks"], to["vs"], to["acc"])
    check_cache(to, want)


@pytest.mark.parametrize("n", [2047, 2048, 2049, 4095, 4096, 4097, 8191, 8192, 8193, 16383, 16384, 16385, 32767, 32768])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_evict_at_the_lengths_where_its_blocks_change(n, kind):
    """256, 512 and 1024 threads of 8 images each, then 16 and 32 images."""
    rng = np.random.RandomState(n)
    H, keep, sink, recent = 3, n // 3, 4, n // 10
    acc = rng.standard_normal((1, H, n)).astype(np.float32)
    if kind == "ties":
        acc = np.round(acc)
    n_tok = np.array([n, n - 1, n // 2])
    idx, n_keep = torch.full((1, 1, H, keep), -3, dtype=torch.int32, device=DEV), torch.full((1, 1, H), -3, dtype=torch.int32, device=DEV)
    context(H=H).cache_evict(1, torch.from_numpy(acc).to(DEV), n, i32([0, n]), i32(n_tok[None, None]), n, keep, sink, recent, idx, n_keep)
    for h in range(H):
        want = R.evict(acc[0, h, : n_tok[h]], keep, sink, recent)
        assert int(n_keep[0, 0, h]) == len(want) and np.array_equal(idx[0, 0, h, : len(want)].cpu().numpy(), want), h


@pytest.mark.parametrize("block", [16, 128])
def test_compact_of_many_heads_in_groups(block):
    """64 heads to another cache: a block takes 384 rows, three groups of 128 with the next one on its way, the last ones fewer."""
    rng = np.random.RandomState(block)
    L, H, B, n, keep = 8, 4, 2, 2700, 2500
    ref, out = filled([0, n + 5, 2 * n + 7], L, H, block, rng), filled([0, n + 5, 2 * n + 7], L, H, block, rng)
    dev, to = device_cache(ref), device_cache(out)
    idx, n_keep = np.full((L, B, H, keep), -9, np.int32), np.zeros((L, B, H), np.int32)
    for l in range(L):
        for b in range(B):
            for h in range(H):
                m = keep - 131 * ((l + b + h) % 5)
                idx[l, b, h, :m], n_keep[l, b, h] = np.sort(rng.permutation(n)[:m]), m
                ref.compact(l, b, h, idx[l, b, h, :m], out)
    ctx = context(L=L, H=H)
    ctx.cache_compact(B, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"], ref.T, block, dev["cu"], i32(idx), keep, i32(n_keep), to["K"], to["V"], to["ks"], to["vs"], to["acc"])
    check_cache(to, out)


# ---- together -------------------------------------------------------------------------------------------------------------

def _loop(dtype, graph):
    """Tokens turned, appended, attended with their weights gathered, evicted and compacted: what a program does, step by step, against the same in 64 bits on
    the codes that the device holds."""
    L, H, G, B, block, keep = 2, 2, 4, 2, 32, 96
    ctx = context(L=L, H=H, G=G, dtype=dtype, batch=B)
    rng = np.random.RandomState(1)
    ref = R.Cache([0, 200, 330], L, H, block)
    dev, T = device_cache(ref), ref.T
    freq = skv.rotary_freqs(128, 10000.0)[0]
    fd, cu_new = freq.to(DEV), i32([0, 1, 2])
    n_tok = torch.zeros(L, B, H, dtype=torch.int32, device=DEV)
    pos = torch.zeros(B, dtype=torch.int32, device=DEV)
    q_in, k_in, v_in = (torch.zeros(L, B, h, D, dtype=TYPES[dtype], device=DEV) for h in (H * G, H, H))
    q, k = torch.zeros_like(q_in), torch.zeros_like(k_in)
    out, lse = torch.zeros(L, B, H * G, D, device=DEV), torch.zeros(L, B, H * G, device=DEV)
    work = torch.empty(ctx.cache_attend_work_bytes(B, 200, True), dtype=torch.uint8, device=DEV)
    idx, n_keep = torch.zeros(L, B, H, keep, dtype=torch.int32, device=DEV), torch.zeros(L, B, H, dtype=torch.int32, device=DEV)

    def step():
        for l in range(L):
            ctx.rotary(B, q_in[l], k_in[l], pos, fd, 128, False, 1.0, q[l], k[l])
            ctx.cache_append(l, B, k[l], v_in[l], B, cu_new, 1, dev["cu"], n_tok[l], dev["K"], dev["V"], dev["ks"], dev["vs"], T, block, dev["acc"])
        n_tok.add_(1)
        for l in range(L):
            ctx.cache_attend(l, B, q[l], dev["K"], dev["V"], dev["ks"], dev["vs"], T, block, dev["cu"], n_tok[l], None, 200, out[l], lse[l], dev["acc"], dev["acc"], 1.0, work)
        pos.add_(1)

    def evict():
        ctx.cache_evict(B, dev["acc"], T, dev["cu"], n_tok, 200, keep, 4, 20, idx, n_keep)
        ctx.cache_compact(B, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"], T, block, dev["cu"], idx, keep, n_keep, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"])
        n_tok.copy_(n_keep)

    results, run_step, run_evict = [], step, evict
    if graph:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            ctx.set_stream(s.cuda_stream)
            g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
            with torch.cuda.graph(g1, stream=s):
                step()
            with torch.cuda.graph(g2, stream=s):
                evict()
        torch.cuda.synchronize()
        run_step, run_evict = g1.replay, g2.replay
    held = 0
    for t in range(150):
        for x in (q_in, k_in, v_in):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape)) * (3.0 if t % 40 == 39 else 1.0)).to(x.dtype))
        torch.cuda.synchronize()
        run_step()
        held += 1
        torch.cuda.synchronize()
        kd, vd = k.cpu().double().numpy(), v_in.cpu().double().numpy()
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    ref.append(l, b, h, held - 1, kd[l, b, h][None], vd[l, b, h][None])
        if t % 29 == 0 or held == 130:
            for l in range(L):
                check_attend(ref, l, q[l], [[held] * H] * B, f64(out[l]), f64(lse[l]))
            ref.acc[...] = f64(dev["acc"])                  # sums of rounded weights: taken over, the rest has to follow from them
            check_cache(dev, ref)
        if held == 130:
            run_evict()
            torch.cuda.synchronize()
            for l in range(L):
                for b in range(B):
                    for h in range(H):
                        want = R.evict(ref.acc[l, h, ref.cu[b]: ref.cu[b] + held].astype(np.float32), keep, 4, 20)
                        assert np.array_equal(idx[l, b, h].cpu().numpy(), want)
                        ref.compact(l, b, h, want)
            held = keep
            check_cache(dev, ref)
        results.append((out.clone(), lse.clone()))
    return results, {x: dev[x].clone() for x in ("K", "V", "ks", "vs", "acc")}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_loop_of_all_of_them_and_its_replay(dtype):
    direct, cache = _loop(dtype, False)
    replayed, cache2 = _loop(dtype, True)
    for (a, b), (c, d) in zip(direct, replayed):
        assert torch.equal(a, c) and torch.equal(b, d)
    assert all(torch.equal(cache[x], cache2[x]) for x in cache)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_graph_made_for_far_more_rows_than_there_are(dtype):
    """What a program captures once is bounded by its capacity: attention in chunks and with the joining launch, eviction in slices, compaction in place, replayed at a few rows, at none, at unlike
    counts of heads and at more rows than fit a slice.  Against 64 bits and, bit for bit, the same calls made directly."""
    H, G, keep, most, rows = 2, 2, 500, 131072, 40000
    ctx, direct = context(H=H, G=G, dtype=dtype), context(H=H, G=G, dtype=dtype)
    rng = np.random.RandomState(6)
    ref = filled([0, rows], 1, H, 32, rng)
    ref.scale[0] = 2.0 ** -8
    start, dev, eager = (device_cache(ref) for _ in range(3))
    n_tok, q = torch.zeros(1, H, dtype=torch.int32, device=DEV), torch.zeros(1, H * G, D, dtype=TYPES[dtype], device=DEV)
    work = torch.empty(ctx.cache_attend_work_bytes(1, most, True), dtype=torch.uint8, device=DEV)

    def outputs():
        return (torch.zeros(1, H * G, D, device=DEV), torch.zeros(1, H * G, device=DEV), torch.full((1, 1, H, keep), -3, dtype=torch.int32, device=DEV),
                torch.zeros(1, 1, H, dtype=torch.int32, device=DEV))

    def calls(ctx, dev, out, lse, idx, n_keep):
        ctx.cache_attend(0, 1, q, dev["K"], dev["V"], dev["ks"], dev["vs"], rows, 32, dev["cu"], n_tok, None, most, out, lse, dev["acc"], dev["acc"], 0.5, work)
        ctx.cache_evict(1, dev["acc"], rows, dev["cu"], n_tok, most, keep, 4, 100, idx, n_keep)
        ctx.cache_compact(1, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"], rows, 32, dev["cu"], idx, keep, n_keep, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"])

    mine, theirs = outputs(), outputs()
    s = torch.cuda.Stream()
    ctx.set_stream(s.cuda_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        calls(ctx, dev, *mine)
    for n in ([2000, 1999], [0, 1], [rows, rows - 1], [129, 3000], [0, 0], [32769, 500]):
        n_tok.copy_(i32([n]))
        q.copy_(torch.from_numpy(rng.standard_normal(tuple(q.shape))))
        for x in start:
            dev[x].copy_(start[x])
            eager[x].copy_(start[x])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        calls(direct, eager, *theirs)
        assert all(torch.equal(a, b) for a, b in zip(mine, theirs)) and all(torch.equal(dev[x], eager[x]) for x in dev)
        check_attend(ref, 0, q, [n], f64(mine[0]), f64(mine[1]))
        assert mine[3].flatten().tolist() == [min(x, keep) for x in n]


def test_selected_rows_and_a_resident_window_meet():
    """skv_select's list over the 8-bit cache, a window over skv_attend, joined by skv_merge_lse: attention over the union."""
    H, G, T, S, W, budget = 2, 4, 640, 40, 50, 200
    ctx = skv.Context(skv.Desc(n_layers=1, n_q_heads=H * G, n_kv_heads=H, kv_dtype=skv.SKV_BF16, max_tokens=T, max_sentences=S, max_budget=budget, max_batch=1))
    rng = np.random.RandomState(0)
    ref = filled([0, T], 1, H, 64, rng)
    ref.scale[0] = 2.0 ** -7
    dev = device_cache(ref)
    q = torch.from_numpy(rng.standard_normal((1, H * G, D))).bfloat16().to(DEV)
    score = torch.from_numpy(rng.standard_normal((H, S))).float().to(DEV)
    idx = torch.full((1, H, budget), -1, dtype=torch.int32, device=DEV)
    n, sel, n_sel = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((1, H), (H, S), (H,)))
    ctx.select(score, i32(np.arange(S + 1) * 16), i32([16] * S), S, budget, sel, n_sel, idx, n)
    out, lse = torch.zeros(1, H * G, D, device=DEV), torch.zeros(1, H * G, device=DEV)
    work = torch.empty(ctx.cache_attend_work_bytes(1, budget), dtype=torch.uint8, device=DEV)
    ctx.cache_attend(0, 1, q, dev["K"], dev["V"], dev["ks"], dev["vs"], T, 64, dev["cu"], n, idx, budget, out, lse, None, None, 1.0, work)
    check_attend(ref, 0, q, n.cpu().numpy(), f64(out), f64(lse), idx.cpu().numpy())
    Kw, Vw = (torch.from_numpy(rng.standard_normal((H, W, D))).bfloat16().to(DEV) for _ in range(2))
    ow, lw, o, l = torch.zeros(H * G, D, device=DEV), torch.zeros(H * G, device=DEV), torch.zeros(H * G, D, device=DEV), torch.zeros(H * G, device=DEV)
    ctx.attend(q[0], Kw, Vw, i32([W] * H), W, ow, lw)
    ctx.merge_lse(H * G, out, lse, ow, lw, o, l)
    for h in range(H):
        rows = idx[0, h, : int(n[0, h])].cpu().numpy()
        K, V = (np.concatenate([ref.rows(kv, 0, h, 0, rows), f64(w[h])]) for kv, w in ((0, Kw), (1, Vw)))
        want, wl, p, _ = R.attend(f64(q)[0, h * G:(h + 1) * G], K, V)
        # skv_attend rounds its weights to bf16: half a step each
        size = np.stack([(p[g][:, None] * np.abs(V)).sum(0) for g in range(G)])
        assert np.all(np.abs(f64(o)[h * G:(h + 1) * G] - want) <= 2 * 2.0 ** -8 * size) and np.all(np.abs(f64(l)[h * G:(h + 1) * G] - wl) <= 2 * 2.0 ** -8)


def test_a_cache_beyond_32_bits_of_bytes():
    """Rows past 2^31 and 2^32 bytes of the pool are read and written at their own places."""
    T, H, block = (1 << 25) + 777, 2, 128                  # 4.3 GB a head
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    ctx = skv.Context(skv.Desc(n_layers=1, n_q_heads=H, n_kv_heads=H, kv_dtype=skv.SKV_BF16, max_tokens=T, max_batch=2))
    K, V = (torch.zeros(1, H, T, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.ones(1, H, T // block + 2, device=DEV) for _ in range(2))
    acc = torch.zeros(1, H, T, device=DEV)
    first = T - 700
    cu, n_tok = i32([0, first, T]), i32([[T - 800, 5], [300, 10]])
    rng = np.random.RandomState(0)
    k, v = (torch.from_numpy(rng.standard_normal((400, H, D))).bfloat16().to(DEV) for _ in range(2))
    ctx.cache_append(0, 2, k, v, 400, i32([0, 0, 400]), 400, cu, i32([[0, 0], [0, 0]]), K, V, ks, vs, T, block, acc)
    part = R.Cache([0, 700], 1, H, block)
    for h in range(H):
        part.append(0, 0, h, 0, k[:, h].cpu().double().numpy(), v[:, h].cpu().double().numpy())
    assert same_codes(K[0, :, first: first + 400].cpu().numpy(), part.codes[0, 0, :, :400]) and same_codes(V[0, :, first: first + 400].cpu().numpy(), part.codes[1, 0, :, :400])
    assert int(K[0, 0, :first].max()) == 0 and int(K[0, 1, :first].max()) == 0
    q = torch.from_numpy(rng.standard_normal((2, H, D))).bfloat16().to(DEV)
    out, lse = torch.zeros(2, H, D, device=DEV), torch.zeros(2, H, device=DEV)
    work = torch.empty(ctx.cache_attend_work_bytes(2, 400, True), dtype=torch.uint8, device=DEV)
    ctx.cache_attend(0, 2, q, K, V, ks, vs, T, block, cu, i32([[0, 0], [400, 390]]), None, 400, out, lse, acc, acc, 1.0, work)
    for h, m in ((0, 400), (1, 390)):
        want, wl, p, _ = R.attend(f64(q)[1, h:h + 1], part.rows(0, 0, h, 0, np.arange(m)), part.rows(1, 0, h, 0, np.arange(m)))
        assert np.abs(f64(out)[1, h] - want).max() <= 1e-4 and abs(f64(lse)[1, h] - wl[0]) <= 1e-4
        assert np.abs(f64(acc[0, h, first: first + m]) - p[0]).max() <= 1e-5
    idx, n_keep = torch.zeros(1, 2, H, 100, dtype=torch.int32, device=DEV), torch.zeros(1, 2, H, dtype=torch.int32, device=DEV)
    ctx.cache_evict(2, acc, T, cu, i32([[[0, 0], [400, 390]]]), 400, 100, 2, 10, idx, n_keep)
    part.acc[0, :, :700] = f64(acc[0, :, first:])
    for h, m in ((0, 400), (1, 390)):
        want = R.evict(part.acc[0, h, :m].astype(np.float32), 100, 2, 10)
        assert np.array_equal(idx[0, 1, h].cpu().numpy(), want)
        part.compact(0, 0, h, want)
    ctx.cache_compact(2, K, V, ks, vs, acc, T, block, cu, idx, 100, n_keep, K, V, ks, vs, acc)
    assert same_codes(K[0, :, first: first + 400].cpu().numpy(), part.codes[0, 0, :, :400]) and same_codes(V[0, :, first: first + 400].cpu().numpy(), part.codes[1, 0, :, :400])
    assert int(K[0, 0, :first].max()) == 0


def test_attend_of_one_long_sequence_among_more_pairs_than_take_shares():
    """Its rows lie in chunks that a 32-bit offset reaches.  All weights are alike, and two rows have values."""
    B, H, rows, block = 2049, 2, (1 << 25) + 999, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    T = rows + B - 1
    ctx = skv.Context(skv.Desc(n_layers=1, n_q_heads=H, n_kv_heads=H, kv_dtype=skv.SKV_BF16, max_tokens=T, max_batch=B))
    K, V = (torch.zeros(1, H, T, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.ones(1, H, T // block + B, device=DEV) for _ in range(2))
    V[0, 1, rows - 3, 5] = V[0, 1, 12, 6] = 0x7e                                  # 448
    cu = i32(np.concatenate([[0], rows + np.arange(B)]))
    n_tok = torch.ones(B, H, dtype=torch.int32, device=DEV)
    n_tok[0, 1] = rows
    q, out = torch.randn(B, H, D, device=DEV).bfloat16(), torch.full((B, H, D), 7.0, device=DEV)
    work = torch.empty(ctx.cache_attend_work_bytes(B, rows), dtype=torch.uint8, device=DEV)
    ctx.cache_attend(0, B, q, K, V, ks, vs, T, block, cu, n_tok, None, rows, out, None, None, None, 1.0, work)
    got, want = f64(out), np.zeros((B, H, D))
    want[0, 1, 5:7] = 448.0 / rows
    # a lane of a wave adds up its rows' weights of 1 one by one, exactly up to 2^24; then waves and parts
    assert np.all(np.abs(got - want) <= 400 * EPS * want)


def test_two_contexts_at_once():
    """Two streams, a context each: parts and their arrivals, shares, slices of an eviction and compactions in place side by side give what each gives alone."""
    H, G, most = 2, 4, 40000
    rng = np.random.RandomState(3)
    ref = filled([0, 30000, 70000], 1, H, 32, rng)
    ref.scale[0] = 2.0 ** -8
    q = torch.from_numpy(rng.standard_normal((2, H * G, D))).bfloat16().to(DEV)
    n = [i32([[30000, 5], [33000, 40000]]), i32([[700, 1], [1000, 999]])]

    def make(i, s):
        ctx, dev = context(H=H, G=G), device_cache(ref)
        if s is not None:
            ctx.set_stream(s.cuda_stream)
        work = torch.empty(ctx.cache_attend_work_bytes(2, most, True), dtype=torch.uint8, device=DEV)
        outs = [torch.zeros(2, H * G, D, device=DEV) for _ in range(3)]
        idx, n_keep = torch.zeros(1, 2, H, 600, dtype=torch.int32, device=DEV), torch.zeros(1, 2, H, dtype=torch.int32, device=DEV)

        def go():
            for out, bound, acc in zip(outs, (most, 1000, most), (None, None, dev["acc"])):
                ctx.cache_attend(0, 2, q, dev["K"], dev["V"], dev["ks"], dev["vs"], ref.T, 32, dev["cu"], n[i], None, bound, out, None, acc, acc, 0.5, work)
            ctx.cache_evict(2, dev["acc"], ref.T, dev["cu"], n[i], most, 600, 4, 100, idx, n_keep)
            ctx.cache_compact(2, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"], ref.T, 32, dev["cu"], idx, 600, n_keep, dev["K"], dev["V"], dev["ks"], dev["vs"], dev["acc"])
        return go, outs + [idx, n_keep] + list(dev.values())

    alone = [make(i, None) for i in range(2)]
    for go, _ in alone:
        for _ in range(5):
            go()
        torch.cuda.synchronize()
    both = [make(i, torch.cuda.Stream()) for i in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for go, _ in both:
            go()
    torch.cuda.synchronize()
    for (_, a), (_, b) in zip(alone, both):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_follow_the_contexts_stream():
    ctx = context(H=2, G=2)
    s = torch.cuda.Stream()
    ctx.set_stream(s.cuda_stream)
    x = torch.zeros(4096, 4, D, dtype=torch.bfloat16, device=DEV)
    y = torch.randn(4096, 4, D, device=DEV).bfloat16()
    pos, freq, out = torch.arange(4096, dtype=torch.int32, device=DEV), skv.rotary_freqs(128, 10000.0)[0].to(DEV), torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(50):
            x.copy_(x + 1)
        x.copy_(y)
        ctx.rotary(4096, x, None, pos, freq, 128, False, 1.0, out, None)
        got = out.clone()
    s.synchronize()
    ctx2 = context(H=2, G=2)
    want = torch.zeros_like(out)
    ctx2.rotary(4096, y, None, pos, freq, 128, False, 1.0, want, None)
    assert torch.equal(got, want)
