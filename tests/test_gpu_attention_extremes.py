"""The scored attentions at the ends of the ranges of their inputs, and key by key, against plain 64-bit forms."""
import pytest
import torch

import attention_reference as ref
from paper_2511_05534_amd import binding as fb
from test_gpu_prompt_attention import Prompt
from test_gpu_quantized_cache import DEV, DT, KINDS, Attention, params, stream

pytestmark = pytest.mark.gpu


def upload(a):
    """The rows and queries that a test has changed on the CPU, to the GPU."""
    a.qd.copy_(a.q.to(DEV))
    if a.rows != "fp8":
        a.dev[0].copy_(a.K.to(DEV))
        a.dev[1].copy_(a.V.to(DEV))
        return
    Kd, Vd = a.K.to(DEV), a.V.to(DEV)
    src = params(a.layers, a.hq, a.hkv, a.d, a.dtype, a.caps)
    fb.flowmm_cache_quantize(src, a.cu, a.caps, a.cu, Kd.data_ptr(), Vd.data_ptr(), a.cache, stream())
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows, dtype", KINDS)
@pytest.mark.parametrize("lens", [[90], [700, 130], [9000]])
@pytest.mark.parametrize("below", [1000.0, 60.0])
def test_large_values_that_weigh_little(rows, dtype, lens, below):
    """V near the type's largest number in rows whose logit is so far below the others' that their weight is 0, or exp(-60)."""
    a = Attention(rows, dtype, 1, 4, 2, 64, lens, scale=0.125, seed=15)
    a.q[:] = 0.0
    a.q[..., 0] = 8.0
    a.K[:] = 0.0
    for b, n in enumerate(lens):
        far = torch.arange(a.cu[b] + 5, a.cu[b] + n, 64)  # (one in a tile: the sum of a tile of them would leave fp32's range)
        a.K[:, :, far, 0] = -below
        a.V[:, :, far] = (3e38 * torch.tensor([1.0, -1.0, 0.5, 1.0]).repeat(len(far))[:len(far), None]).to(a.V.dtype)
    upload(a)
    a.run()
    a.check(f"{rows} {dtype} {lens} below {below}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 2000.0])
@pytest.mark.parametrize("L, hq", [(400, 1), (700, 40), (900, 140)])  # keys split over four waves, two, one
@pytest.mark.parametrize("below", [1000.0, 20.0])
def test_prompt_infinite_values_that_weigh_little(dtype, cap, L, hq, below):
    """An infinite value times its weight: infinite where the weight is small, undefined where it is 0, whichever way the row's blocks are taken."""
    a = Prompt(dtype, 1, hq, hq, 64, [L], cap=cap, scale=0.125, spans=[[(0, 20, 0), (20, L - 150, 1), (L - 150, L, 0)]], image_spans=True, seed=25)
    a.Q[:] = 0.0
    a.Q[..., 0] = 8.0
    a.K[:] = 0.0
    # key, channel, value, first row that sees it
    places = [(10, 1, float("inf"), 10), (25, 3, float("inf"), 20), (L // 2, 5, float("-inf"), 20), (L - 160, 7, float("nan"), 20), (L - 120, 9, float("inf"), L - 120),
              (L - 65, 11, float("-inf"), L - 65), (L - 2, 13, float("inf"), L - 2)]
    for row, ch, x, _ in places:
        a.V[0, :, row, ch] = x
        a.K[0, :, row, 0] = -below
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu().float()
    other = [c for c in range(64) if c not in [p[1] for p in places]]
    assert torch.isfinite(got[..., other]).all()
    for _, ch, x, first in places:
        o = got[0, :, :, ch]
        assert torch.isfinite(o[:, :first]).all(), ch
        assert (o[:, first:].isnan() if below > 100 or x != x else o[:, first:] == x).all(), (ch, x)


@pytest.fixture
def much_memory():
    """Memory that later tests do not find taken."""
    yield lambda gib: torch.cuda.mem_get_info()[0] >= gib << 30 or pytest.skip("not enough memory")
    torch.cuda.empty_cache()


def test_positions_of_more_than_two_to_the_thirty_rows(much_memory):
    """The bias of merged rows whose positions lie more than 4 GiB behind the first one's: the last rows alone are near the query."""
    d, n, near, q_pos = 64, (1 << 30) + 1000, 700, 1 << 29
    much_memory(80)
    p = params(1, 1, 1, d, "bf16", [n], [n])
    cu = [0, n]
    codes = torch.zeros((1, 1, n, d), dtype=torch.uint8, device=DEV)
    codes[0, 0, n - near:] = 0x38  # 1, in the rows near the query
    codes = codes.view(torch.float8_e4m3fn)
    scales = torch.ones((1, 1, -(-n // 32)), device=DEV)
    cache = fb.QuantizedCache(p, cu, tensors=[codes, codes, scales, scales])
    pos = torch.zeros(n, dtype=torch.int32, device=DEV)
    pos[n - near:] = q_pos
    slopes = torch.ones(1, device=DEV)
    q, out = torch.zeros((1, 1, 1, d), dtype=torch.bfloat16, device=DEV), torch.full((1, 1, 1, d), 9.0, dtype=torch.bfloat16, device=DEV)
    size = fb.flowmm_cache_sizes(p, cu)[2]
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    scoring = fb.Scoring(slopes=slopes.data_ptr(), row_pos=pos.data_ptr(), q_pos=[q_pos])
    fb.flowmm_cache_attention_quantized(p, cu, [n], scoring, q.data_ptr(), cache, out.data_ptr(), ws.data_ptr(), size, stream())
    assert (out == 1.0).all(), out


def test_a_sequence_of_nearly_two_to_the_thirty_one_rows(much_memory):
    """The longest sequence there is, in the most parts: its length and a part's do not add up to an int."""
    d, n, near = 64, (1 << 31) - 65537, 40
    much_memory(150)
    p = params(1, 1, 1, d, "bf16", [n])
    cu = [0, n]
    codes = torch.zeros((1, 1, n, d), dtype=torch.uint8, device=DEV)
    codes[0, 0, n - near:] = 0x38  # 1, in the rows near the query
    codes = codes.view(torch.float8_e4m3fn)
    scales = torch.ones((1, 1, -(-n // 32)), device=DEV)
    cache = fb.QuantizedCache(p, cu, tensors=[codes, codes, scales, scales])
    slopes = torch.full((1,), 4.0, device=DEV)
    q, out = torch.zeros((1, 1, 1, d), dtype=torch.bfloat16, device=DEV), torch.full((1, 1, 1, d), 9.0, dtype=torch.bfloat16, device=DEV)
    size = fb.flowmm_cache_sizes(p, cu)[2]
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    fb.flowmm_cache_attention_quantized(p, cu, [n], fb.Scoring(slopes=slopes.data_ptr()), q.data_ptr(), cache, out.data_ptr(), ws.data_ptr(), size, stream())
    assert (out == 1.0).all(), out  # the rows behind them weigh exp(-160) and less


def check_where_seen(a, got, q, K, V, hidden, dtype, weight_error, what):
    """One head's rows against the 64-bit form over the keys that are not hidden (whose logits are -infinity)."""
    want, tol = ref.attend(q, K.nan_to_num(0.0, 0.0, 0.0), V, a.scale, 0.0, None, None, hidden, DT[dtype], weight_error)
    ref.check(got, want, tol, what)


@pytest.mark.parametrize("rows, dtype", [k for k in KINDS if k[0] != "fp8"])
@pytest.mark.parametrize("lens", [[40, 50], [9000, 600]])  # whole, cut into parts
def test_logits_that_are_all_minus_infinity(rows, dtype, lens):
    """0 / 0 where every logit is -infinity; where some are not, the others weigh nothing, also where they are all that a workgroup sees."""
    a = Attention(rows, dtype, 1, 4, 2, 64, lens, seed=16)
    a.q[..., 0] = 1.0
    a.K[0, 0, :a.cu[1], 0] = float("-inf")                       # sequence 0, kv head 0: all
    a.K[0, 1, :lens[0] * 3 // 5, 0] = float("-inf")              # kv head 1: the first three fifths
    a.K[0, :, a.cu[1] + 5:a.cu[1] + lens[1], 0] = float("-inf")  # sequence 1: all but five
    upload(a)
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu()
    for b, n in enumerate(lens):
        r = slice(a.cu[b], a.cu[b] + n)
        for h in range(4):
            K = a.K[0, h // 2, r]
            check_where_seen(a, got[0, h, b][None], a.q[0, h, b][None], K, a.V[0, h // 2, r], K[:, 0].isinf()[None], dtype, 2.0 ** -15 if dtype == "bf16" else 0.0, (b, h))
    assert got[0, :2, 0].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L, hq", [(400, 1), (700, 40), (900, 140)])  # keys split over four waves, two, one
def test_prompt_logits_that_are_all_minus_infinity(dtype, L, hq):
    a = Prompt(dtype, 1, hq, hq, 64, [L], seed=26)
    a.Q[..., 0] = 1.0
    a.K[0, :, :L // 2 + 3, 0] = float("-inf")
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu()
    for h in (0, hq - 1):
        hidden = a.hidden(0) | a.K[0, h, :, 0].isinf()[None]
        check_where_seen(a, got[0, h], a.Q[0, h], a.K[0, h], a.V[0, h], hidden, dtype, 2.0 ** -8 if dtype == "bf16" else 0.0, h)
    assert got[0, :, :L // 2 + 3].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, hq, hkv, lens, window", [(128, 40, 1, [70], 1), (128, 34, 2, [33, 5], 1), (64, 64, 1, [129], 1), (128, 6, 2, [3, 20, 100], 64), (64, 4, 4, [40], 5000)])
def test_prompt_layouts_of_its_own(dtype, d, hq, hkv, lens, window):
    """More query heads to a kv head than the plan takes, and prompts shorter than its window."""
    a = Prompt(dtype, 2, hq, hkv, d, lens, cap=20.0, seed=27) if hq // hkv < 10 else None
    if a is None:  # (the workspace of such a layout is that of one query head to a kv head)
        one = Prompt(dtype, 2, hkv, hkv, d, lens, seed=27)
        a = Prompt.__new__(Prompt)
        a.__dict__.update(one.__dict__, hq=hq, scoring=None, cap=0.0)
        a.Q = torch.randn((2, hq, sum(lens), d), generator=torch.Generator().manual_seed(28)).to(DT[dtype])
        a.q_strides = (hq * sum(lens) * d, sum(lens) * d, d)
        a.upload()
    T = sum(lens)
    a.p = fb.Params(2, hq, hkv, d, dtype, lens, lens, a.spans, window, 0.25, [1.0] * len(lens), k_strides=(hkv * T * d, T * d, d))
    a.run()
    a.check(f"{dtype} {d} {hq}/{hkv} {lens} window {window}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k_size, q_size, v_size", [(1.0, 1.0, 2.0 ** -117), (2.0 ** -113, 2.0 ** 119, 1.0), (2.0 ** 100, 2.0 ** -100, 2.0 ** 118), (1.0, 1.0, 2.0 ** -60)])
def test_rows_in_8_bits_of_any_magnitude(dtype, k_size, q_size, v_size):
    """Blocks of tiny and of huge numbers: the logits and the outputs are those of rows of ordinary size, scaled."""
    lens = [300, 33]
    a = Attention("fp8", dtype, 1, 4, 2, 64, lens, scale=0.125 / (k_size * q_size), seed=17)
    a.q = (a.q.double() * q_size).to(a.q.dtype)
    a.K, a.V = ((x.double().clamp(-60, 60) * s).to(x.dtype) for x, s in ((a.K, k_size), (a.V, v_size)))
    upload(a)
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu()
    K, V = a.values()
    for b, n in enumerate(lens):
        r = slice(a.cu[b], a.cu[b] + n)
        for h in range(4):
            want, tol = ref.attend(a.q[0, h, b][None], K[0, h // 2, r], V[0, h // 2, r] / v_size, a.scale, 0.0, None, None, None, DT[dtype], 2.0 ** -15 if dtype == "bf16" else 0.0)
            ref.check(got[0, h, b][None].double() / v_size, want, tol, (b, h))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_in_8_bits_at_any_scale(dtype, d):
    """Scales that the library does not write: no powers of two, negative ones, 0, subnormal ones."""
    lens = [310, 64]
    a = Attention("fp8", dtype, 1, 4, 2, d, lens, scale=1.0, seed=18)
    g = torch.Generator().manual_seed(19)
    for scales, size in ((a.cache.k_scales, 2.0 ** -8), (a.cache.v_scales, 0.01)):
        some = torch.tensor([0.3712, -1.7, 0.0, 1.0, 1.99999, 1e-36, -1e-40, 0.75]) * size
        scales.copy_(some[torch.randint(0, len(some), scales.shape, generator=g)])
    for codes in (a.cache.k_codes, a.cache.v_codes):
        codes.view(torch.uint8).copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8) & 0xbf)  # (numbers of up to 1.875)
    a.run()
    a.check(f"{dtype} {d} any scale")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("below", [1000.0, 60.0])
def test_codes_that_stand_for_more_than_the_largest_float(dtype, below):
    """The largest numbers, which e4m3 rounds up to 2^128, in rows that weigh 0, or exp(-60)."""
    lens = [90, 700]
    a = Attention("fp8", dtype, 1, 4, 2, 64, lens, scale=0.125, seed=31)
    a.q[:] = 0.0
    a.q[..., 0] = 8.0
    a.K[:] = 0.0
    for b, n in enumerate(lens):
        far = torch.arange(a.cu[b] + 5, a.cu[b] + n, 64)
        a.K[:, :, far, 0] = -below
        a.V[:, :, far] = torch.finfo(a.V.dtype).max
    upload(a)
    a.run()
    assert float(a.cache.v_scales.max()) == 2.0 ** 120 and float(a.values()[1].max()) == 2.0 ** 128
    a.check(f"{dtype} below {below}")


def watched(units, L, d):
    """V in which channel c of unit g is 1 in row g * d + c alone: every row of L <= units * d has a channel of its own."""
    v = torch.zeros(units, L, d)
    r = torch.arange(L)
    v[r // d, r, r % d] = 1.0
    return v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq, hkv, L, masks", [(8, 8, 1000, False), (40, 8, 1000, False), (34, 17, 2100, False), (8, 8, 1000, True), (40, 8, 1000, True), (34, 17, 2100, True)])
def test_every_key_of_a_prompt_counts_once(dtype, hq, hkv, L, masks):
    """All keys weigh the same, so that every output is 1 / their number where the row sees the channel's key, and 0 where it does not."""
    d, G = 128, hq // hkv
    spans = [[(0, 100, 0), (100, 333, 1), (333, 700, 0), (700, 790, 1), (790, L, 0)]]
    a = Prompt(dtype, 1, hq, hkv, d, [L], spans=spans, prefix=[57] if masks else None, image_spans=masks, seed=29)
    a.Q[:] = 0.0
    a.V[0] = watched(hkv, L, d).to(DT[dtype])
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu().double()[0]
    seen = (~a.hidden(0)).double()
    want = seen / seen.sum(-1, keepdim=True)
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * 1.001 * want  # the result's rounding; fp32: that of 1 / z before it as well
    for h in range(hq):
        keys = slice(h // G * d, min(L, h // G * d + d))
        n = keys.stop - keys.start
        if n > 0:
            assert ((got[h, :, :n] - want[:, keys]).abs() <= tol[:, keys]).all(), h
            assert (got[h, :, n:] == 0).all()


@pytest.mark.parametrize("rows, dtype", KINDS)
@pytest.mark.parametrize("hkv, G, lens", [(8, 1, [1000]), (8, 3, [257, 31, 640]), (40, 2, [2500]), (64, 1, [1, 700, 16, 900, 33]), (16, 17, [1100, 5])])
def test_every_row_of_a_cache_counts_once(rows, dtype, hkv, G, lens):
    d = 64
    a = Attention(rows, dtype, 1, hkv * G, hkv, d, lens, seed=30)
    a.q[:] = 0.0
    a.V[:] = 0.0
    for b, n in enumerate(lens):
        m = min(n, hkv * d)
        a.V[0, :, a.cu[b]:a.cu[b] + m] = watched(hkv, m, d).to(DT[dtype])
    upload(a)
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu().double()[0]
    for b, n in enumerate(lens):
        there = (torch.arange(hkv * d) < n).double().view(hkv, d) / n
        want = there.repeat_interleave(G, 0)
        # the result's rounding; fp32: that of the quotient and, beside codes, of none of the terms (weights are 1)
        assert ((got[:, b] - want).abs() <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * 1.001 * want).all(), b


@pytest.mark.parametrize("dtype, layers, hq, hkv, L", [("bf16", 1, 36, 36, 2100), ("bf16", 1, 72, 72, 2100), ("bf16", 10, 16, 8, 1500), ("f32", 4, 17, 17, 3700), ("bf16", 9, 10, 10, 40)])
def test_units_in_groups(dtype, layers, hq, hkv, L):
    """More (layer, kv head) units than a group takes, in numbers that do not divide: every row of every head, the mean of what it sees."""
    a = Prompt(dtype, layers, hq, hkv, 64, [L], seed=32)
    a.Q[:] = 0.0
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got, seen = a.out.double(), torch.arange(1, L + 1, dtype=torch.float64, device=DEV)[:, None]
    V = a.dev[1].double().repeat_interleave(hq // hkv, 1)
    want, size = V.cumsum(2) / seen, V.abs().cumsum(2) / seen
    # the result's rounding and the sum's (weights are 1: exact)
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * want.abs() + L * 2.0 ** -24 * size
    assert ((got - want).abs() <= tol).all()
