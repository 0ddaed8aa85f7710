"""The cache in 8 bits and the attention over a cache with head room, against plain 64-bit forms."""
import pytest
import torch

import attention_reference as ref
from paper_2511_05534_amd import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def stream():
    return torch.cuda.current_stream().cuda_stream


def params(layers, hq, hkv, d, dtype, caps, budgets=None, **kw):
    return fb.Params(layers, hq, hkv, d, dtype, caps, budgets or caps, [[(0, c, 0)] for c in caps], 1, 0.25, [1.0] * len(caps), **kw)


def sums(x):
    out = [0]
    for n in x:
        out.append(out[-1] + n)
    return out


def blocks_of(caps):
    return [-(-c // 32) for c in caps]


def rows_like_a_cache(shape, dtype, seed):
    """N(0,1) rows, some eight times as long, on the CPU."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    gain = torch.where(torch.rand(shape[:-1], generator=g) < 0.05, 8.0, 1.0)
    return (x * gain[..., None]).to(dtype)


def codes_as_numbers(t):
    return t.cpu().to(torch.float64)


# ---- rows into 8 bits and back -----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens, room", [([1], 0), ([31, 32, 33], 5), ([100, 0, 7, 64], 40), ([0], 3), ([5] * 70, 2)])
def test_quantize_and_back(dtype, d, lens, room):
    layers, hkv = 2, 3
    caps = [n + room if n + room else 1 for n in lens]
    cu, cb = sums(caps), sums(blocks_of(caps))
    starts = [s + 3 for s in sums(lens)[:-1]]  # the rows lie densely, three tokens in
    T = sum(lens) + 4
    p = params(layers, hkv, hkv, d, dtype, caps, k_strides=(hkv * T * d, T * d, d))
    K, V = (rows_like_a_cache((layers, hkv, T, d), DT[dtype], s) for s in (1, 2))
    marked = [torch.full((layers, hkv, cu[-1], d), 0x2a, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2)]
    marked += [torch.full((layers, hkv, cb[-1]), 7.0, device=DEV) for _ in range(2)]
    cache = fb.QuantizedCache(p, cu, tensors=marked)
    Kd, Vd = K.to(DEV), V.to(DEV)
    fb.flowmm_cache_quantize(p, cu, lens, starts, Kd.data_ptr(), Vd.data_ptr(), cache, stream())
    back = [torch.full_like(Kd, 5.0), torch.full_like(Vd, 5.0)]
    fb.flowmm_cache_dequantize(p, cu, lens, starts, cache, back[0].data_ptr(), back[1].data_ptr(), stream())
    torch.cuda.synchronize()
    for x, codes, scales, y in ((K, cache.k_codes, cache.k_scales, back[0].cpu()), (V, cache.v_codes, cache.v_scales, back[1].cpu())):
        codes, raw, scales = codes_as_numbers(codes), codes.view(torch.uint8).cpu(), scales.cpu()
        touched, seen = torch.zeros(cu[-1], dtype=torch.bool), torch.zeros(T, dtype=torch.bool)
        touched_blocks = torch.zeros(cb[-1], dtype=torch.bool)
        for b, n in enumerate(lens):
            touched[cu[b]:cu[b] + n] = True
            seen[starts[b]:starts[b] + n] = True
            for j in range(-(-n // 32)):
                touched_blocks[cb[b] + j] = True
                r0, r1 = 32 * j, min(n, 32 * j + 32)
                for l in range(layers):
                    for g in range(hkv):
                        want, scale = ref.quantize_block(x[l, g, starts[b] + r0:starts[b] + r1])
                        assert float(scales[l, g, cb[b] + j]) == scale
                        assert torch.equal(codes[l, g, cu[b] + r0:cu[b] + r1], want)
                        assert torch.equal(y[l, g, starts[b] + r0:starts[b] + r1], (want * scale).to(DT[dtype]))
        assert (raw[:, :, ~touched] == 0x2a).all() and (scales[:, :, ~touched_blocks] == 7.0).all()
        assert (y[:, :, ~seen] == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_extremes(dtype):
    """Infinities, NaN, zeros of either sign, subnormals, the largest numbers, numbers next to the steps, each in a block of its own."""
    d, n = 64, 32
    big = torch.finfo(DT[dtype]).max
    blocks = [torch.zeros(n, d), torch.full((n, d), -0.0), torch.full((n, d), float("inf")), torch.full((n, d), float("nan")),
              torch.full((n, d), big), torch.full((n, d), 1e-40), torch.linspace(-448, 448, n * d).view(n, d),
              torch.full((n, d), 448.0), torch.full((n, d), 450.0), torch.full((n, d), 2.0 ** -130)]
    mixed = torch.linspace(-3, 3, n * d).view(n, d).clone()
    mixed[0, 0], mixed[5, 7], mixed[31, 63] = float("inf"), float("-inf"), float("nan")
    # every tie between neighbouring codes: (m + 1/2) steps at every exponent
    ties = torch.tensor([(m + 0.5) / 8 * 2.0 ** e * s for e in range(-6, 9) for m in range(8, 16) for s in (1, -1)] + [(m + 0.5) * 2.0 ** -9 for m in range(8)])
    tie = torch.zeros(n * d)
    tie[:ties.numel()] = ties.clamp(-448, 448)
    tie[-1] = 448.0
    blocks += [mixed, tie.view(n, d)]
    x = torch.cat(blocks).to(DT[dtype])[None, None]
    N = x.shape[2]
    p = params(1, 1, 1, d, dtype, [N])
    cache = fb.QuantizedCache(p, [0, N], DEV)
    xd = x.to(DEV)
    back = [torch.empty_like(xd) for _ in range(2)]
    fb.flowmm_cache_quantize(p, [0, N], [N], [0], xd.data_ptr(), xd.data_ptr(), cache, stream())
    fb.flowmm_cache_dequantize(p, [0, N], [N], [0], cache, back[0].data_ptr(), back[1].data_ptr(), stream())
    codes, scales = codes_as_numbers(cache.k_codes)[0, 0], cache.k_scales.cpu()[0, 0]
    for j in range(N // n):
        want, scale = ref.quantize_block(x[0, 0, n * j:n * j + n])
        assert float(scales[j]) == scale, j
        assert torch.equal(codes[n * j:n * j + n].nan_to_num(999.0), want.nan_to_num(999.0)), j
        assert torch.equal(back[0].cpu()[0, 0, n * j:n * j + n].nan_to_num(999.0), (want * scale).to(DT[dtype]).nan_to_num(999.0)), j
    assert torch.equal(cache.v_codes.view(torch.uint8), cache.k_codes.view(torch.uint8))


def test_dequantize_every_code_at_any_scale():
    d = 64
    codes = torch.arange(256, dtype=torch.uint8).repeat(16).view(64, d)
    for dtype in ("bf16", "f32"):
        p = params(1, 1, 1, d, dtype, [64])
        cache = fb.QuantizedCache(p, [0, 64], DEV)
        for t in (cache.k_codes, cache.v_codes):
            t.view(torch.uint8).copy_(codes.to(DEV)[None, None])
        scales = torch.tensor([[[0.3712, 2.0 ** -30]]])
        cache.k_scales.copy_(scales)
        cache.v_scales.copy_(scales)
        out = [torch.empty((1, 1, 64, d), dtype=DT[dtype], device=DEV) for _ in range(2)]
        fb.flowmm_cache_dequantize(p, [0, 64], [64], [0], cache, out[0].data_ptr(), out[1].data_ptr(), stream())
        want = codes.view(torch.float8_e4m3fn).float() * scales[0, 0].repeat_interleave(32)[:, None]
        for o in out:
            assert torch.equal(o.cpu()[0, 0].nan_to_num(999.0), want.to(DT[dtype]).nan_to_num(999.0))


# ---- append ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, batch", [(128, 3), (64, 9), (128, 66)])
def test_append_step_by_step(dtype, d, batch):
    """From empty caches over block borders; rows of growing and falling size, so that scales are raised, kept and set anew."""
    layers, hkv, steps = 1, 2, 70 if batch < 60 else 5
    caps = [steps + (b % 3) for b in range(batch)]
    cu, cb = sums(caps), sums(blocks_of(caps))
    p = params(layers, hkv, hkv, d, dtype, caps)
    cache = fb.QuantizedCache(p, cu, DEV)
    cache.k_codes.view(torch.uint8).fill_(0x31)
    cache.v_codes.view(torch.uint8).fill_(0x31)
    g = torch.Generator().manual_seed(d + batch)
    news = []
    for i in range(steps):
        size = 2.0 ** ((i * 7) % 11 - 5)
        new = [(torch.randn((layers, hkv, batch, d), generator=g) * size).to(DT[dtype]) for _ in range(2)]
        if i == 40:
            new[0][:] = 0.0
        if i == 41:
            new[0][0, 0, 0, 3], new[1][0, 1, 1, 5] = float("inf"), float("nan")
        news.append(new)
        kd, vd = (x.to(DEV) for x in new)
        fb.flowmm_cache_append_quantized(p, cu, [i] * batch, cache, kd.data_ptr(), vd.data_ptr(), stream())
    torch.cuda.synchronize()
    for t, (codes, scales) in enumerate(((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales))):
        raw, codes, scales = codes.view(torch.uint8).cpu(), codes_as_numbers(codes), scales.cpu()
        for b in range(batch):
            for h in range(hkv):
                block, scale = torch.zeros(32, d, dtype=torch.float64), 1.0
                for i in range(steps):
                    block, scale = ref.append_row(block, scale, news[i][t][0, h, b], i % 32)
                    if i % 32 == 31 or i == steps - 1:
                        at = cu[b] + i // 32 * 32
                        assert float(scales[0, h, cb[b] + i // 32]) == scale, (b, h, i)
                        assert torch.equal(codes[0, h, at:at + i % 32 + 1].nan_to_num(999.0), block[:i % 32 + 1].nan_to_num(999.0)), (b, h, i)
            assert (raw[:, :, cu[b] + steps:cu[b + 1]] == 0x31).all()


def test_append_to_any_scale():
    """A block whose scale is no power of two: a row within it is divided by it, a larger one brings its own power of two."""
    d = 64
    p = params(1, 1, 1, d, "f32", [32])
    cache = fb.QuantizedCache(p, [0, 32], DEV)
    old = torch.linspace(-440, 440, 3 * d).view(3, d).to(torch.float8_e4m3fn)
    small, large = torch.linspace(-100, 100, d), torch.linspace(-1000, 1000, d)
    for row, keeps in ((small, True), (large, False)):
        for t, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
            t.view(torch.uint8)[0, 0, :3] = old.view(torch.uint8).to(DEV)
            s.fill_(0.37)
        new = row.to(DEV)[None, None, None].contiguous()
        fb.flowmm_cache_append_quantized(p, [0, 32], [3], cache, new.data_ptr(), new.data_ptr(), stream())
        had = float(torch.tensor(0.37))
        scale = had if keeps else ref.e4m3_scale(1000.0)
        assert float(cache.k_scales.cpu()) == scale
        want = old if keeps else (old.float() * (torch.tensor(had) / scale)).to(torch.float8_e4m3fn)
        got = cache.k_codes.cpu()[0, 0]
        assert torch.equal(got[:3].float(), want.float())
        assert torch.equal(got[3].float(), (row / torch.tensor(scale)).to(torch.float8_e4m3fn).float())


# ---- attention over a cache --------------------------------------------------------------------------------
class Attention:
    """One call: inputs on the CPU and on the GPU, its reference."""

    def __init__(self, rows, dtype, layers, hq, hkv, d, lens, room=7, cap=0.0, slopes=False, merged=None, seed=0, pad=0, scale=0.0):
        self.rows, self.dtype, self.lens, self.cap = rows, dtype, lens, cap
        self.layers, self.hq, self.hkv, self.d = layers, hq, hkv, d
        self.caps = [max(1, n + room) for n in lens]
        self.cu, self.cb, C = sums(self.caps), sums(blocks_of(self.caps)), sum(self.caps)
        dt = DT[dtype]
        self.scale = scale or d ** -0.5
        self.K, self.V = rows_like_a_cache((layers, hkv, C, d), dt, seed + 1), rows_like_a_cache((layers, hkv, C, d), dt, seed + 2)
        self.q = torch.randn((layers, hq, len(lens), d), generator=torch.Generator().manual_seed(seed + 3)).to(dt)
        self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]) if slopes else None
        self.merged = merged
        strides = (hkv * C * (d + pad), C * (d + pad), d + pad)
        self.p = params(layers, hq, hkv, d, dtype, self.caps, merged, k_strides=strides, scale=scale)
        self.far = []
        if merged:
            g = torch.Generator().manual_seed(seed + 4)
            self.slots = sums(merged)
            self.row_pos = torch.cumsum(torch.randint(1, 6, (layers, hkv, self.slots[-1]), generator=g, dtype=torch.int32), -1, dtype=torch.int32)
            self.q_pos = [int(self.row_pos[:, :, self.slots[b]:self.slots[b + 1]].max()) + max(0, n - m) for b, (n, m) in enumerate(zip(lens, merged))]
        if rows == "fp8":
            self.cache = fb.QuantizedCache(self.p, self.cu, DEV)
            if pad:  # codes with a token stride of their own
                wide = [torch.zeros((layers, hkv, C, d + pad), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)[..., :d] for _ in range(2)]
                self.cache = fb.QuantizedCache(self.p, self.cu, tensors=[*wide, self.cache.k_scales, self.cache.v_scales])
            src = params(layers, hq, hkv, d, dtype, self.caps)
            Kd, Vd = self.K.to(DEV), self.V.to(DEV)
            fb.flowmm_cache_quantize(src, self.cu, self.caps, self.cu, Kd.data_ptr(), Vd.data_ptr(), self.cache, stream())
            torch.cuda.synchronize()
        else:
            wide = torch.zeros((2, layers, hkv, C, d + pad), dtype=dt)
            wide[0, ..., :d], wide[1, ..., :d] = self.K, self.V
            self.dev = wide.to(DEV)
        self.workspace_bytes = fb.flowmm_cache_sizes(self.p, self.cu)[2]
        self.workspace = torch.empty(max(256, self.workspace_bytes), dtype=torch.uint8, device=DEV)
        self.qd = self.q.to(DEV)
        self.out = torch.full_like(self.qd, 77.0)
        sl = self.slopes.to(DEV) if slopes else None
        rp = self.row_pos.to(DEV) if merged else None
        self.keep = (sl, rp)
        self.scoring = None
        if cap or slopes or merged:
            self.scoring = fb.Scoring(cap=cap, slopes=sl.data_ptr() if slopes else 0, row_pos=rp.data_ptr() if merged else 0, q_pos=self.q_pos if merged else None)

    def run(self, on=None):
        on = stream() if on is None else on
        rest = (self.out.data_ptr(), self.workspace.data_ptr(), self.workspace_bytes, on)
        if self.rows == "fp8":
            fb.flowmm_cache_attention_quantized(self.p, self.cu, self.lens, self.scoring, self.qd.data_ptr(), self.cache, *rest)
        else:
            fb.flowmm_cache_attention(self.p, self.cu, self.lens, self.scoring, self.qd.data_ptr(), self.dev[0].data_ptr(), self.dev[1].data_ptr(), *rest)
        return self.out

    def values(self):
        """K, V as the call sees them."""
        if self.rows != "fp8":
            return self.K, self.V
        got = []
        for codes, scales in ((self.cache.k_codes, self.cache.k_scales), (self.cache.v_codes, self.cache.v_scales)):
            x, s = codes_as_numbers(codes), scales.cpu().double()
            for b, c in enumerate(self.caps):
                x[:, :, self.cu[b]:self.cu[b] + c] *= s[:, :, self.cb[b]:self.cb[b + 1]].repeat_interleave(32, -1)[:, :, :c, None]
            got.append(x)
        return got

    def check(self, what=""):
        torch.cuda.synchronize()
        got = self.out.cpu()
        K, V = self.values()
        G, worst = self.hq // self.hkv, 0.0
        for b, n in enumerate(self.lens):
            if n == 0:
                assert (got[:, :, b] == 0).all(), what
                continue
            r = slice(self.cu[b], self.cu[b] + n)
            far = (n - 1 - torch.arange(n)).double()
            for l in range(self.layers):
                for h in range(self.hq):
                    g = h // G
                    if self.merged:
                        m = min(n, self.merged[b])
                        far = (n - 1 - torch.arange(n)).double()
                        far[:m] = (self.q_pos[b] - self.row_pos[l, g, self.slots[b]:self.slots[b] + m]).double().abs()
                    want, tol = ref.attend(self.q[l, h, b][None], K[l, g, r], V[l, g, r], self.scale, self.cap, None if self.slopes is None else float(self.slopes[h]),
                                           far[None], None, DT[self.dtype], 2.0 ** -15 if self.dtype == "bf16" else 0.0)
                    worst = max(worst, ref.check(got[l, h, b][None], want, tol, (what, b, l, h)))
        print(f"{what} of the tolerance: {worst:.3f}", flush=True)


KINDS = [("bf16", "bf16"), ("f32", "f32"), ("fp8", "bf16"), ("fp8", "f32")]


@pytest.mark.parametrize("rows, dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq, hkv, lens", [(3, 3, [1, 2, 15, 16, 17, 31, 32, 33]), (14, 2, [0, 130, 0, 257]), (16, 1, [700]), (17, 1, [5, 300]), (40, 1, [64])])
def test_attention_lengths_and_heads(rows, dtype, d, hq, hkv, lens):
    a = Attention(rows, dtype, 2, hq, hkv, d, lens, seed=hq)
    a.run()
    a.check(f"{rows} {dtype} {d} {hq}/{hkv} {lens}")


@pytest.mark.parametrize("rows, dtype", KINDS)
@pytest.mark.parametrize("cap, slopes, positions", [(20.0, False, False), (0.0, True, False), (0.0, True, True), (3.0, True, True), (5.0, False, True)])
def test_attention_scores(rows, dtype, cap, slopes, positions):
    lens = [9, 450, 40, 33]
    a = Attention(rows, dtype, 2, 8, 2, 128, lens, cap=cap, slopes=slopes, merged=[5, 400, 40, 36] if positions else None, seed=5)
    a.run()
    a.check(f"{rows} {dtype} cap {cap} slopes {slopes} positions {positions}")


@pytest.mark.parametrize("rows, dtype", KINDS)
@pytest.mark.parametrize("cap", [0.5, 512.0, 513.0, 1e5, 1e30])
def test_attention_caps_of_any_size(rows, dtype, cap):
    """Caps far above the logits leave them as they are, small ones flatten them."""
    a = Attention(rows, dtype, 1, 4, 2, 64, [70, 33], cap=cap, seed=14)
    a.run()
    a.check(f"{rows} {dtype} cap {cap}")


@pytest.mark.parametrize("rows, dtype", KINDS)
def test_attention_long_sequences_in_parts(rows, dtype):
    """One unit and a long sequence: many workgroups and the fold; beside it a short one and an empty one."""
    a = Attention(rows, dtype, 1, 4, 1, 128, [9001, 3, 0], cap=30.0, slopes=True, seed=6)
    a.run()
    a.check(f"{rows} {dtype} parts")
    first = a.out.clone()
    a.out.fill_(3.0)
    a.workspace.fill_(0xff)
    a.run()
    assert torch.equal(a.out, first)  # nothing depends on what the workspace held, nor on the order of the workgroups


@pytest.mark.parametrize("rows, dtype", KINDS)
@pytest.mark.parametrize("layers, hkv, G, d, lens", [
    (8, 8, 1, 128, [0, 700, 30, 1500, 0, 90]),    # unequal sequences' order, empty ones in it
    (16, 16, 1, 64, [0, 600, 5, 300, 33]),        # .. with units whose tasks go one after the other
    (2, 1, 20, 128, [5000, 1]),                   # more heads than one pass takes, in parts
    (8, 8, 1, 64, [60, 1, 31, 64, 50]), (16, 16, 1, 64, [100, 3]), (16, 16, 2, 128, [400, 37]),  # fewer waves
])
def test_attention_schedules(rows, dtype, layers, hkv, G, d, lens):
    a = Attention(rows, dtype, layers, hkv * G, hkv, d, lens, slopes=True, merged=[max(1, n // 2) for n in lens], seed=21)
    a.run()
    a.check(f"{rows} {dtype} {layers} x {hkv} {lens}")


def test_two_streams_with_workspaces_of_their_own():
    """Two calls at once, on caches of their own."""
    a, b = (Attention("fp8", "bf16", 1, 4, 1, 128, [6000, 10], cap=20.0, seed=s) for s in (30, 31))
    for x in (a, b):
        x.run()
    torch.cuda.synchronize()
    want = [x.out.clone() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for x in (a, b):
        x.out.fill_(0)
    torch.cuda.synchronize()
    for _ in range(5):
        for x, st in zip((a, b), streams):
            x.run(st.cuda_stream)
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        assert torch.equal(x.out, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_in_a_graph(dtype):
    """Quantize, append and dequantize captured together: every replay starts from the same rows and ends with the same codes."""
    layers, hkv, d, lens, caps = 2, 2, 64, [40, 7, 0], [64, 32, 33]
    cu, cb = sums(caps), sums(blocks_of(caps))
    p = params(layers, hkv, hkv, d, dtype, caps)
    K, V = (rows_like_a_cache((layers, hkv, cu[-1], d), DT[dtype], s).to(DEV) for s in (40, 41))
    k, v = (100 * rows_like_a_cache((layers, hkv, 3, d), DT[dtype], s).to(DEV) for s in (42, 43))
    cache = fb.QuantizedCache(p, cu, DEV)
    back = [torch.zeros_like(K) for _ in range(2)]

    def run():
        st = stream()
        fb.flowmm_cache_quantize(p, cu, lens, cu, K.data_ptr(), V.data_ptr(), cache, st)
        fb.flowmm_cache_append_quantized(p, cu, lens, cache, k.data_ptr(), v.data_ptr(), st)
        fb.flowmm_cache_dequantize(p, cu, [n + 1 for n in lens], cu, cache, back[0].data_ptr(), back[1].data_ptr(), st)

    run()
    torch.cuda.synchronize()
    want = [t.view(torch.uint8).clone() for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, *back)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, *back):
            t.view(torch.uint8).zero_()
        torch.randn(1 << 20, device=DEV).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, *back), want):
            assert torch.equal(t.view(torch.uint8), w)


@pytest.mark.parametrize("rows, dtype", KINDS)
def test_attention_of_many_sequences(rows, dtype):
    """More sequences than one launch takes, positions among them."""
    lens = [(7 * b) % 50 for b in range(70)]
    a = Attention(rows, dtype, 1, 2, 2, 64, lens, slopes=True, merged=[max(1, n // 2) for n in lens], seed=8)
    a.run()
    a.check(f"{rows} {dtype} many")


@pytest.mark.parametrize("rows, dtype", KINDS)
def test_attention_reads_nothing_behind_the_rows(rows, dtype):
    """NaN and infinities in every row behind the valid ones, and a scale of NaN for the blocks behind them."""
    lens = [1, 40, 300, 0]
    a = Attention(rows, dtype, 1, 4, 2, 64, lens, room=70, seed=9)
    dirty = torch.ones(a.cu[-1], dtype=torch.bool)
    for b, n in enumerate(lens):
        dirty[a.cu[b]:a.cu[b] + n] = False
    dirty = dirty.to(DEV)
    if rows == "fp8":
        a.cache.k_codes.view(torch.uint8)[:, :, dirty] = 0x7f
        a.cache.v_codes.view(torch.uint8)[:, :, dirty] = 0xff
        for s in (a.cache.k_scales, a.cache.v_scales):
            for b, n in enumerate(lens):
                s[:, :, a.cb[b] + -(-n // 32):a.cb[b + 1]] = float("nan")
    else:
        a.dev[0][:, :, dirty] = float("nan")
        a.dev[1][:, :, dirty] = float("inf")
    a.run()
    K, V = a.values()
    a.values = lambda: (K.nan_to_num(0.0, 0.0, 0.0), V.nan_to_num(0.0, 0.0, 0.0)) if rows == "fp8" else (a.K, a.V)
    a.check(f"{rows} {dtype} dirty")


@pytest.mark.parametrize("rows, dtype", [("bf16", "bf16"), ("f32", "f32")])
def test_attention_infinite_values(rows, dtype):
    """An infinite value in a row makes its channel infinite, in the last row too, whose tile reads it again for the rows that are not there."""
    a = Attention(rows, dtype, 1, 4, 2, 64, [21, 35], seed=10)
    a.V[0, 0, a.cu[0] + 20, 5] = float("inf")
    a.V[0, 1, a.cu[1] + 3, 7] = float("-inf")
    a.V[0, 1, a.cu[1] + 34, 9] = float("nan")
    a.dev[1].copy_(a.V.to(DEV))
    a.run()
    a.check(f"{rows} {dtype} infinite")


@pytest.mark.parametrize("rows, dtype", KINDS)
def test_attention_strides_and_scale(rows, dtype):
    a = Attention(rows, dtype, 2, 6, 3, 64, [50, 90], pad=16, scale=0.3, seed=11)
    a.run()
    a.check(f"{rows} {dtype} strides")


@pytest.mark.parametrize("rows, dtype", KINDS)
def test_attention_beyond_32_bit_offsets(rows, dtype):
    """Rows a megabyte apart: the sequence's last ones lie more than 4 GiB behind its first."""
    d, n, stride = 64, 4400, 1 << 20
    es = 1 if rows == "fp8" else 2 if rows == "bf16" else 4
    a = Attention(rows, dtype, 1, 2, 1, d, [n], room=0, seed=12)
    far = torch.empty(n * stride, dtype=torch.uint8, device=DEV)
    at = (torch.arange(n, device=DEV) * stride)[:, None] + torch.arange(2 * d * es, device=DEV)[None, :]
    if rows == "fp8":
        both = torch.cat([a.cache.k_codes[0, 0].view(torch.uint8), a.cache.v_codes[0, 0].view(torch.uint8)], -1)
    else:
        both = torch.cat([a.dev[0][0, 0].view(torch.uint8), a.dev[1][0, 0].view(torch.uint8)], -1)
    far[at.reshape(-1)] = both.reshape(-1)
    if rows == "fp8":
        a.cache.c.k_codes, a.cache.c.v_codes, a.cache.c.stride_token = far.data_ptr(), far.data_ptr() + d, stride
        a.run()
    else:
        p = params(1, 2, 1, d, dtype, [n], k_strides=(0, 0, stride // es))
        fb.flowmm_cache_attention(p, a.cu, a.lens, None, a.qd.data_ptr(), far.data_ptr(), far.data_ptr() + d * es, a.out.data_ptr(), a.workspace.data_ptr(),
                                  a.workspace_bytes, stream())
    a.check(f"{rows} {dtype} far")


@pytest.mark.parametrize("rows, dtype", KINDS)
def test_attention_in_a_graph_and_on_another_stream(rows, dtype):
    a = Attention(rows, dtype, 1, 8, 2, 128, [2000, 77], cap=10.0, slopes=True, merged=[1500, 60], seed=13)
    a.run()
    torch.cuda.synchronize()
    want = a.out.clone()
    side = torch.cuda.Stream()
    a.out.fill_(1.0)
    side.wait_stream(torch.cuda.current_stream())
    a.run(side.cuda_stream)
    side.synchronize()
    assert torch.equal(a.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for _ in range(3):
        a.out.fill_(2.0)
        torch.randn(1 << 20, device=DEV).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want)


def test_a_growing_conversation():
    """The calls as a serving program makes them: merge the prompt, hold the cache in 8 bits, append and attend token by token, and, when it is
    full, bring one sequence back, re-merge it and hold it in 8 bits again."""
    from paper_2511_05534_amd import workloads as wl
    w = wl.make_workload("conversation", "bf16", 77, 2, 6, 2, 64, 16, [[40, 100, 60], [30, 80, 25]], [20, 20])
    K, V, Q = fb.upload_workload(w, DEV)
    p = fb.Params.from_workload(w)
    buf = fb.DeviceBuffers(p)
    buf.plan_merge(K, V, Q, stream())
    caps = [b + 12 for b in w.budgets]
    cu, lens = sums(caps), list(w.budgets)
    cp = params(w.n_layers, w.n_q_heads, w.n_kv_heads, w.head_dim, "bf16", caps, w.budgets)
    cache = fb.QuantizedCache(cp, cu, DEV)
    kept = params(w.n_layers, w.n_q_heads, w.n_kv_heads, w.head_dim, "bf16", w.budgets)  # the strides of the merged rows
    fb.flowmm_cache_quantize(kept, cu, lens, sums(w.budgets), buf.K_out.data_ptr(), buf.V_out.data_ptr(), cache, stream())
    torch.cuda.synchronize()
    a = Attention("fp8", "bf16", w.n_layers, w.n_q_heads, w.n_kv_heads, w.head_dim, [0, 0], room=0)  # (its checks are used on this cache)
    a.caps, a.cu, a.cb, a.p, a.cache = caps, cu, sums(blocks_of(caps)), cp, cache
    a.slopes = torch.tensor([2.0 ** -(h + 1) for h in range(w.n_q_heads)])
    slopes = a.slopes.to(DEV)
    a.merged, a.slots, a.row_pos, a.cap = list(w.budgets), sums(w.budgets), buf.kept_idx.cpu(), 15.0
    a.workspace_bytes = fb.flowmm_cache_sizes(cp, cu)[2]
    a.workspace = torch.empty(max(256, a.workspace_bytes), dtype=torch.uint8, device=DEV)
    gen = torch.Generator().manual_seed(3)
    for step in range(12):
        k, v = (torch.randn((w.n_layers, w.n_kv_heads, 2, w.head_dim), generator=gen).bfloat16().to(DEV) for _ in range(2))
        fb.flowmm_cache_append_quantized(cp, cu, lens, cache, k.data_ptr(), v.data_ptr(), stream())
        lens = [n + 1 for n in lens]
        a.lens, a.q_pos = lens, [L + step for L in w.seqlens]
        a.q = torch.randn((w.n_layers, w.n_q_heads, 2, w.head_dim), generator=gen).bfloat16()
        a.qd, a.out = a.q.to(DEV), torch.full_like(a.q, 9.0).to(DEV)
        a.scoring = fb.Scoring(cap=15.0, slopes=slopes.data_ptr(), row_pos=buf.kept_idx.data_ptr(), q_pos=a.q_pos)
        a.run()
        a.check(f"token {step}")
    with pytest.raises(fb.FlowMMError, match="full"):
        fb.flowmm_cache_append_quantized(cp, cu, lens, cache, k.data_ptr(), v.data_ptr(), stream())
    # sequence 1 back to bf16, re-merged there, and into 8 bits again; sequence 0 is not touched
    before = [t.view(torch.uint8)[:, :, :cu[1]].clone() for t in (cache.k_codes, cache.v_codes)]
    back = [torch.zeros((w.n_layers, w.n_kv_heads, cu[-1], w.head_dim), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    fb.flowmm_cache_dequantize(cp, cu, [0, lens[1]], cu, cache, back[0].data_ptr(), back[1].data_ptr(), stream())
    assert (back[0][:, :, :cu[1]] == 0).all()
    rp = params(w.n_layers, w.n_q_heads, w.n_kv_heads, w.head_dim, "bf16", caps, w.budgets)
    sizes, ws = fb.flowmm_cache_remerge_sizes(rp, cu, 1, lens[1])
    plan = [torch.empty(max(n, 16), dtype=torch.uint8, device=DEV) for n in sizes]
    scratch = torch.empty(ws, dtype=torch.uint8, device=DEV)
    win = torch.randn((w.n_layers, w.n_q_heads, 2, w.head_dim), generator=gen).bfloat16().to(DEV)  # (two sequences of a window of one)
    fb.flowmm_cache_remerge(rp, cu, lens, 1, back[0].data_ptr(), back[1].data_ptr(), win.data_ptr(), [t.data_ptr() for t in plan], scratch.data_ptr(), ws, stream())
    lens[1] = w.budgets[1]
    fb.flowmm_cache_quantize(rp, cu, [0, lens[1]], cu, back[0].data_ptr(), back[1].data_ptr(), cache, stream())
    torch.cuda.synchronize()
    for t, was in zip((cache.k_codes, cache.v_codes), before):
        assert torch.equal(t.view(torch.uint8)[:, :, :cu[1]], was)
    for x, codes, scales in ((back[0], cache.k_codes, cache.k_scales), (back[1], cache.v_codes, cache.v_scales)):
        want, scale = ref.quantize_block(x.cpu()[1, 0, cu[1]:cu[1] + min(32, lens[1])])
        assert torch.equal(codes_as_numbers(codes)[1, 0, cu[1]:cu[1] + min(32, lens[1])], want) and float(scales[1, 0, a.cb[1]]) == scale
    a.lens, a.merged, a.slopes, a.cap, a.scoring = lens, None, None, 0.0, None
    a.run()
    a.check("after the re-merge")
