"""The prompt's attention (flowmm_prompt_attention) against a plain 64-bit form."""
import numpy as np
import pytest
import torch

import attention_reference as ref
from paper_2511_05534_amd import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def stream():
    return torch.cuda.current_stream().cuda_stream


def sums(x):
    return [0, *np.cumsum(x).tolist()]


def alternating(L, lengths):
    """Spans of text and images in turn, of the given lengths over and over."""
    spans, at, i = [], 0, 0
    while at < L:
        n = min(lengths[i % len(lengths)], L - at)
        spans.append((at, at + n, i & 1))
        at, i = at + n, i + 1
    return spans


class Prompt:
    def __init__(self, dtype, layers, hq, hkv, d, lens, cap=0.0, slopes=False, prefix=None, spans=None, image_spans=False, token_major=False, seed=0, scale=0.0):
        self.dtype, self.layers, self.hq, self.hkv, self.d, self.lens = dtype, layers, hq, hkv, d, lens
        self.cap, self.prefix, self.image_spans, self.scale = cap, prefix, image_spans, scale or d ** -0.5
        self.spans = spans or [[(0, L, 0)] for L in lens]
        dt, T, self.cu = DT[dtype], sum(lens), sums(lens)
        g = torch.Generator().manual_seed(seed)
        gain = torch.where(torch.rand(T, generator=g) < 0.03, 8.0, 1.0)
        self.K = (torch.randn((layers, hkv, T, d), generator=g) * gain[:, None]).to(dt)
        self.V, self.Q = torch.randn((layers, hkv, T, d), generator=g).to(dt), torch.randn((layers, hq, T, d), generator=g).to(dt)
        self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]) if slopes else None
        self.token_major = token_major
        if token_major:  # [Lyr][T][heads][d], as a projection leaves them
            k_strides, self.q_strides = (T * hkv * d, d, hkv * d), (T * hq * d, d, hq * d)
        else:
            k_strides, self.q_strides = (hkv * T * d, T * d, d), (hq * T * d, T * d, d)
        self.p = fb.Params(layers, hq, hkv, d, dtype, lens, lens, self.spans, 1, 0.25, [1.0] * len(lens), k_strides=k_strides, scale=scale)
        self.ws_bytes = fb.flowmm_plan_sizes(self.p)[1]
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=DEV)
        self.sl = self.slopes.to(DEV) if slopes else None
        self.scoring = fb.Scoring(cap=cap, slopes=self.sl.data_ptr() if slopes else 0, prefix=prefix, image_spans=image_spans) \
            if cap or slopes or prefix is not None or image_spans else None
        self.upload()

    def upload(self):
        lay = (lambda x: x.transpose(1, 2).contiguous().to(DEV)) if self.token_major else (lambda x: x.to(DEV))
        self.dev = [lay(x) for x in (self.K, self.V, self.Q)]
        self.out = torch.full_like(self.dev[2], 55.0)

    def run(self, on=None):
        k, v, q = self.dev
        fb.flowmm_prompt_attention(self.p, self.scoring, k.data_ptr(), v.data_ptr(), q.data_ptr(), self.q_strides, self.out.data_ptr(), self.ws.data_ptr(),
                                   self.ws_bytes, stream() if on is None else on)
        return self.out

    def hidden(self, b):
        L = self.lens[b]
        i = np.arange(L)
        seen = i[None, :] <= i[:, None]
        if self.prefix is not None:
            seen |= (i[:, None] < self.prefix[b]) & (i[None, :] < self.prefix[b])
        if self.image_spans:
            for s, e, image in self.spans[b]:
                if image:
                    seen[s:e, s:e] = True
        return torch.from_numpy(~seen)

    def check(self, what="", heads=None):
        torch.cuda.synchronize()
        got = self.out.cpu()
        got = got.transpose(1, 2) if self.token_major else got
        G, worst = self.hq // self.hkv, 0.0
        for b, L in enumerate(self.lens):
            r, hidden = slice(self.cu[b], self.cu[b] + L), self.hidden(b)
            i = torch.arange(L)
            far = (i[:, None] - i[None, :]).abs().double() if self.slopes is not None else None
            for l in range(self.layers):
                for h in heads or range(self.hq):
                    want, tol = ref.attend(self.Q[l, h, r], self.K[l, h // G, r], self.V[l, h // G, r], self.scale, self.cap,
                                           None if self.slopes is None else float(self.slopes[h]), far, hidden, DT[self.dtype], 2.0 ** -8 if self.dtype == "bf16" else 0.0)
                    worst = max(worst, ref.check(got[l, h, r], want, tol, (what, b, l, h)))
        print(f"{what} of the tolerance: {worst:.3f}", flush=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq, hkv, lens", [(3, 3, [1, 2, 31, 32, 33, 64, 65]), (14, 2, [127, 128, 129]), (8, 1, [300]), (9, 1, [5, 200]), (2, 2, [513])])
def test_lengths_and_heads(dtype, d, hq, hkv, lens):
    a = Prompt(dtype, 2, hq, hkv, d, lens, seed=hq)
    a.run()
    a.check(f"{dtype} {d} {hq}/{hkv} {lens}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap, slopes, prefix, image_spans", [(20.0, False, False, False), (0.0, True, False, False), (0.0, False, True, False),
                                                             (0.0, False, False, True), (2.0, True, True, True)])
def test_scores_and_masks(dtype, cap, slopes, prefix, image_spans):
    lens = [200, 1, 333, 96]
    a = Prompt(dtype, 1, 8, 2, 128, lens, cap=cap, slopes=slopes, prefix=[90, 1, 333, 0] if prefix else None, spans=[alternating(L, [17, 45, 3]) for L in lens],
               image_spans=image_spans, seed=7)
    a.run()
    a.check(f"{dtype} cap {cap} slopes {slopes} prefix {prefix} spans {image_spans}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap, slopes", [(0.5, False), (512.0, False), (513.0, False), (1e5, False), (1e5, True), (1e30, False)])
def test_caps_of_any_size(dtype, cap, slopes):
    """Caps far above the logits leave them as they are, small ones flatten them."""
    a = Prompt(dtype, 1, 4, 2, 64, [130], cap=cap, slopes=slopes, seed=18)
    a.run()
    a.check(f"{dtype} cap {cap}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_spans_and_sequences(dtype):
    """More words of description than a kernel's arguments hold."""
    lens = [30 + b for b in range(40)]
    a = Prompt(dtype, 1, 2, 2, 64, lens, spans=[alternating(L, [1, 2, 1, 3]) for L in lens], image_spans=True, seed=8)
    assert sum(len(s) for s in a.spans) > 500
    a.run()
    a.check(f"{dtype} many spans")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("units", [(1, 1), (3, 8)])
def test_long_prompt(dtype, units):
    """Many key tiles, with few workgroups (the keys split among waves) and with many."""
    hkv, G = units
    a = Prompt(dtype, 1, hkv * G, hkv, 64, [2100], slopes=hkv > 1, seed=9)
    a.run()
    a.check(f"{dtype} long {units}", heads=[0, hkv * G - 1])
    first = a.out.clone()
    a.out.fill_(1.0)
    a.run()
    assert torch.equal(a.out, first)


@pytest.mark.parametrize("dtype, L, cap, slopes", [("bf16", 2100, 0.0, False), ("bf16", 2100, 15.0, False), ("bf16", 2090, 0.0, True), ("bf16", 2100, 600.0, True), ("f32", 3700, 0.0, False)])
@pytest.mark.parametrize("d", [64, 128])
def test_more_rows_than_the_compute_units_take_at_once(dtype, L, cap, slopes, d):
    """Every wave has rows of its own and whole blocks of keys two at a time."""
    a = Prompt(dtype, 1, 32, 8, d, [L], cap=cap, slopes=slopes, seed=19)
    a.run()
    a.check(f"{dtype} {L} {d} cap {cap} slopes {slopes}", heads=[0, 31])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L, hq", [(700, 24), (1100, 32)])
def test_pictures_of_most_of_the_prompt(dtype, L, hq):
    """Rows that nearly all see as much: another split of the keys."""
    a = Prompt(dtype, 1, hq, hq, 64, [L], spans=[[(0, 20, 0), (20, L - 30, 1), (L - 30, L, 0)]], image_spans=True, seed=20)
    a.run()
    a.check(f"{dtype} {L} {hq}", heads=[0, hq - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [0, 20, 60])
def test_scores_of_any_size(dtype, power):
    """Logits 2^power apart, the largest beyond 2^24 or 1e18: the visible keys of the largest one weigh the same, the others nothing."""
    L = 300
    a = Prompt(dtype, 1, 2, 1, 64, [L], seed=22)
    level = torch.randint(-3, 4, (L,), generator=torch.Generator().manual_seed(5)).float()
    a.Q[:] = 0.0
    a.Q[..., 0] = 2.0 ** power * 8 * 128  # (scale is an eighth)
    a.K[:] = 0.0
    a.K[0, 0, :, 0] = level.to(a.K.dtype)
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got, V = a.out.cpu().double()[0, 0], a.V[0, 0].double()
    top = torch.cummax(level, 0).values
    weight = torch.tril((level[None, :] == top[:, None]).double())
    want, size = weight @ V / weight.sum(-1, keepdim=True), weight @ V.abs() / weight.sum(-1, keepdim=True)
    assert ((got - want).abs() <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -14) * size + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_scale(dtype):
    a = Prompt(dtype, 2, 6, 2, 64, [70, 45], token_major=True, scale=0.21, seed=10)
    a.run()
    a.check(f"{dtype} token major")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_token_does_not_see_does_not_reach_it(dtype, d):
    """Infinities and NaN in keys and values: in the results of the tokens that see them (by the formula), in no other's."""
    lens = [100, 70]
    a = Prompt(dtype, 1, 4, 2, d, lens, seed=11)
    a.V[0, 0, 40, 3], a.V[0, 0, 41, 5], a.V[0, 0, 99, 7] = float("inf"), float("-inf"), float("nan")
    a.V[0, 0, 45, 5] = float("inf")   # with the -inf of token 41: NaN from here on
    a.V[0, 1, 100 + 33, 0] = float("nan")
    a.K[0, 1, 77, 2] = float("nan")   # sequence 0, kv head 1: rows from 77 on are NaN
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu().float()
    for h in (0, 1):
        o = got[0, h, :100]
        assert torch.isfinite(o[:40]).all()
        assert (o[40:, 3] == float("inf")).all() and torch.isfinite(o[:40, 3]).all()
        assert (o[41:45, 5] == float("-inf")).all() and o[45:, 5].isnan().all() and torch.isfinite(o[:41, 5]).all()
        assert o[99, 7].isnan() and torch.isfinite(o[:99, 7]).all()
        other = [c for c in range(d) if c not in (3, 5, 7)]
        assert torch.isfinite(o[:, other]).all()
        assert torch.isfinite(got[0, h, 100:]).all()
    for h in (2, 3):
        o = got[0, h, :100]
        assert torch.isfinite(o[:77]).all() and o[77:].isnan().all()
        o = got[0, h, 100:]
        assert o[33:, 0].isnan().all() and torch.isfinite(o[:33]).all() and torch.isfinite(o[:, 1:]).all()
    # the finite rest is what the formula says without them
    clean = Prompt(dtype, 1, 4, 2, d, lens, seed=11)
    for t in ("K", "V"):
        setattr(clean, t, getattr(a, t).nan_to_num(0.0, 0.0, 0.0))
    clean.upload()
    clean.run()
    torch.cuda.synchronize()
    want = clean.out.cpu().float()
    assert torch.equal(got[0, :2, :40], want[0, :2, :40]) and torch.equal(got[0, 2:, :77], want[0, 2:, :77])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("L, hq", [(400, 1), (700, 40), (900, 140)])  # keys split over four waves, two, one
def test_infinities_in_pictures_of_many_blocks(dtype, cap, L, hq):
    """The first block of rows sees the picture in part: its text rows get what they get without the picture's infinities, bit for bit."""
    a = Prompt(dtype, 1, hq, hq, 64, [L], cap=cap, spans=[[(0, 20, 0), (20, L - 30, 1), (L - 30, L, 0)]], image_spans=True, seed=24)
    a.run()
    torch.cuda.synchronize()
    clean = a.out.cpu().float()
    places = [(25, 3, float("inf"), 20), (L // 2, 5, float("-inf"), 20), (L // 2 + 33, 5, float("-inf"), 20), (L - 40, 7, float("nan"), 20), (L - 10, 9, float("inf"), L - 10)]
    for row, ch, x, _ in places:
        a.V[0, :, row, ch] = x
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu().float()
    for _, ch, x, first in places:
        o = got[0, :, first:, ch]
        assert (o.isnan() if x != x else o == x).all(), (ch, x)
    for _, ch, _, first in places:
        got[0, :, first:, ch] = clean[0, :, first:, ch]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lowest_values_in_the_logits(dtype):
    """Logits of the lowest finite size and of -infinity beside ordinary ones: they weigh nothing."""
    a = Prompt(dtype, 1, 1, 1, 64, [40], seed=12)
    a.Q[:] = 0.0
    a.Q[..., 0] = 8.0
    a.K[0, 0, :, 0] = 0.25
    a.K[0, 0, 5, 0], a.K[0, 0, 9, 0], a.K[0, 0, 0, 0] = -torch.finfo(DT[dtype]).max, float("-inf"), -1e30
    a.upload()
    a.run()
    torch.cuda.synchronize()
    got = a.out.cpu().double()[0, 0]
    weight = torch.tril(torch.ones(40, 40, dtype=torch.float64))
    weight[1:, [0]] = 0.0
    weight[6:, 5], weight[:, 9] = 0.0, 0.0
    weight[5, 5] = 0.0
    want = weight @ a.V[0, 0].double() / weight.sum(-1, keepdim=True)
    tol = (2.0 ** -8 + 2.0 ** -8 if dtype == "bf16" else 2.0 ** -18) * (weight @ a.V[0, 0].double().abs() / weight.sum(-1, keepdim=True)) + 1e-30
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_beyond_32_bit_offsets(dtype):
    """Keys and values 2 MB apart, so that a tile's rows are not addressed with 32 bits and a sequence spans more than 4 GiB."""
    L, d, step = 2200, 64, 1 << 21
    es = 2 if dtype == "bf16" else 4
    a = Prompt(dtype, 1, 1, 1, d, [L], seed=13)
    far = torch.empty(L * step, dtype=torch.uint8, device=DEV)
    both = torch.cat([a.dev[0][0, 0].view(torch.uint8), a.dev[1][0, 0].view(torch.uint8)], -1)
    at = (torch.arange(L, device=DEV) * step)[:, None] + torch.arange(2 * d * es, device=DEV)[None, :]
    far[at.reshape(-1)] = both.reshape(-1)
    p = fb.Params(1, 1, 1, d, dtype, [L], [L], [[(0, L, 0)]], 1, 0.25, [1.0], k_strides=(0, 0, step // es))
    ws = torch.empty(fb.flowmm_plan_sizes(p)[1], dtype=torch.uint8, device=DEV)
    fb.flowmm_prompt_attention(p, None, far.data_ptr(), far.data_ptr() + d * es, a.dev[2].data_ptr(), a.q_strides, a.out.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    a.check(f"{dtype} far")


def test_rows_too_far_apart_for_a_tile():
    """Keys 40 MB apart (a tile of 128 spans more than 4 GiB)."""
    L, d, step = 150, 64, 40 << 20
    a = Prompt("bf16", 1, 1, 1, d, [L], seed=14)
    far = torch.empty(L * step, dtype=torch.uint8, device=DEV)
    both = torch.cat([a.dev[0][0, 0].view(torch.uint8), a.dev[1][0, 0].view(torch.uint8)], -1)
    at = (torch.arange(L, device=DEV) * step)[:, None] + torch.arange(4 * d, device=DEV)[None, :]
    far[at.reshape(-1)] = both.reshape(-1)
    p = fb.Params(1, 1, 1, d, "bf16", [L], [L], [[(0, L, 0)]], 1, 0.25, [1.0], k_strides=(0, 0, step // 2))
    ws = torch.empty(fb.flowmm_plan_sizes(p)[1], dtype=torch.uint8, device=DEV)
    fb.flowmm_prompt_attention(p, None, far.data_ptr(), far.data_ptr() + 2 * d, a.dev[2].data_ptr(), a.q_strides, a.out.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    a.check("far tile")


def test_in_a_graph_and_on_another_stream():
    lens = [30 + b for b in range(40)]
    for a in (Prompt("bf16", 1, 8, 2, 128, [400, 77], cap=10.0, slopes=True, prefix=[30, 0], seed=15),
              Prompt("bf16", 1, 2, 2, 64, lens, spans=[alternating(L, [1, 2, 1, 3]) for L in lens], image_spans=True, seed=16)):  # (its description goes through the workspace)
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
            a.ws.fill_(0xff)
            torch.randn(1 << 20, device=DEV).sum().item()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(a.out, want)


def test_buffers_entry_point():
    from paper_2511_05534_amd import workloads as wl
    w = wl.make_workload("prompt", "bf16", 3, 1, 4, 2, 64, 8, [[20, 50, 12]], [40])
    a = Prompt("bf16", 1, 4, 2, 64, w.seqlens, spans=w.spans, image_spans=True, seed=17)
    want = a.run().clone()
    buf = fb.DeviceBuffers(fb.Params.from_workload(w))
    out = torch.empty_like(want)
    buf.prompt_attention(a.dev[0], a.dev[1], a.dev[2], out, a.scoring, stream())
    torch.cuda.synchronize()
    assert torch.equal(out, want)
