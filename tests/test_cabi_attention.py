"""What the scored attentions and the calls on a cache in 8 bits refuse, on the host, before anything is launched; no GPU needed."""
import ctypes as C

import pytest

from paper_2511_05534_amd import binding as fb

good, far = 0x10000, [1 << 40, 1 << 41, 1 << 42, 1 << 43, 1 << 44]
CAP = [0, 40, 90]
BIG = 1 << 40


def params(**kw):
    base = dict(n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=128, dtype="bf16", seqlens=[40, 50], budgets=[30, 40], spans=[[(0, 40, 0)], [(0, 10, 0), (10, 50, 1)]],
                window=8, theta=0.25, tau=[0.1, 0.2])
    base.update(kw)
    return fb.Params(**base)


class Cache:
    def __init__(self, **kw):
        f = dict(k_codes=good, v_codes=far[0], k_scales=good + 4, v_scales=good + 8, stride_layer=2 * 90 * 128, stride_head=90 * 128, stride_token=128)
        f.update(kw)
        self.c = fb.flowmm_quantized_cache(**f)


def refused(call, word, status=fb.FLOWMM_EINVAL):
    with pytest.raises(fb.FlowMMError) as e:
        call()
    assert e.value.status == status and word in e.value.message, e.value.message


def test_struct_layouts():
    assert C.sizeof(fb.flowmm_scoring) == 48 and C.sizeof(fb.flowmm_quantized_cache) == 56


def test_sizes():
    p = params()
    codes, scales, ws = fb.flowmm_cache_sizes(p, CAP)
    assert codes == 2 * 2 * 90 * 128 and scales == 2 * 2 * (2 + 2) * 4 and ws > 0 and ws % 256 == 0
    refused(lambda: fb.flowmm_cache_sizes(p, [0, 40, 40]), "increasing")
    refused(lambda: fb.flowmm_cache_sizes(params(head_dim=96), CAP), "head_dim", fb.FLOWMM_EUNSUPPORTED)
    with pytest.raises(ValueError, match="cu_capacity"):
        fb.flowmm_cache_sizes(p, [0, 40])


COMMON = [
    (dict(n_q_heads=5), dict(), "multiple", fb.FLOWMM_EINVAL),
    (dict(head_dim=96), dict(), "head_dim", fb.FLOWMM_EUNSUPPORTED),
    (dict(), dict(lengths=[41, 50]), "outside", fb.FLOWMM_EINVAL),
    (dict(), dict(lengths=[-1, 50]), "outside", fb.FLOWMM_EINVAL),
    (dict(), dict(cap=[0, 40, 30]), "increasing", fb.FLOWMM_EINVAL),
    (dict(), dict(cap=[1, 40, 90]), "cu_capacity[0]", fb.FLOWMM_EINVAL),
    (dict(), dict(cap=[0, 40, 2 ** 31 - 65536]), "rows", fb.FLOWMM_EUNSUPPORTED),
]
CALLS = {
    "quantize": lambda p, cap, ln, c: fb.flowmm_cache_quantize(p, cap, ln, [0, 40], good, far[0], c),
    "dequantize": lambda p, cap, ln, c: fb.flowmm_cache_dequantize(p, cap, ln, [0, 40], c, good, far[0]),
    "append": lambda p, cap, ln, c: fb.flowmm_cache_append_quantized(p, cap, ln, c, good, far[0]),
    "attention": lambda p, cap, ln, c: fb.flowmm_cache_attention(p, cap, ln, None, good, far[0], far[1], far[2], far[3], BIG),
    "attention_quantized": lambda p, cap, ln, c: fb.flowmm_cache_attention_quantized(p, cap, ln, None, good, c, far[2], far[3], BIG),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_descriptions_of_the_cache(name):
    for kw, over, word, status in COMMON:
        refused(lambda: CALLS[name](params(**kw), over.get("cap", CAP), over.get("lengths", [30, 49]), Cache()), word, status)
    for short in ([30], []):
        with pytest.raises(ValueError, match="lengths"):
            CALLS[name](params(), CAP, short, Cache())
    with pytest.raises(ValueError, match="cu_capacity"):
        CALLS[name](params(), [0, 40], [30, 49], Cache())


@pytest.mark.parametrize("name", ["quantize", "dequantize", "append", "attention_quantized"])
def test_descriptions_of_the_codes(name):
    for kw, word in ((dict(k_codes=None), "NULL"), (dict(v_scales=None), "NULL"), (dict(v_codes=far[0] + 8), "aligned"), (dict(k_scales=good + 2), "aligned"),
                     (dict(stride_token=120), "16 bytes"), (dict(stride_token=112), "head_dim"), (dict(stride_head=-16), "16 bytes")):
        refused(lambda: CALLS[name](params(), CAP, [30, 49], Cache(**kw)), word)


def test_rows():
    p = params()
    refused(lambda: fb.flowmm_cache_quantize(p, CAP, [30, 49], [0, -1], good, far[0], Cache()), "cu_rows")
    refused(lambda: fb.flowmm_cache_quantize(p, CAP, [30, 49], [0, 40], 0, far[0], Cache()), "NULL")
    refused(lambda: fb.flowmm_cache_dequantize(p, CAP, [30, 49], [0, 40], Cache(), good, far[0] + 4), "aligned")
    refused(lambda: fb.flowmm_cache_quantize(params(k_strides=(1024, 1024, 100)), CAP, [30, 49], [0, 40], good, far[0], Cache()), "16 bytes")
    refused(lambda: fb.flowmm_cache_append_quantized(p, CAP, [30, 50], Cache(), good, far[0]), "full")
    refused(lambda: fb.flowmm_cache_append_quantized(p, CAP, [30, 49], Cache(), good + 4, far[0]), "aligned")
    refused(lambda: fb.flowmm_cache_append_quantized(p, CAP, [30, 49], Cache(), good, 0), "NULL")
    with pytest.raises(ValueError, match="cu_rows"):
        fb.flowmm_cache_quantize(p, CAP, [30, 49], [0], good, far[0], Cache())


SCORING = [(dict(cap=-1.0), "cap"), (dict(cap=float("nan")), "cap"), (dict(cap=float("inf")), "cap"), (dict(cap=1e-45), "cap"), (dict(cap=1e-39), "cap"), (dict(cap=2e36), "cap"), (dict(slopes=good + 2), "slopes")]


def test_attention_over_a_cache():
    p, ws = params(), fb.flowmm_cache_sizes(params(), CAP)[2]

    def plain(p=p, scoring=None, q=good, K=far[0], V=far[1], out=far[2], w=far[3], n=BIG):
        return lambda: fb.flowmm_cache_attention(p, CAP, [30, 49], scoring, q, K, V, out, w, n)

    def quantized(p=p, scoring=None, q=good, out=far[2], w=far[3], n=BIG, cache=None):
        return lambda: fb.flowmm_cache_attention_quantized(p, CAP, [30, 49], scoring, q, cache or Cache(), out, w, n)

    for call in (plain, quantized):
        for kw, word in ((dict(q=0), "NULL"), (dict(out=0), "NULL"), (dict(w=0), "NULL"), (dict(q=good + 8), "aligned"), (dict(out=good + 256), "overlap"),
                         (dict(p=params(scale=-1.0)), "scale"), (dict(scoring=fb.Scoring(row_pos=good)), "together"), (dict(scoring=fb.Scoring(q_pos=[1, 2])), "together"),
                         (dict(scoring=fb.Scoring(row_pos=good + 1, q_pos=[1, 2])), "row_pos"),
                         (dict(p=params(budgets=[0, 40]), scoring=fb.Scoring(row_pos=good, q_pos=[1, 2])), "budget"),
                         (dict(p=params(budgets=[41, 40]), scoring=fb.Scoring(row_pos=good, q_pos=[1, 2])), "budget")):
            refused(call(**kw), word)
        for kw, word in SCORING:
            refused(call(scoring=fb.Scoring(**kw)), word)
        refused(call(n=ws - 1), "workspace", fb.FLOWMM_EWORKSPACE)
        with pytest.raises(ValueError, match="q_pos"):
            call(scoring=fb.Scoring(row_pos=good, q_pos=[1]))()
    refused(plain(K=0), "NULL")
    refused(plain(V=far[1] + 4), "aligned")
    refused(plain(p=params(k_strides=(0, 0, 1 << 27))), "4 GiB", fb.FLOWMM_EUNSUPPORTED)
    refused(quantized(cache=Cache(stride_token=1 << 28)), "4 GiB", fb.FLOWMM_EUNSUPPORTED)


def test_prompt_attention():
    p = params()
    ws = fb.flowmm_plan_sizes(p)[1]
    qs = (4 * 90 * 128, 90 * 128, 128)

    def call(p=p, scoring=None, K=good, V=far[0], Q=far[1], qs=qs, out=far[2], w=far[3], n=BIG):
        return lambda: fb.flowmm_prompt_attention(p, scoring, K, V, Q, qs, out, w, n)

    for kw, word in ((dict(K=0), "NULL"), (dict(out=0), "NULL"), (dict(w=0), "NULL"), (dict(V=far[0] + 8), "aligned"), (dict(out=far[1] + 256), "overlap"), (dict(out=good + 256), "overlap"),
                     (dict(qs=(qs[0], qs[1], 100)), "16 bytes"), (dict(qs=(qs[0], qs[1], 64)), "head_dim"), (dict(qs=(qs[0], -8, 128)), "16 bytes"),
                     (dict(p=params(window=0)), "window"), (dict(p=params(scale=float("inf"))), "scale"),
                     (dict(scoring=fb.Scoring(prefix=[41, 0])), "prefix[0]"), (dict(scoring=fb.Scoring(prefix=[0, -1])), "prefix[1]")):
        refused(call(**kw), word)
    for kw, word in SCORING:
        refused(call(scoring=fb.Scoring(**kw)), word)
    refused(call(qs=(qs[0], 0, 128)), "one place")
    refused(call(qs=(0, qs[1], 128)), "one place")
    refused(call(qs=(128, 128, 1 << 27)), "4 GiB", fb.FLOWMM_EUNSUPPORTED)
    refused(call(n=ws - 1), "workspace", fb.FLOWMM_EWORKSPACE)
    with pytest.raises(ValueError, match="prefix"):
        call(scoring=fb.Scoring(prefix=[1]))()


def test_integer_arrays_of_any_form():
    """Strided and wider arrays are read as what they hold."""
    import numpy as np
    p = params()
    wide = np.array([0, 7, 40, 7, 90])[::2]
    assert fb.flowmm_cache_sizes(p, wide) == fb.flowmm_cache_sizes(p, CAP)
    assert fb.flowmm_cache_sizes(p, wide.astype(np.int32)[::1]) == fb.flowmm_cache_sizes(p, np.array([0, 9, 40, 9, 90], np.int32)[::2])
    for values in ([3, 4], (3, 4), np.array([3, 4]), np.array([3, 9, 4, 9], np.int32)[::2]):
        s = fb.Scoring(prefix=values, q_pos=values, row_pos=good)
        assert [s.c.prefix[i] for i in range(2)] == [3, 4] and [s.c.q_pos[i] for i in range(2)] == [3, 4]


def test_rows_that_would_share_a_place():
    p = params()
    for name in ("quantize", "append"):
        for kw in (dict(stride_layer=0), dict(stride_head=0)):
            refused(lambda: CALLS[name](p, CAP, [30, 49], Cache(**kw)), "one place")
    for strides in ((0, 90 * 128, 128), (2 * 90 * 128, 0, 128)):
        refused(lambda: CALLS["dequantize"](params(k_strides=strides), CAP, [30, 49], Cache()), "one place")
    for rows in ([0, 29], [7, 7], [48, 0]):
        refused(lambda: fb.flowmm_cache_dequantize(p, CAP, [30, 49], rows, Cache(), good, far[0]), "one place")


def test_prompt_attention_takes_layouts_that_the_plan_refuses():
    """Its own limits are those of the queries' strides alone: what follows gets as far as the size of its workspace, which is that of the description of the batch."""
    for kw in (dict(n_q_heads=48), dict(n_q_heads=1024, n_kv_heads=1), dict(window=41), dict(budgets=[0, 40]), dict(budgets=[41, 40]), dict(n_q_heads=48, head_dim=64, dtype="f32"),
               dict(seqlens=[60000, 50], budgets=[60000, 40], spans=[[(0, 60000, 0)], [(0, 10, 0), (10, 50, 1)]])):
        p = params(**kw)
        with pytest.raises(fb.FlowMMError):
            fb.flowmm_plan_sizes(p)
        like = dict(kw, window=1, budgets=[1, 1], n_q_heads=kw.get("n_kv_heads", 2))
        need = fb.flowmm_plan_sizes(params(**like))[1]
        T, d = sum(kw.get("seqlens", [40, 50])), kw.get("head_dim", 128)
        hq = kw.get("n_q_heads", 4)
        places = [1 << 40, 1 << 44, 1 << 48, 1 << 52, 1 << 56]

        def call(n, p=p, qs=(hq * T * d, T * d, d)):
            return lambda: fb.flowmm_prompt_attention(p, None, places[0], places[1], places[2], qs, places[3], places[4], n)

        refused(call(0), "workspace", fb.FLOWMM_EWORKSPACE)
        with pytest.raises(fb.FlowMMError) as e:
            call(255)()
        assert int(e.value.message.split()[-2]) <= need, e.value.message
        refused(call(need, qs=(hq * T * d, T * d, 8)), "head_dim")
    for kw, word in ((dict(n_q_heads=2048, n_kv_heads=1), "1024"), (dict(n_q_heads=5), "multiple"), (dict(window=0), "window"), (dict(window=-3, budgets=[0, 0]), "window"), (dict(head_dim=96), "head_dim")):
        with pytest.raises(fb.FlowMMError, match=word):
            fb.flowmm_prompt_attention(params(**kw), None, good, far[0], far[1], (4 * 90 * 128, 90 * 128, 128), far[2], far[3], BIG)


def test_the_last_error_is_that_of_a_call_that_failed():
    refused(lambda: fb.flowmm_prompt_attention(params(window=0), None, good, far[0], far[1], (4 * 90 * 128, 90 * 128, 128), far[2], far[3], BIG), "window")
    refused(lambda: fb.flowmm_prompt_attention(params(n_q_heads=48), None, good, far[0], far[1], (48 * 90 * 128, 90 * 128, 8), far[2], far[3], BIG), "head_dim")


def test_a_cache_in_8_bits_lies_on_a_gpu():
    """Tensors of the host's memory, whose addresses mean nothing to the kernels, and of the wrong shape, type or order."""
    import torch
    p = params()

    def tensors(codes=(2, 2, 90, 128), scales=(2, 2, 4), dtype=torch.float8_e4m3fn, order=lambda t: t):
        return [order(torch.zeros(codes, dtype=torch.uint8).view(dtype)) for _ in range(2)] + [torch.zeros(scales) for _ in range(2)]

    for kw, word in ((dict(), "GPU"), (dict(codes=(2, 2, 89, 128)), "shape"), (dict(scales=(2, 2, 3)), "shape"), (dict(dtype=torch.uint8), "float8"),
                     (dict(codes=(2, 2, 128, 90), order=lambda t: t.transpose(2, 3)), "contiguous")):
        with pytest.raises(ValueError, match=word):
            fb.QuantizedCache(p, CAP, tensors=tensors(**kw))
    with pytest.raises(ValueError, match="GPU"):
        fb.QuantizedCache(p, CAP, "cpu")


def test_prompt_attention_without_its_arrays():
    """Refused before anything of the batch's size is allocated."""
    for name in ("cu_seqlens", "budget_tokens", "spans", "cu_spans", "tau"):
        p = params(n_q_heads=48)
        setattr(p.c, name, None)
        p.c.batch = 2 ** 31 - 1
        refused(lambda: fb.flowmm_prompt_attention(p, None, good, far[0], far[1], (48 * 90 * 128, 90 * 128, 128), far[2], far[3], BIG), "NULL")
