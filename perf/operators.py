"""What the performance of the cache's 8-bit operators and of the attention with scored, masked prompts is measured on.

Six calls of a serving program: the prompt's attention (`flowmm_prompt_attention`), the step of one token over a cache
that has grown past its merged rows (`flowmm_cache_attention`), the same over a cache held in 8 bits
(`flowmm_cache_attention_quantized`), the merged rows' way into 8 bits (`flowmm_cache_quantize`) and back for a re-merge
(`flowmm_cache_dequantize`), and a new token's rows (`flowmm_cache_append_quantized`).

Inputs follow `workloads.py`: text rows N(0,1), image rows shifted, 1 % sink keys eight times as long.  An 8-bit cache holds
e4m3 numbers with a power of two for every 32 rows of a (layer, kv head, sequence).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
BLOCK = 32  # rows that share a scale
FP8_MOST = 448.0


def listed():
    mha = {"q_heads": 32, "kv_heads": 32, "head_dim": 128}
    gqa7 = {"q_heads": 28, "kv_heads": 4, "head_dim": 128}
    gqa4 = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}
    small = {"q_heads": 16, "kv_heads": 4, "head_dim": 64}
    plain = {"cap": 0.0, "slopes": 0}
    return [
        # a generated token of one conversation: the smallest call, as often as there are tokens
        {"name": "append_450", "kind": "append", "dtype": "bf16", **gqa7, "layers": 28, "batch": 1, "rows": 450, "room": 62, "ragged": 0},
        # a generated token of each of 64 conversations
        {"name": "append_batch64", "kind": "append", "dtype": "bf16", **gqa4, "layers": 32, "batch": 64, "rows": 500, "room": 12, "ragged": 1},
        # the merged rows of one picture and a short question
        {"name": "quantize_410", "kind": "quantize", "dtype": "bf16", **gqa7, "layers": 28, "batch": 1, "rows": 410, "room": 102, "ragged": 0},
        # the merged rows of eight long prompts of different lengths
        {"name": "quantize_ragged8", "kind": "quantize", "dtype": "bf16", **gqa4, "layers": 32, "batch": 8, "rows": 4096, "room": 256, "ragged": 1},
        # a cache that has grown a quarter beyond its budget, on its way to a re-merge
        {"name": "dequantize_1023", "kind": "dequantize", "dtype": "bf16", **gqa4, "layers": 32, "batch": 1, "rows": 1023, "room": 1, "ragged": 0},
        # a token of one conversation over 410 merged rows and 40 decoded ones
        {"name": "attention_quantized_450", "kind": "attention_quantized", "dtype": "bf16", **gqa7, "layers": 28, "batch": 1, "rows": 450, "room": 62, "ragged": 0,
         "merged": 0, **plain},
        # a token of each of 32 conversations of up to 16384 rows, capped scores: four layers of a large batch
        {"name": "attention_quantized_ragged32", "kind": "attention_quantized", "dtype": "bf16", **gqa4, "layers": 4, "batch": 32, "rows": 16384, "room": 64,
         "ragged": 1, "merged": 0, "cap": 30.0, "slopes": 0},
        # a token over 3277 merged rows at their positions in the prompt and 411 decoded ones, scores that fall with distance
        {"name": "attention_3688", "kind": "attention", "dtype": "bf16", **gqa4, "layers": 32, "batch": 1, "rows": 3688, "room": 408, "ragged": 0, "merged": 3277,
         "cap": 0.0, "slopes": 1},
        # a small fp32 model, four conversations
        {"name": "attention_900_fp32", "kind": "attention", "dtype": "f32", **small, "layers": 8, "batch": 4, "rows": 900, "room": 100, "ragged": 1, "merged": 0,
         "cap": 20.0, "slopes": 1},
        # one layer's prompt: one picture whose patches see each other, and a short question
        {"name": "prompt_675", "kind": "prompt", "dtype": "bf16", **mha, "layers": 1, "batch": 1, "length": 675, "ragged": 0, "images": 1, "both_ways": 1, "prefix": 0,
         **plain},
        # one layer's prompts, eight of them packed, odd lengths, capped scores, the first 200 tokens visible to all of their prompt
        {"name": "prompt_ragged8", "kind": "prompt", "dtype": "bf16", **gqa7, "layers": 1, "batch": 8, "length": 8192, "ragged": 1, "images": 1, "both_ways": 0,
         "prefix": 200, "cap": 50.0, "slopes": 0},
        # one layer's long prompt with many pictures: the largest
        {"name": "prompt_16384", "kind": "prompt", "dtype": "bf16", **gqa4, "layers": 1, "batch": 1, "length": 16384, "ragged": 0, "images": 8, "both_ways": 0,
         "prefix": 0, **plain},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Time of a call, roughly, in seconds."""
    w = work(case)
    return 1e-5 + w["bytes"] / 4e12 + w["flops"] / (7e14 if case["dtype"] == "bf16" else 5e13)


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in {c["kind"] for c in listed()}}
    while True:
        case = _draw_any(rng)
        if _cost(case) <= most[case["kind"]]:
            return case


def _draw_any(rng):
    kind = rng.choice(["append", "quantize", "dequantize", "attention_quantized", "attention_quantized", "attention", "prompt", "prompt"])
    case = {"kind": kind, "dtype": "f32" if rng.random() < 0.25 else "bf16"}
    case.update(rng.choice([
        {"q_heads": 32, "kv_heads": 32, "head_dim": 128},
        {"q_heads": 28, "kv_heads": 4, "head_dim": 128},
        {"q_heads": 32, "kv_heads": 8, "head_dim": 128},
        {"q_heads": 16, "kv_heads": 4, "head_dim": 64},
        {"q_heads": 16, "kv_heads": 1, "head_dim": 64},
    ]))
    scored = {"cap": rng.choice([0.0, 0.0, round(rng.uniform(5.0, 60.0), 1)]), "slopes": rng.choice([0, 0, 1])}
    if kind == "prompt":
        batch = rng.choice([1, 1, rng.randint(2, 8)])
        case.update(layers=rng.randint(1, 2), batch=batch, length=_log_int(rng, 1, 2048 if case["dtype"] == "f32" else 16384 if batch == 1 else 8192),
                    ragged=rng.randint(0, 1), images=rng.randint(1, 8), both_ways=rng.randint(0, 1), prefix=rng.choice([0, 0, rng.randint(1, 500)]), **scored)
        return case
    case.update(layers=rng.choice([rng.randint(1, 8), rng.randint(1, 32), 28, 32]), batch=rng.choice([1, rng.randint(2, 8), rng.randint(9, 64)]),
                rows=_log_int(rng, 1, 16384 if "attention" in kind else 4096), room=rng.randint(1, 300), ragged=rng.randint(0, 1))
    if "attention" in kind:
        case.update(merged=rng.choice([0, max(1, case["rows"] * 4 // 5)]), **scored)
    return case


# ---- shapes of a case --------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens of every prompt, or valid rows of every sequence's cache."""
    n, L = case["batch"], case["length"] if case["kind"] == "prompt" else case["rows"]
    if not case["ragged"]:
        return [L] * n
    rng = random.Random(n * 100003 + L)
    return [rng.randint(max(L // 4, 1), L) for _ in range(n)]


def _capacities(case):
    return [n + case["room"] for n in _lengths(case)]


def _merged(case):
    """Merged rows at the head of every sequence's cache."""
    return [max(1, n * case["merged"] // case["rows"]) if case["merged"] else n for n in _lengths(case)]


def _spans(case):
    """(begin, end, modality) of every prompt: text and images in turn, the question at the end."""
    spans = []
    for L in _lengths(case):
        k = min(case["images"], max(1, L // 64))
        image = L * 3 // 4 // k
        text = (L - k * image) // (k + 1)
        one, at = [], 0
        for i, n in enumerate([text, image] * k + [L]):
            n = min(n, L - at)
            if n > 0:
                one.append((at, at + n, i & 1))
                at += n
        spans.append(one)
    return spans


def _reach(case):
    """The last key that every token of every prompt sees, int64 arrays."""
    got = []
    for L, spans in zip(_lengths(case), _spans(case)):
        r = np.arange(L, dtype=np.int64)
        p = min(case["prefix"], L)
        r[:p] = np.maximum(r[:p], p - 1)
        if case["both_ways"]:
            for s, e, image in spans:
                if image:
                    r[s:e] = np.maximum(r[s:e], e - 1)
        got.append(r)
    return got


def _blocks(case):
    return [-(-c // BLOCK) for c in _capacities(case)]


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    d, units, lens = case["head_dim"], case["layers"] * case["kv_heads"], _lengths(case)
    kind, n, batch = case["kind"], sum(lens), case["batch"]
    if kind == "prompt":
        pairs = sum(int((r + 1).sum()) for r in _reach(case))
        heads = case["layers"] * case["q_heads"]
        return {"bytes": es * d * n * 2 * (heads + units), "flops": 4 * d * heads * pairs}
    scales = 2 * units * sum(-(-x // BLOCK) for x in lens) * 4
    if kind == "append":
        return {"bytes": units * batch * (2 * d * (es + 1) + 2 * 2 * 4), "flops": units * batch * 4 * d}
    if kind in ("quantize", "dequantize"):
        return {"bytes": 2 * units * n * d * (es + 1) + scales, "flops": 2 * units * n * d * 2}
    q = case["layers"] * case["q_heads"] * batch * d * es
    rows = 2 * units * n * d * (1 if kind == "attention_quantized" else es) + (scales if kind == "attention_quantized" else 0)
    return {"bytes": rows + 2 * q + (4 * units * sum(_merged(case)) if case["merged"] else 0), "flops": 4 * d * case["layers"] * case["q_heads"] * n}


# ---- inputs ------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _keys(gen, shape, dt, gain=8.0):
    """Rows N(0,1), one in a hundred of them `gain` times as long."""
    x = torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)
    if gain != 1.0:
        sink = torch.rand(shape[-2], generator=gen, device=DEVICE) < 0.01
        x *= torch.where(sink, gain, 1.0)[:, None]
    return x.to(dt)


def _padded(lens, starts, width):
    """Where row r of sequence b lies, [batch][width] (rows past the last one: the sequence's first), and whether it is there."""
    at = torch.arange(width, device=DEVICE)[None, :]
    there = at < torch.tensor(lens, device=DEVICE)[:, None]
    return torch.where(there, at, 0) + torch.tensor(starts, device=DEVICE)[:, None], there


def _prefix_sums(x):
    return [int(v) for v in np.concatenate([[0], np.cumsum(x)])]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt, d, lens = _dtype(case), case["head_dim"], _lengths(case)
    layers, hq, hkv, batch = case["layers"], case["q_heads"], case["kv_heads"], case["batch"]
    s = {"case": case, "lens": lens}
    if case.get("slopes"):
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=DEVICE)
    if case["kind"] == "prompt":
        T = sum(lens)
        s["cu"] = _prefix_sums(lens)
        s["K"], s["V"] = _keys(gen, (layers, hkv, T, d), dt), _keys(gen, (layers, hkv, T, d), dt, 1.0)
        for b, spans in enumerate(_spans(case)):
            for i, e, image in spans:
                if image:
                    s["K"][:, :, s["cu"][b] + i:s["cu"][b] + e] += 0.5
                    s["V"][:, :, s["cu"][b] + i:s["cu"][b] + e] += 0.5
        s["Q"] = _keys(gen, (layers, hq, T, d), dt, 1.0)
        width = max(lens)
        s["index"], s["there"] = _padded(lens, s["cu"][:-1], width)
        reach = np.zeros((batch, width), dtype=np.int64)
        for b, r in enumerate(_reach(case)):
            reach[b, :len(r)] = r
        s["reach"] = torch.from_numpy(reach).to(DEVICE)
        return s
    caps = _capacities(case)
    s["cu"] = _prefix_sums(caps)
    C = s["cu"][-1]
    s["cu_blocks"] = _prefix_sums(_blocks(case))
    K, V = _keys(gen, (layers, hkv, C, d), dt), _keys(gen, (layers, hkv, C, d), dt, 1.0)
    if case["kind"] in ("quantize", "attention"):
        s["K"], s["V"] = K, V
    if case["kind"] == "quantize":
        s["cache"] = _empty_cache(s)
    if case["kind"] in ("append", "dequantize", "attention_quantized"):
        s["cache"] = _empty_cache(s)
        _plain_quantize(s, K, V)
    if case["kind"] == "dequantize":
        s["K"], s["V"] = torch.zeros_like(K), torch.zeros_like(V)
    del K, V
    if case["kind"] == "append":
        s["k_new"], s["v_new"] = _keys(gen, (layers, hkv, batch, d), dt), _keys(gen, (layers, hkv, batch, d), dt, 1.0)
    if "attention" in case["kind"]:
        s["q"] = _keys(gen, (layers, hq, batch, d), dt, 1.0)
        s["out"] = torch.empty_like(s["q"])
        s["index"], s["there"] = _padded(lens, s["cu"][:-1], max(lens))
        if case["merged"]:
            # the merged rows' places in a prompt four times as long, ascending, each (layer, kv head) its own
            merged, slots = _merged(case), _prefix_sums(_merged(case))
            pos = torch.zeros((layers, hkv, slots[-1]), dtype=torch.int32, device=DEVICE)
            for b, n in enumerate(merged):
                steps = torch.randint(1, 8, (layers, hkv, n), generator=gen, device=DEVICE, dtype=torch.int32)
                pos[:, :, slots[b]:slots[b + 1]] = torch.cumsum(steps, -1, dtype=torch.int32)
            s["row_pos"], s["slots"], s["merged"] = pos, slots, merged
            s["q_pos"] = [8 * n + (x - n) for n, x in zip(merged, lens)]
    return s


def _empty_cache(s):
    case = s["case"]
    u = (case["layers"], case["kv_heads"])
    codes = [torch.zeros((*u, s["cu"][-1], case["head_dim"]), dtype=torch.float8_e4m3fn, device=DEVICE) for _ in "kv"]
    return codes + [torch.ones((*u, s["cu_blocks"][-1]), dtype=torch.float32, device=DEVICE) for _ in "kv"]


# ---- the plain forms ---------------------------------------------------------------------------------------
def _scale_for(most):
    """The power of two that brings numbers of up to `most` into e4m3's range."""
    m, e = torch.frexp(most)
    k = torch.where(m <= FP8_MOST / 512, e - 9, e - 8).clamp_min(-120)
    return torch.ldexp(torch.ones_like(most), torch.where(most > 0, k, -120))


def _to_fp8(x):
    return x.clamp(-FP8_MOST, FP8_MOST).to(torch.float8_e4m3fn)  # (a NaN stays one)


def _finite_most(x, dims):
    a = x.abs()
    return torch.where(torch.isfinite(a), a, 0.0).amax(dims)


def _block_rows(s):
    """Where the rows of every sequence's blocks lie, [blocks][32], whether they are valid, and the blocks with a valid row."""
    if "block_rows" not in s:
        rows, there, blocks = [], [], []
        for b, n in enumerate(s["lens"]):
            k = -(-n // BLOCK)
            at = np.arange(k * BLOCK).reshape(k, BLOCK)
            rows.append(s["cu"][b] + np.minimum(at, n - 1))
            there.append(at < n)
            blocks.append(s["cu_blocks"][b] + np.arange(k))
        s["block_rows"] = [torch.from_numpy(np.concatenate(x)).to(DEVICE) for x in (rows, there, blocks)]
    return s["block_rows"]


def _plain_quantize(s, K, V):
    rows, there, blocks = _block_rows(s)
    for x, codes, scales in ((K, s["cache"][0], s["cache"][2]), (V, s["cache"][1], s["cache"][3])):
        y = x[:, :, rows].float()  # [layers][kv heads][blocks][32][d]
        sc = _scale_for(_finite_most(torch.where(there[:, :, None], y, 0.0), (-1, -2)))
        y = _to_fp8(y / sc[..., None, None])
        # (bytes: indexed writes know no 8-bit floats)
        codes.view(torch.uint8)[:, :, rows[there]] = y.view(torch.uint8)[:, :, there]
        scales[:, :, blocks] = sc
    return s["cache"]


def _plain_dequantize(s):
    rows, there, blocks = _block_rows(s)
    for x, codes, scales in ((s["K"], s["cache"][0], s["cache"][2]), (s["V"], s["cache"][1], s["cache"][3])):
        y = codes.view(torch.uint8)[:, :, rows].view(torch.float8_e4m3fn).float() * scales[:, :, blocks][..., None, None]
        x[:, :, rows[there]] = y[:, :, there].to(x.dtype)
    return [s["K"], s["V"]]


def _plain_append(s):
    if "append_at" not in s:
        first = [n // BLOCK * BLOCK for n in s["lens"]]
        most = [c - 1 for c in _capacities(s["case"])]
        rows = [[s["cu"][b] + min(f + i, most[b]) for i in range(BLOCK)] for b, f in enumerate(first)]
        s["append_at"] = (torch.tensor(rows, device=DEVICE), torch.tensor([n % BLOCK for n in s["lens"]], device=DEVICE),
                          torch.tensor([s["cu_blocks"][b] + n // BLOCK for b, n in enumerate(s["lens"])], device=DEVICE),
                          torch.tensor([s["cu"][b] + n for b, n in enumerate(s["lens"])], device=DEVICE))
    rows, inside, block, at = s["append_at"]
    older = torch.arange(BLOCK, device=DEVICE)[None, :] < inside[:, None]  # [batch][32]
    for x, codes, scales in ((s["k_new"], s["cache"][0], s["cache"][2]), (s["v_new"], s["cache"][1], s["cache"][3])):
        new = x.float()
        wanted = _scale_for(_finite_most(new, -1))
        had = scales[:, :, block]
        sc = torch.where(inside > 0, torch.maximum(had, wanted), wanted)
        old = codes.view(torch.uint8)[:, :, rows].view(torch.float8_e4m3fn).float()  # [layers][kv heads][batch][32][d]
        old = _to_fp8(old * (had / sc)[..., None, None])
        codes.view(torch.uint8)[:, :, rows[older]] = old.view(torch.uint8)[:, :, older]
        codes.view(torch.uint8)[:, :, at] = _to_fp8(new / sc[..., None]).view(torch.uint8)
        scales[:, :, block] = sc
    return s["cache"]


def _softmax_times(logits, v):
    m = logits.amax(-1, keepdim=True)
    p = logits.sub_(torch.where(torch.isfinite(m), m, 0.0)).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v)
    return torch.where(z > 0, o / z, 0.0)


def _plain_attention(s, k, v):
    """k, v [layers][kv heads][batch][rows][d], fp32."""
    case = s["case"]
    layers, hkv, batch, width, d = k.shape
    G = case["q_heads"] // hkv
    q = s["q"].float().reshape(layers, hkv, G, batch, d).transpose(2, 3).contiguous()  # [layers][kv heads][batch][G][d]
    logits = torch.matmul(q, k.transpose(-1, -2)) * d ** -0.5
    if case["cap"] > 0:
        logits = torch.tanh(logits / case["cap"]) * case["cap"]
    if case["slopes"]:
        logits -= s["slopes"].reshape(1, hkv, 1, G, 1) * _plain_distance(s).abs().unsqueeze(-2).float()
    logits = torch.where(s["there"][None, None, :, None, :], logits, -math.inf)
    o = _softmax_times(logits, v)
    return o.transpose(2, 3).reshape(layers, case["q_heads"], batch, d).to(s["q"].dtype)


def _plain_distance(s):
    """Distance of every cache row from its query, [layers or 1][kv heads or 1][batch][rows]."""
    lens = torch.tensor(s["lens"], device=DEVICE)
    at = torch.arange(max(s["lens"]), device=DEVICE)
    back = (lens[:, None] - 1 - at[None, :])[None, None]
    if not s["case"]["merged"]:
        return back
    merged = torch.tensor(s["merged"], device=DEVICE)
    slot = torch.tensor(s["slots"][:-1], device=DEVICE)[:, None] + torch.minimum(at[None, :], merged[:, None] - 1)
    far = torch.tensor(s["q_pos"], device=DEVICE)[:, None] - s["row_pos"][:, :, slot]
    return torch.where(at[None, :] < merged[:, None], far, back)


def _plain_prompt(s):
    case = s["case"]
    layers, hq, T, d = s["Q"].shape
    hkv, (batch, width) = case["kv_heads"], s["index"].shape
    G = hq // hkv
    # [layers][kv heads][batch] G heads' queries below each other
    q = s["Q"].float()[:, :, s["index"]].reshape(layers, hkv, G, batch, width, d).transpose(2, 3).reshape(layers, hkv, batch, G * width, d)
    k, v = s["K"].float()[:, :, s["index"]], s["V"].float()[:, :, s["index"]]
    logits = torch.matmul(q, k.transpose(-1, -2)).mul_(d ** -0.5).view(layers, hkv, batch, G, width, width)
    if case["cap"] > 0:
        logits.div_(case["cap"]).tanh_().mul_(case["cap"])
    at = torch.arange(width, device=DEVICE)
    if case["slopes"]:
        logits.addcmul_(s["slopes"].reshape(1, hkv, 1, G, 1, 1), (at[:, None] - at[None, :]).abs().float(), value=-1.0)
    hidden = (at[None, None, :] > s["reach"][:, :, None])[:, None]
    logits.masked_fill_(hidden, -math.inf)
    o = _softmax_times(logits.view(layers, hkv, batch, G * width, width), v)
    o = o.view(layers, hkv, batch, G, width, d).transpose(2, 3).reshape(layers, hq, batch, width, d)
    out = torch.empty_like(s["Q"])
    out[:, :, s["index"][s["there"]]] = o[:, :, s["there"]].to(out.dtype)
    return out


# ---- one pass ----------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own_run(s)
    if kind == "quantize":
        return _plain_quantize(s, s["K"], s["V"])
    if kind == "dequantize":
        return _plain_dequantize(s)
    if kind == "append":
        return _plain_append(s)
    if kind == "prompt":
        return _plain_prompt(s)
    if kind == "attention":
        return _plain_attention(s, s["K"][:, :, s["index"]].float(), s["V"][:, :, s["index"]].float())
    # the rows' scales: that of the block a row lies in
    row = torch.arange(s["index"].shape[1], device=DEVICE)[None, :].expand_as(s["index"])
    block = torch.tensor(s["cu_blocks"][:-1], device=DEVICE)[:, None] + torch.where(s["there"], row // BLOCK, 0)
    k, v = (codes.view(torch.uint8)[:, :, s["index"]].view(torch.float8_e4m3fn).float() * scales[:, :, block][..., None]
            for codes, scales in (s["cache"][0::2], s["cache"][1::2]))
    return _plain_attention(s, k, v)


def _own_state(s):
    """What a program keeps of the library beside its tensors: the parameters, the cache's description, a workspace."""
    from paper_2511_05534_amd import binding as fb
    case, h = s["case"], {"fb": fb}
    prompt = case["kind"] == "prompt"
    shape = (case["layers"], case["q_heads"], case["kv_heads"], case["head_dim"], case["dtype"])
    if prompt:
        h["params"] = p = fb.Params(*shape, s["lens"], s["lens"], _spans(case), 1, 0.25, [1.0] * case["batch"])
        h["out"] = torch.empty_like(s["Q"])
        h["workspace_bytes"] = fb.flowmm_plan_sizes(p)[1]
    else:
        caps = _capacities(case)
        merged = s["merged"] if case.get("merged") else s["lens"]
        h["params"] = p = fb.Params(*shape, caps, merged, [[(0, c, 0)] for c in caps], 1, 0.25, [1.0] * case["batch"])
        h["workspace_bytes"] = fb.flowmm_cache_sizes(p, s["cu"])[2]
    h["workspace"] = torch.empty(max(h["workspace_bytes"], 256), dtype=torch.uint8, device=DEVICE)
    if "cache" in s:
        h["cache"] = fb.QuantizedCache(p, s["cu"], tensors=s["cache"])
    h["scoring"] = None
    if prompt:
        prefix = [min(case["prefix"], n) for n in s["lens"]] if case["prefix"] else None
        h["scoring"] = fb.Scoring(cap=case["cap"], slopes=s["slopes"].data_ptr() if case["slopes"] else 0, prefix=prefix, image_spans=bool(case["both_ways"]))
    elif "attention" in case["kind"]:
        h["scoring"] = fb.Scoring(cap=case["cap"], slopes=s["slopes"].data_ptr() if case["slopes"] else 0,
                                  row_pos=s["row_pos"].data_ptr() if case["merged"] else 0, q_pos=s["q_pos"] if case["merged"] else None)
    s["own"] = h
    return h


def _own_run(s):
    h = s.get("own") or _own_state(s)
    fb, p, kind, stream = h["fb"], h["params"], s["case"]["kind"], torch.cuda.current_stream().cuda_stream
    if kind == "quantize":
        fb.flowmm_cache_quantize(p, s["cu"], s["lens"], s["cu"], s["K"].data_ptr(), s["V"].data_ptr(), h["cache"], stream)
        return s["cache"]
    if kind == "dequantize":
        fb.flowmm_cache_dequantize(p, s["cu"], s["lens"], s["cu"], h["cache"], s["K"].data_ptr(), s["V"].data_ptr(), stream)
        return [s["K"], s["V"]]
    if kind == "append":
        fb.flowmm_cache_append_quantized(p, s["cu"], s["lens"], h["cache"], s["k_new"].data_ptr(), s["v_new"].data_ptr(), stream)
        return s["cache"]
    ws = (h["workspace"].data_ptr(), h["workspace_bytes"], stream)
    if kind == "prompt":
        layers, hq, T, d = s["Q"].shape
        fb.flowmm_prompt_attention(p, h["scoring"], s["K"].data_ptr(), s["V"].data_ptr(), s["Q"].data_ptr(), (hq * T * d, T * d, d), h["out"].data_ptr(), *ws)
        return h["out"]
    if kind == "attention":
        fb.flowmm_cache_attention(p, s["cu"], s["lens"], h["scoring"], s["q"].data_ptr(), s["K"].data_ptr(), s["V"].data_ptr(), s["out"].data_ptr(), *ws)
    else:
        fb.flowmm_cache_attention_quantized(p, s["cu"], s["lens"], h["scoring"], s["q"].data_ptr(), h["cache"], s["out"].data_ptr(), *ws)
    return s["out"]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        return [*_exact_blocks(s, s["K"], s["V"])]
    if kind == "append":
        return _exact_append(s)
    if kind == "dequantize":
        k, v = _exact_rows(s)
        outs = [s["K"].double(), s["V"].double()]
        for o, x in zip(outs, (k, v)):
            for b, n in enumerate(s["lens"]):
                o[:, :, s["cu"][b]:s["cu"][b] + n] = x[:, :, s["cu"][b]:s["cu"][b] + n]
        return outs
    return _exact_prompt(s) if kind == "prompt" else _exact_attention(s)


def _nearest_e4m3(x):
    """The e4m3 number nearest to x (|x| <= 448): three bits behind the leading one, steps of 2^-9 at the least."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))).clamp(-6, 8)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_scale(most):
    k = torch.ceil(torch.log2(most.clamp_min(1e-300) / FP8_MOST))
    k = k - (most <= FP8_MOST * torch.exp2(k - 1)).double() + (most > FP8_MOST * torch.exp2(k)).double()  # (a logarithm next to a whole number)
    return torch.exp2(k.clamp_min(-120.0))


def _exact_blocks(s, K, V):
    codes, scales = [x.double() for x in s["cache"][:2]], [x.double() for x in s["cache"][2:]]
    for x, c, sc in zip((K, V), codes, scales):
        for b, n in enumerate(s["lens"]):
            for g in range(x.shape[1]):
                rows = x[:, g, s["cu"][b]:s["cu"][b] + n].double()
                k = -(-n // BLOCK)
                most = torch.nn.functional.pad(rows.abs().amax(-1), (0, k * BLOCK - n)).view(-1, k, BLOCK).amax(-1)
                got = _exact_scale(most)
                sc[:, g, s["cu_blocks"][b]:s["cu_blocks"][b] + k] = got
                c[:, g, s["cu"][b]:s["cu"][b] + n] = _nearest_e4m3(rows / got.repeat_interleave(BLOCK, -1)[:, :n, None])
    return codes + scales


def _exact_append(s):
    codes, scales = [x.double() for x in s["cache"][:2]], [x.double() for x in s["cache"][2:]]
    for x, c, sc in zip((s["k_new"], s["v_new"]), codes, scales):
        for b, n in enumerate(s["lens"]):
            row, blk, first = s["cu"][b] + n, s["cu_blocks"][b] + n // BLOCK, s["cu"][b] + n // BLOCK * BLOCK
            new = x[:, :, b].double()
            want = _exact_scale(new.abs().amax(-1))
            if n % BLOCK:
                had = sc[:, :, blk].clone()
                want = torch.maximum(had, want)
                c[:, :, first:row] = _nearest_e4m3(c[:, :, first:row] * (had / want)[:, :, None, None])
            sc[:, :, blk] = want
            c[:, :, row] = _nearest_e4m3(new / want[:, :, None])
    return codes + scales


def _exact_rows(s):
    """The numbers that an 8-bit cache stands for, in the cache's layout."""
    got = []
    for codes, scales in (s["cache"][0::2], s["cache"][1::2]):
        x = codes.double()
        for b, n in enumerate(s["lens"]):
            k = -(-n // BLOCK)
            sc = scales[:, :, s["cu_blocks"][b]:s["cu_blocks"][b] + k].double().repeat_interleave(BLOCK, -1)[:, :, :n]
            x[:, :, s["cu"][b]:s["cu"][b] + n] *= sc[..., None]
        got.append(x)
    return got


def _exact_softmax(case, logits, slope, distance, hidden):
    if case["cap"] > 0:
        logits = case["cap"] * torch.tanh(logits / case["cap"])
    if case["slopes"]:
        logits = logits - slope * distance
    if hidden is not None:
        logits = logits.masked_fill(hidden, -math.inf)
    return torch.softmax(logits, -1)


def _exact_attention(s):
    case = s["case"]
    K, V = _exact_rows(s) if case["kind"] == "attention_quantized" else (s["K"], s["V"])
    G, d = case["q_heads"] // case["kv_heads"], case["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lens"]):
        rows = slice(s["cu"][b], s["cu"][b] + n)
        far = (n - 1 - torch.arange(n, device=DEVICE)).double()
        for l in range(case["layers"]):
            for g in range(case["kv_heads"]):
                if case["merged"]:
                    m = s["merged"][b]
                    far = far.clone()
                    far[:m] = (s["q_pos"][b] - s["row_pos"][l, g, s["slots"][b]:s["slots"][b] + m]).double().abs()
                q = s["q"][l, g * G:(g + 1) * G, b].double()
                slope = s["slopes"][g * G:(g + 1) * G, None].double() if case["slopes"] else None
                p = _exact_softmax(case, q @ K[l, g, rows].double().T / math.sqrt(d), slope, far, None)
                out[l, g * G:(g + 1) * G, b] = p @ V[l, g, rows].double()
    return out


def _exact_prompt(s):
    case = s["case"]
    G, d = case["q_heads"] // case["kv_heads"], case["head_dim"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lens"]):
        rows = slice(s["cu"][b], s["cu"][b] + n)
        i = torch.arange(n, device=DEVICE)
        hidden = i[None, :] > s["reach"][b, :n, None]
        far = (i[:, None] - i[None, :]).abs().double() if case["slopes"] else None
        for l in range(case["layers"]):
            for h in range(case["q_heads"]):
                logits = s["Q"][l, h, rows].double() @ s["K"][l, h // G, rows].double().T / math.sqrt(d)
                p = _exact_softmax(case, logits, s["slopes"][h].double() if case["slopes"] else None, far, hidden)
                out[l, h, rows] = p @ s["V"][l, h // G, rows].double()
    return out
