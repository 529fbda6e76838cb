"""Operators of language models in 4 bits beside the denoiser's own: what a program that serves a decoder on the same card calls.

  norm    h = x + residual and the root-mean-square norm of h, in bf16 or in E4M3 with a scale per row
          (lvx_rmsnorm_residual, lvx_rmsnorm_residual_fp8)
  linear  a product with E2M1 weights that have an E8M0 scale per 32 input channels, for bf16 rows or E4M3 rows with a scale each
          (lvx_linear_fp4, lvx_linear_fp8_fp4)
  append  new keys and values of all sequences into the 4-bit cache, and the layer read back (lvx_kv4_append, lvx_kv4_gather)
  attend  attention of the new tokens' grouped heads over the 4-bit cache (lvx_kv4_attention)

The 4-bit values are E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, nearest, ties to the even code.  Weights and keys: groups of 32
channels share 2^e with the smallest e >= -120 for which the group's largest magnitude is at most 7 * 2^e.  Values: the head's vector
shares s = max(bf16(largest magnitude / 6), 2^-120).
"""
import math

import torch

own = False

DEV = "cuda:0"
EPI = {"store": 0, "gelu": 1, "resid": 2, "resid32": 3}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
SMALLEST = 2.0 ** -120


def _norm(n, d, stream32, fp8):
    return dict(kind="norm", n=n, d=d, stream32=stream32, fp8=fp8)


def _linear(m, n, k, fp8, epi):
    return dict(kind="linear", m=m, n=n, k=k, fp8=fp8, epi=epi)


def _append(seqs, tokens, kv_heads, d, ragged):
    return dict(kind="append", seqs=seqs, tokens=tokens, kv_heads=kv_heads, d=d, ragged=ragged)


def _attend(seqs, tokens, keys, heads, kv_heads, d, causal, ragged):
    return dict(kind="attend", seqs=seqs, tokens=tokens, keys=keys, heads=heads, kv_heads=kv_heads, d=d, causal=causal, ragged=ragged)


def listed():
    return [
        # one sequence, one new token: nothing but latency
        dict(_norm(1, 5120, False, False), name="norm_token"),
        # a batch of ragged prompts of a small model, 8-bit rows for the linear behind
        dict(_norm(777, 1280, False, True), name="norm_small_fp8"),
        # as many tokens as a chunk has, fp32 residual stream, 8-bit rows
        dict(_norm(4680, 5120, True, True), name="norm_chunk_fp8"),
        # the fused q | k | v projection of one token: the weights are read once
        dict(_linear(1, 15360, 5120, False, "store"), name="linear_token"),
        # sixteen sequences decoded together, the wide projection with its activation
        dict(_linear(16, 13824, 5120, True, "gelu"), name="linear_batch_fp8"),
        # sizes that are no multiple of a tile, into the fp32 residual stream
        dict(_linear(37, 2568, 1184, False, "resid32"), name="linear_odd"),
        # a prompt: the product is bound by the matrix cores
        dict(_linear(544, 5120, 13824, True, "resid"), name="linear_prompt_fp8"),
        # prompts of four sequences enter the cache
        dict(_append(4, 1560, 8, 128, True), name="append_prompts"),
        # one sequence, one token
        dict(_attend(1, 1, 4680, 40, 8, 128, True, False), name="attend_token"),
        # a batch of sequences of different lengths, one of them idle
        dict(_attend(32, 1, 24960, 40, 8, 128, True, True), name="attend_batch"),
        # a few tokens each (a speculative step), small heads, odd lengths, every key visible
        dict(_attend(5, 7, 1301, 12, 4, 64, False, True), name="attend_odd"),
        # a long prompt's next part
        dict(_attend(1, 1560, 24960, 40, 8, 128, True, False), name="attend_prompt"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "linear", "linear", "append", "attend", "attend"))
    if kind == "norm":
        d = 16 * _log(rng, 8, 512)
        return _norm(max(1, min(_log(rng, 1, 8192), (4680 * 5120) // d)), d, rng.random() < 0.5, rng.random() < 0.5)
    if kind == "linear":
        n, k = 8 * _log(rng, 8, 1728), 32 * _log(rng, 4, 432)
        return _linear(_log(rng, 1, 544), n, k, rng.random() < 0.5, rng.choice(tuple(EPI)))
    kv, d = rng.choice((1, 2, 4, 5, 8)), rng.choice((64, 128))
    if kind == "append":
        seqs = _log(rng, 1, 32)
        return _append(seqs, max(1, _log(rng, 1, 6240) // seqs), kv, d, rng.random() < 0.5)
    seqs = _log(rng, 1, 32)
    tokens = 1 if rng.random() < 0.5 else _log(rng, 2, 1024)
    heads = kv * rng.choice((1, 2, 3, 4, 5, 7, 8))
    tokens = max(1, min(tokens, 1560 * 40 // (seqs * max(heads, 40))))
    keys = max(tokens, _log(rng, 16, 24960))
    return _attend(seqs, tokens, keys, heads, kv, d, rng.random() < 0.7, rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------------------------------------------------
def _lengths(most, seqs, ragged):
    """Lengths from `most` down to a quarter of it; the second sequence of a larger ragged batch is idle."""
    if not ragged:
        return [most] * seqs
    return [0 if s == 1 and seqs >= 4 else most - (most - most // 4 - 1) * s // max(1, seqs - 1) for s in range(seqs)]


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2 + 1)
    s, kind = {}, case["kind"]
    if kind == "norm":
        n, d = case["n"], case["d"]
        s["x"] = _normal(g, n, d).to(torch.bfloat16)
        r = _normal(g, n, d) * torch.exp(0.5 * _normal(g, d)) * 3
        s["resid"] = r if case["stream32"] else r.to(torch.bfloat16)
        s["gain"] = 1 + 0.2 * _normal(g, d)
    elif kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        a = _normal(g, m, k) * torch.exp(0.5 * _normal(g, k))
        s["w"] = (_normal(g, n, k) * torch.exp(0.3 * _normal(g, n, 1)) / math.sqrt(k)).to(torch.bfloat16)
        if case["fp8"]:
            s["a_scale"] = a.abs().amax(1) / 448
            s["a"] = (a / s["a_scale"][:, None]).to(torch.float8_e4m3fn)
        else:
            s["a"] = a.to(torch.bfloat16)
        if case["epi"].startswith("resid"):
            r = 2 * _normal(g, m, n)
            s["resid"] = r if case["epi"] == "resid32" else r.to(torch.bfloat16)
            s["gate"] = 1 + 0.2 * _normal(g, n)
    else:
        S, KV, D = case["seqs"], case["kv_heads"], case["d"]
        L = case["tokens"] if kind == "append" else case["keys"]
        wide = torch.exp(0.7 * _normal(g, KV, D))  # some channels of the keys are much larger than others
        s["k"] = torch.empty(S, L, KV, D, dtype=torch.bfloat16, device=DEV)
        s["v"] = torch.empty_like(s["k"])
        for i in range(S):
            s["k"][i] = _normal(g, L, KV, D) * wide
            s["v"][i] = _normal(g, L, KV, D)
        counts = _lengths(L, S, case["ragged"])
        tokens = counts if kind == "append" else [min(case["tokens"], max(c, 1)) for c in counts]
        s["starts"] = torch.tensor([0] + tokens, device=DEV).cumsum(0).to(torch.int32)
        s["counts"] = torch.tensor(counts, dtype=torch.int32, device=DEV)
        s["tokens"] = sum(tokens)
        if kind == "attend":
            s["q"] = _normal(g, s["tokens"], case["heads"] * D).to(torch.bfloat16)
    return s


# ---- the plain form ---------------------------------------------------------------------------------------------------------------------
def _codes(x, scale):
    """E2M1 codes of x / scale (sign in bit 3): how many of the borders between the levels lie below."""
    a, b = x.abs(), scale
    up = (a > 0.25 * b).to(torch.uint8) + (a >= 0.75 * b) + (a > 1.25 * b) + (a >= 1.75 * b) + (a > 2.5 * b) + (a >= 3.5 * b) + (a > 5.0 * b)
    return up | (torch.signbit(x).to(torch.uint8) << 3)


def _level(codes):
    return torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)[codes.int()]


def _packed(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpacked(packed):
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2)


def _group_scale(x):
    """E8M0 byte of each 32 channels: 2^e, e the smallest with max |x| <= 7 * 2^e."""
    m, e = torch.frexp(x.float().unflatten(-1, (-1, 32)).abs().amax(-1))
    e = torch.where(m <= 0.875, e - 3, e - 2)
    return (torch.where(m == 0, torch.full_like(e, -120), e.clamp(min=-120)) + 127).to(torch.uint8)


def _power(bytes_):
    return torch.ldexp(torch.ones((), device=bytes_.device), bytes_.int() - 127)


def _quantised(x):
    """bf16 rows -> packed E2M1 codes and E8M0 bytes of each 32."""
    e = _group_scale(x)
    return _packed(_codes(x.float(), _power(e).repeat_interleave(32, -1))), e


def _decoded(packed, e):
    return _level(_unpacked(packed)) * _power(e).repeat_interleave(32, -1)


def _quantised_values(v):
    s = (v.float().abs().amax(-1, keepdim=True) / 6).to(torch.bfloat16).float().clamp(min=SMALLEST)
    return _packed(_codes(v.float(), s)), s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"], kind = case, case["kind"]
    if kind == "norm":
        s["sum"] = torch.empty_like(s["resid"])
        s["y"] = torch.empty(case["n"], case["d"], dtype=torch.uint8 if case["fp8"] else torch.bfloat16, device=DEV)
        s["scale"] = torch.empty(case["n"], device=DEV)
    elif kind == "linear":
        s["w"], s["w_scale"] = _quantised(s.pop("w"))  # the weights that the program holds
        s["c"] = torch.empty(case["m"], case["n"], dtype=torch.float32 if case["epi"] == "resid32" else torch.bfloat16, device=DEV)
    elif own:
        import paper_2512_04677_amd as lvx
        S, KV, D, L = case["seqs"], case["kv_heads"], case["d"], case["tokens" if kind == "append" else "keys"]
        s["cache"] = lvx.KV4Cache(lvx.kv4_desc(1, S, KV, D, L), DEV)
        if kind == "attend":
            # a slot holds keys behind its sequence's last one: those of the request before
            whole = torch.full((S,), L, dtype=torch.int32, device=DEV)
            lvx.lvx_kv4_append(s["cache"], 0, s.pop("k").view(S * L, KV * D), s.pop("v").view(S * L, KV * D), whole, max_tokens=L)
            s["out"] = torch.empty_like(s["q"])
            s["workspace"] = torch.empty(lvx.lvx_kv4_attention_workspace_bytes(s["cache"], case["heads"], case["tokens"]), dtype=torch.uint8, device=DEV)
        else:
            s["k_out"], s["v_out"] = (torch.empty(S, L, KV * D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    elif kind == "attend":
        s["kq"], s["ks"] = _quantised(s.pop("k").transpose(1, 2).contiguous())  # [seq][kv head][key][...]
        s["vq"], s["vs"] = _quantised_values(s.pop("v").transpose(1, 2).contiguous())
    if kind == "append":  # the new tokens' rows, one sequence behind the other
        keep = (torch.arange(case["tokens"], device=DEV)[None, :] < s["counts"][:, None]).flatten()
        s["k"], s["v"] = (s[n].flatten(0, 1)[keep].flatten(1).contiguous() for n in "kv")
    return s


def _gelu(x):
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


def _rows(starts, most):
    """[sequence][most]: the packed row of each token, and which of them there are."""
    i = torch.arange(most, device=starts.device)[None, :]
    first, n = starts[:-1, None].long(), (starts[1:] - starts[:-1])[:, None].long()
    return first + torch.minimum(i, (n - 1).clamp(min=0)), i < n


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        h = s["x"].float() + s["resid"].float()
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6) * s["gain"]
        if not case["fp8"]:
            return {"sum": h.to(s["resid"].dtype), "y": y.to(torch.bfloat16)}
        most = y.abs().amax(1, keepdim=True)
        return {"sum": h.to(s["resid"].dtype), "y": (y * (448 / most)).to(torch.float8_e4m3fn), "scale": most[:, 0] / 448}
    if kind == "linear":
        c = s["a"].float() @ _decoded(s["w"], s["w_scale"]).T
        if case["fp8"]:
            c = c * s["a_scale"][:, None]
        if case["epi"] == "gelu":
            c = _gelu(c)
        elif case["epi"].startswith("resid"):
            c = s["resid"].float() + s["gate"] * c
        return c.to(s["c"].dtype)
    if kind == "append":
        k, e = _quantised(s["k"])
        v, sv = _quantised_values(s["v"].unflatten(1, (case["kv_heads"], case["d"])))
        rows, there = _rows(s["starts"], case["tokens"])
        blank = there[:, :, None]
        back = (_decoded(k, e), (_level(_unpacked(v)) * sv).flatten(1))
        return [torch.where(blank, x[rows], torch.zeros((), device=x.device)).to(torch.bfloat16) for x in back]
    S, KV, D, L = case["seqs"], case["kv_heads"], case["d"], case["keys"]
    H, Q = case["heads"], case["tokens"]
    rows, there = _rows(s["starts"], Q)
    q = s["q"].float()[rows].view(S, Q, KV, H // KV, D).permute(0, 2, 1, 3, 4).reshape(S, KV, Q * (H // KV), D)
    k, v = _decoded(s["kq"], s["ks"]), _level(_unpacked(s["vq"])) * s["vs"]
    n = (s["starts"][1:] - s["starts"][:-1])[:, None]
    seen = s["counts"][:, None] - (n - 1 - torch.arange(Q, device=q.device)[None, :] if case["causal"] else 0 * n)
    seen = seen.expand(S, Q)[:, None, :, None].expand(S, 1, Q, H // KV).reshape(S, 1, Q * (H // KV), 1)
    x = torch.matmul(q, k.transpose(-1, -2)) * (1 / math.sqrt(D))
    x = x.masked_fill_(torch.arange(L, device=q.device) >= seen, -math.inf)
    p = torch.exp_(x.sub_(x.amax(-1, keepdim=True).clamp(min=-1e30)))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.view(S, KV, Q, H // KV, D).permute(0, 2, 1, 3, 4).reshape(S * Q, H * D)
    return o[there.flatten()].to(torch.bfloat16)


# ---- one pass ---------------------------------------------------------------------------------------------------------------------------
def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_2512_04677_amd as lvx
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        if case["fp8"]:
            lvx.lvx_rmsnorm_residual_fp8(s["x"], s["resid"], s["gain"], 1e-6, s["y"], s["scale"], sum_out=s["sum"])
            return {"sum": s["sum"], "y": s["y"].view(torch.float8_e4m3fn), "scale": s["scale"]}
        lvx.lvx_rmsnorm_residual(s["x"], s["resid"], s["gain"], 1e-6, s["y"], sum_out=s["sum"])
        return {"sum": s["sum"], "y": s["y"]}
    if kind == "linear":
        epi, resid, gate = EPI[case["epi"]], s.get("resid"), s.get("gate")
        if case["fp8"]:
            lvx.lvx_linear_fp8_fp4(s["a"].view(torch.uint8), s["a_scale"], s["w"], s["w_scale"], s["c"], epi, resid=resid, gate=gate)
        else:
            lvx.lvx_linear_fp4(s["a"], s["w"], s["w_scale"], s["c"], epi, resid=resid, gate=gate)
        return s["c"]
    if kind == "append":
        lvx.lvx_kv4_append(s["cache"], 0, s["k"], s["v"], s["counts"], starts=s["starts"], max_tokens=case["tokens"])
        lvx.lvx_kv4_gather(s["cache"], 0, s["counts"], s["k_out"], s["v_out"])
        return [s["k_out"], s["v_out"]]
    lvx.lvx_kv4_attention(s["cache"], 0, s["q"], case["heads"], 1 / math.sqrt(case["d"]), s["counts"], s["out"], s["workspace"], starts=s["starts"],
                          max_tokens=case["tokens"], causal=case["causal"])
    return s["out"]


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, d, stream = case["n"], case["d"], 4 if case["stream32"] else 2
        return {"bytes": n * d * (2 + 2 * stream + (1 if case["fp8"] else 2)) + 4 * d + 4 * n * case["fp8"], "flops": 6 * n * d}
    if kind == "linear":
        m, n, k, c = case["m"], case["n"], case["k"], 4 if case["epi"] == "resid32" else 2
        a = m * k + 4 * m if case["fp8"] else 2 * m * k
        resid = case["epi"].startswith("resid")
        return {"bytes": n * k // 2 + n * k // 32 + a + m * n * c * (2 if resid else 1) + 4 * n * resid, "flops": 2 * m * n * k}
    KV, D = case["kv_heads"], case["d"]
    key = KV * (D // 2 + D // 32 + D // 2 + 2)  # bytes of a key and its value
    if kind == "append":
        n = sum(_lengths(case["tokens"], case["seqs"], case["ragged"]))
        return {"bytes": n * (4 * KV * D + 2 * key) + case["seqs"] * case["tokens"] * 4 * KV * D, "flops": 8 * n * KV * D}
    counts = _lengths(case["keys"], case["seqs"], case["ragged"])
    tokens = [min(case["tokens"], max(c, 1)) for c in counts]
    pairs = sum(t * c - (t * (t - 1) // 2 if case["causal"] and c else 0) for t, c in zip(tokens, counts))
    return {"bytes": sum(counts) * key + 4 * sum(tokens) * case["heads"] * D, "flops": 4 * D * case["heads"] * pairs}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------------------
def _nearest(x, step):
    """x / step rounded to the nearest level, times step: within a binade the levels are evenly spaced, so rint does it."""
    r = (x / step).abs()
    gap = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0)).to(r.dtype)
    return torch.sign(x) * (torch.round(r / gap) * gap).clamp(max=6.0) * step


def _exact_groups(x):
    x = x.double()
    g = x.unflatten(-1, (-1, 32))
    most = g.abs().amax(-1, keepdim=True).clamp(min=SMALLEST)
    return _nearest(g, torch.exp2(torch.ceil(torch.log2(most / 7)).clamp(min=-120))).flatten(-2)


def _exact_values(v):
    v = v.double()
    s = (v.abs().amax(-1, keepdim=True) / 6).float().to(torch.bfloat16).double().clamp(min=SMALLEST)
    return _nearest(v, s)


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "norm":
        h = s["x"].double() + s["resid"].double()
        y = s["gain"].double() * h * (h.pow(2).sum(1, keepdim=True) / case["d"] + 1e-6).rsqrt()
        if not case["fp8"]:
            return {"sum": h, "y": y}
        most = y.abs().max(1, keepdim=True).values
        return {"sum": h, "y": y * 448 / most, "scale": most.squeeze(1) / 448}
    if kind == "linear":
        a = s["a"].double() * s["a_scale"].double().unsqueeze(1) if case["fp8"] else s["a"].double()
        c = torch.mm(a, _exact_groups(s["w"]).t())
        if case["epi"] == "gelu":
            return c * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (c + 0.044715 * c * c * c))
        return s["resid"].double() + c * s["gate"].double() if "resid" in s else c
    counts = s["counts"].tolist()
    if kind == "append":
        k, v = _exact_groups(s["k"]), _exact_values(s["v"])
        for i, c in enumerate(counts):
            k[i, c:], v[i, c:] = 0, 0
        return [k.flatten(2), v.flatten(2)]
    starts, D, group = s["starts"].tolist(), case["d"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["tokens"], case["heads"], D, dtype=torch.float64, device=DEV)
    for i, c in enumerate(counts):
        if c == 0:
            continue
        k, v = _exact_groups(s["k"][i, :c]), _exact_values(s["v"][i, :c])
        q = s["q"][starts[i]:starts[i + 1]].double().view(-1, case["heads"], D)
        n = q.shape[0]
        hide = torch.zeros(n, c, dtype=torch.bool, device=DEV)
        if case["causal"]:
            hide = torch.ones(n, c, dtype=torch.bool, device=DEV).triu(c - n + 1)
        for h in range(case["heads"]):
            x = torch.mm(q[:, h], k[:, h // group].t()) / math.sqrt(D)
            out[starts[i]:starts[i + 1], h] = torch.mm(torch.softmax(x.masked_fill(hide, -math.inf), 1), v[:, h // group])
    return out.flatten(1)
