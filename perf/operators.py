"""Operators around the sparse FFN of a decode step, as cases whose time is measured:

  linear    a projection whose weights are held in 4 bits with a scale per group of inputs (prox_w4_linear)
  ffn       Stage 2 of the sparse FFN, for a given channel mask, over weights in 4 bits (prox_w4_stage2_ffn)
  logprobs  log probabilities of given tokens, entropy and top alternatives from logits (prox_token_logprobs)

`run` computes them in plain torch operations in 32 bits, or, where `own` is true, by the library's calls.

A weight matrix [rows, cols] in 4 bits is a triple: codes uint8 [rows, cols / 2] (byte i: column 2i in the low
four bits, column 2i + 1 in the high ones), scales fp16 [rows, groups], zeros uint8 [rows, groups] or None (8
everywhere); a weight is scale * (code - zero).  A group is `group` consecutive columns, or the row where it is 0.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_CODES = {"bf16": 0, "fp32": 1, "fp16": 2}                   # as the library numbers them


def _linear(name, N, K, group, B, zeros=False, x="bf16", y="bf16"):
    return {"name": name, "op": "linear", "N": N, "K": K, "group": group, "B": B, "zeros": zeros, "x": x, "y": y}


def _ffn(name, D, F, k2, group, B, counts=False, y="bf16"):
    return {"name": name, "op": "ffn", "D": D, "F": F, "k2": k2, "group": group, "B": B, "counts": counts, "y": y}


def _logprobs(name, T, V, given, top, x="bf16", temperature=1.0, pad=0, masked=0.0):
    return {"name": name, "op": "logprobs", "T": T, "V": V, "given": given, "top": top, "x": x, "temperature": temperature,
            "pad": pad, "masked": masked}


def listed():
    return [
        # A projection of a small model, one token: nothing but latency.
        _linear("linear_small", 1024, 1024, 128, 1),
        # A projection of a mid-sized model while one sequence is decoded; a checkpoint with zero points.
        _linear("linear_proj", 4096, 4096, 128, 1, zeros=True),
        # The down projection of a dense FFN for eight sequences: long rows.
        _linear("linear_long_b8", 4096, 14336, 128, 8),
        # The head of a model with a large vocabulary, one token, logits in fp32: the weights alone fill the time.
        _linear("linear_head", 131072, 4096, 128, 1, y="fp32"),
        # Odd sizes, small groups, fp16: a checkpoint of another maker, three drafted tokens.
        _linear("linear_odd", 5003, 1376, 32, 3, zeros=True, x="fp16", y="fp16"),
        # A draft model's FFN: latency again.
        _ffn("ffn_toy", 512, 1536, 461, 0, 1, y="fp32"),
        # The headline FFN at 70 % sparsity, one token.
        _ffn("ffn_8b", 4096, 12288, 2867, 128, 1),
        # Four tokens whose masks come from calibrated thresholds: lists of different lengths, one of them empty.
        _ffn("ffn_threshold_b4", 4096, 14336, 3345, 128, 4, counts=True, y="fp32"),
        # A large model's FFN at the largest batch, every token with a mask of its own.
        _ffn("ffn_70b_b8", 8192, 28672, 6690, 128, 8),
        # A decode step's logits, the sampled token and the twenty likeliest beside it: one row, the whole card.
        _logprobs("logprobs_step", 1, 131072, 1, 20),
        # Scoring choices: a few positions, four answer tokens each, a vocabulary that is no multiple of anything.
        _logprobs("logprobs_choices", 37, 50001, 4, 5, x="fp32", temperature=0.7, pad=3, masked=0.2),
        # Perplexity over a window of text: one given token a row, no alternatives.
        _logprobs("logprobs_window", 2048, 131072, 1, 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges.  linear: 16 .. 131072 outputs, 32 .. 16384 inputs (multiples of 32), 1 .. 32
    tokens, every group size and type.  ffn: d_model 256 .. 8192, d_ff 2.5 to 4 times that, 1 .. 8 tokens, 5 % to 60 % of
    the channels kept.  logprobs: 1 .. 4096 rows, 1000 .. 262144 logits."""
    most = {"linear": 131072 * 4096, "ffn": 8192 * 28672, "logprobs": 2048 * 131072}
    op = rng.choice(["linear", "linear", "ffn", "logprobs"])
    if op == "linear":
        N, K = _log_int(rng, 16, 131072), 32 * _log_int(rng, 1, 512)
        B = rng.choice([1, 1, 1, 2, 3, 4, 5, 7, 8, 11, 16, 25, 32])
        N = max(16, min(N, most[op] // (K * max(1, B // 4))))
        x = rng.choice(["bf16", "bf16", "fp16"])
        case = _linear("", N, K, rng.choice([0, 32, 64, 128, 128]), B, rng.random() < 0.5, x, rng.choice([x, "fp32"]))
    elif op == "ffn":
        D = 128 * _log_int(rng, 2, 64)
        F = min(28672, 64 * round(D * rng.uniform(2.5, 4.0) / 64))
        case = _ffn("", D, F, max(1, int(F * rng.uniform(0.05, 0.6))), rng.choice([0, 128]), rng.choice([1, 1, 1, 2, 3, 4, 5, 6, 7, 8]),
                    rng.random() < 0.3, rng.choice(["bf16", "fp32"]))
    else:
        V = _log_int(rng, 1000, 262144)
        top = rng.choice([0, 1, 5, 20, 32])
        T = _log_int(rng, 1, min(4096, most[op] // V // (8 if top else 1)))
        x = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        T = max(1, T // 2) if x == "fp32" else T
        case = _logprobs("", T, V, rng.choice([0, 1, 1, 4, 9]), top, x, rng.choice([1.0, 0.7, 1.3]), rng.choice([0, 0, 1, 8]),
                         rng.choice([0.0, 0.2]))
        if not case["given"] and not top:
            case["given"] = 1
    del case["name"]
    return case


def _groups(cols, group):
    return -(-cols // group) if group else 1


def _quantize(w, group, with_zeros):
    """codes, scales, zeros of w (fp32): round to nearest, symmetric in -7 .. 7, or over the group's range with a zero point."""
    rows, cols = w.shape
    n, width = _groups(cols, group), group or cols
    padded = torch.nn.functional.pad(w, (0, n * width - cols)).view(rows, n, width)
    if with_zeros:
        lo, hi = padded.amin(2, keepdim=True).clamp_(max=0), padded.amax(2, keepdim=True).clamp_(min=0)
        scale = ((hi - lo) / 15).clamp_(min=1e-6).half().float()
        zero = (-lo / scale).round_().clamp_(0, 15)
        code = ((padded / scale).round_() + zero).clamp_(0, 15)
        zeros = zero.view(rows, n).to(torch.uint8)
    else:
        scale = (padded.abs().amax(2, keepdim=True) / 7).clamp_(min=1e-6).half().float()
        code = (padded / scale).round_().clamp_(-7, 7) + 8
        zeros = None
    code = code.view(rows, n * width)[:, :cols].to(torch.uint8)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), scale.view(rows, n).half(), zeros


def _weights(gen, rows, cols, group, zeros=False):
    """Normal weights, with the deviation that keeps the products near 1."""
    parts = []
    step = max(1, (1 << 28) // cols)
    for r in range(0, rows, step):
        w = torch.empty(min(step, rows - r), cols, device="cuda").normal_(0.0, 0.96 / math.sqrt(cols), generator=gen)
        parts.append(_quantize(w, group, zeros))
    return tuple(torch.cat([p[i] for p in parts]) if parts[0][i] is not None else None for i in range(3))


def _tokens(gen, B, D, dtype):
    """Inputs while decoding: Laplace(0, 1), and 0.5 % of the channels 30 times larger in every token."""
    u = torch.rand(B, D, device="cuda", generator=gen, dtype=torch.float64).clamp_(1e-12, 1 - 1e-12)
    x = torch.where(u < 0.5, torch.log(2 * u), -torch.log(2 - 2 * u))
    x[:, torch.randperm(D, device="cuda", generator=gen)[: max(1, D // 200)]] *= 30.0
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}
    if case["op"] == "linear":
        st["w"] = _weights(gen, case["N"], case["K"], case["group"], case["zeros"])
        st["x"] = _tokens(gen, case["B"], case["K"], _DTYPES[case["x"]])
        st["y"] = torch.empty(case["B"], case["N"], dtype=_DTYPES[case["y"]], device="cuda")
    elif case["op"] == "ffn":
        D, F, B, k2 = case["D"], case["F"], case["B"], case["k2"]
        st["gate"], st["up"], st["down_t"] = (_weights(gen, F, D, case["group"]) for _ in range(3))
        st["x"] = _tokens(gen, B, D, torch.bfloat16)
        kept = torch.rand(B, F, device="cuda", generator=gen).argsort(1)[:, :k2].sort(1).values
        st["sel"], st["count"] = kept.to(torch.int32).contiguous(), None
        if case["counts"]:                                   # from k2 / 2 to k2 channels; the second token keeps none
            st["count"] = torch.randint(k2 - k2 // 2, k2 + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
            st["count"][1:2] = 0
        st["y"] = torch.empty(B, D, dtype=_DTYPES[case["y"]], device="cuda")
        if own:
            from paper_2607_27591_b200 import binding as pb
            st["workspace"] = torch.empty(pb.prox_w4_stage2_workspace(D, F, B), dtype=torch.uint8, device="cuda")
    else:
        T, V, stride = case["T"], case["V"], case["V"] + case["pad"]
        x = torch.empty(T, stride, dtype=_DTYPES[case["x"]], device="cuda")
        step = max(1, (1 << 28) // stride)
        for r in range(0, T, step):                          # a few likely tokens over a broad floor, as a head gives them
            z = torch.empty(min(step, T - r), stride, device="cuda").normal_(0.0, 2.0, generator=gen)
            z += torch.empty_like(z).exponential_(1.0, generator=gen)
            if case["masked"]:                               # tokens that a grammar or a filter forbids
                z.masked_fill_(torch.rand(z.shape, device="cuda", generator=gen) < case["masked"], -math.inf)
            z[:, 0] = 1.0
            x[r:r + step] = z
        st["x"] = x[:, :V]
        st["given"] = torch.randint(0, V, (T, case["given"]), device="cuda", generator=gen, dtype=torch.int32)
        for key, n, dtype in (("logprob", case["given"], torch.float32), ("top_logprob", case["top"], torch.float32),
                              ("top_index", case["top"], torch.int32)):
            st[key] = torch.empty(T, n, dtype=dtype, device="cuda")
        st["entropy"] = torch.empty(T, dtype=torch.float32, device="cuda")
    return st


def _values(w, group):
    """The weights that a triple stands for, in fp32."""
    codes, scales, zeros = w
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    width = group or q.shape[-1]
    spread = lambda t: t.float().repeat_interleave(width, -1)[..., : q.shape[-1]]
    return spread(scales) * (q - (8.0 if zeros is None else spread(zeros)))


def _rows(w, index):
    return tuple(None if t is None else t[index] for t in w)


def _plain_ffn(st):
    case, sel = st["case"], st["sel"].long()
    x, group = st["x"].float(), case["group"]
    g = torch.matmul(_values(_rows(st["gate"], sel), group), x.unsqueeze(-1)).squeeze(-1)
    u = torch.matmul(_values(_rows(st["up"], sel), group), x.unsqueeze(-1)).squeeze(-1)
    h = u * g / (1.0 + torch.exp(-g))
    if st["count"] is not None:
        h = h * (torch.arange(case["k2"], device=h.device) < st["count"].unsqueeze(1))
    y = torch.matmul(h.unsqueeze(1), _values(_rows(st["down_t"], sel), group)).squeeze(1)
    return y.to(_DTYPES[case["y"]])


def _plain_logprobs(st):
    case, raw = st["case"], st["x"].float()
    z = raw / case["temperature"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    seen = torch.where(e > 0, z - lse, 0.0)
    entropy = -(e * seen).sum(1) / total[:, 0]
    logprob = z.gather(1, st["given"].long()) - lse
    bits = (raw + 0.0).view(torch.int32).long()              # an order of whole numbers: value first, then the lower index
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 20) - torch.arange(case["V"], device=raw.device)
    top = order.topk(case["top"], dim=1).indices
    return {"logprob": logprob, "entropy": entropy, "top_logprob": z.gather(1, top) - lse, "top_index": top.to(torch.int32)}


def run(st):
    case = st["case"]
    if not own:
        if case["op"] == "linear":
            return torch.matmul(st["x"].float(), _values(st["w"], case["group"]).t()).to(st["y"].dtype)
        return _plain_ffn(st) if case["op"] == "ffn" else _plain_logprobs(st)
    from paper_2607_27591_b200 import binding as pb
    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "linear":
        pb.prox_w4_linear(st["w"], case["N"], case["K"], case["group"], st["x"], case["K"], _CODES[case["x"]], case["B"], st["y"],
                          case["N"], _CODES[case["y"]], stream)
        return st["y"]
    if case["op"] == "ffn":
        pb.prox_w4_stage2_ffn(st["gate"], st["up"], st["down_t"], case["D"], case["F"], case["group"], st["x"], case["B"], st["sel"],
                              case["k2"], st["count"], case["k2"], st["y"], _CODES[case["y"]], st["workspace"], st["workspace"].numel(),
                              stream)
        return st["y"]
    pb.prox_token_logprobs(st["x"], _CODES[case["x"]], case["T"], case["V"], st["x"].stride(0), case["temperature"], st["given"],
                           case["given"], st["logprob"], st["entropy"], case["top"], st["top_logprob"], st["top_index"], stream)
    return {k: st[k] for k in ("logprob", "entropy", "top_logprob", "top_index")}


def work(case):
    if case["op"] == "linear":
        N, K, B = case["N"], case["K"], case["B"]
        scales = (3.0 if case["zeros"] else 2.0) * N * _groups(K, case["group"])
        return {"bytes": N * K / 2 + scales + 2.0 * B * K + B * N * (4 if case["y"] == "fp32" else 2), "flops": 2.0 * B * N * K}
    if case["op"] == "ffn":
        D, F, B = case["D"], case["F"], case["B"]
        kept = [case["k2"] * (0.75 if case["counts"] else 1.0) * (0 if case["counts"] and b == 1 else 1) for b in range(B)]
        rows = F * (1.0 - math.prod(1.0 - k / F for k in kept))   # the tokens' masks are independent of one another
        row = D / 2 + 2.0 * _groups(D, case["group"])
        return {"bytes": 3 * rows * row + 4.0 * sum(kept) + B * D * (2 + (4 if case["y"] == "fp32" else 2)), "flops": 6.0 * D * sum(kept)}
    T, V = case["T"], case["V"]
    size = 4 if case["x"] == "fp32" else 2
    return {"bytes": T * (V * size + 8.0 * case["given"] + 4 + 8.0 * case["top"]), "flops": 6.0 * T * V}


def _exact_weight(w, group):
    codes, scales, zeros = w
    rows, half = codes.shape
    out = torch.empty(rows, 2 * half, dtype=torch.float64, device=codes.device)
    out[:, 0::2] = (codes % 16).double()
    out[:, 1::2] = (codes // 16).double()
    width = group if group else 2 * half
    for i, c in enumerate(range(0, 2 * half, width)):
        block = out[:, c:c + width]
        block -= 8.0 if zeros is None else zeros[:, i:i + 1].double()
        block *= scales[:, i:i + 1].double()
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "linear":
        y = torch.empty(case["B"], case["N"], dtype=torch.float64, device="cuda")
        step = max(1, (1 << 28) // case["K"])
        for r in range(0, case["N"], step):
            y[:, r:r + step] = st["x"].double() @ _exact_weight(tuple(None if t is None else t[r:r + step] for t in st["w"]), case["group"]).T
        return y
    if case["op"] == "ffn":
        y = torch.zeros(case["B"], case["D"], dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            n = case["k2"] if st["count"] is None else int(st["count"][b])
            index = st["sel"][b, :n].long()
            gate, up, down = (_exact_weight(tuple(None if t is None else t[index] for t in st[k]), case["group"]) for k in ("gate", "up", "down_t"))
            x = st["x"][b].double()
            g = gate @ x
            y[b] = ((up @ x) * g * torch.sigmoid(g)) @ down
        return y
    x, T, V, top = st["x"], case["T"], case["V"], case["top"]
    out = {"logprob": torch.empty(T, case["given"], dtype=torch.float64, device="cuda"), "entropy": torch.empty(T, dtype=torch.float64, device="cuda"),
           "top_logprob": torch.empty(T, top, dtype=torch.float64, device="cuda"), "top_index": torch.empty(T, top, dtype=torch.int32, device="cuda")}
    step = max(1, (1 << 27) // V)
    for r in range(0, T, step):
        part = x[r:r + step].double() / case["temperature"]
        logp = torch.log_softmax(part, 1)
        p = logp.exp()
        out["logprob"][r:r + step] = logp.gather(1, st["given"][r:r + step].long())
        out["entropy"][r:r + step] = -torch.where(p > 0, p * logp, 0.0).sum(1)
        if top:
            first = torch.sort(x[r:r + step], dim=1, descending=True, stable=True).indices[:, :top]
            out["top_logprob"][r:r + step] = logp.gather(1, first)
            out["top_index"][r:r + step] = first.to(torch.int32)
    return out
