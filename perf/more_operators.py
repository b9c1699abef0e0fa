"""The operators around the Linears of a denoiser's block, as timed cases: the update of the residual stream with the norms before and after
it, the gated feed-forward block, and a projection with low-rank adapters of many requests beside it.

A case names one operator with its sizes; `prepare` makes what a program holds before the call, `run` makes one pass, in elementary torch
operations or, where `own` is true, by the public binding.  Sizes are those of the workload configurations of
`paper_2603_25872_amd/inputs.py` (hidden 384 and 1152; 256, 1024 and 4096 tokens, 77 of a text; 6 to 64 slots a pass), video latents of the
same models, and shapes that no tile divides.

Tensors are [slots, tokens, columns].  "packed" ones are a column range of wider rows, the others lie by themselves.
"""
import math

import torch

own = False
EPS = 1e-6


def _norm(name, slots, tokens, width, stream, branch, after, before, packed, ragged=False):
    return dict(name=name, op="norm", slots=slots, tokens=tokens, width=width, stream=stream, branch=branch, after=after, before=before,
                packed=packed, ragged=ragged)


def _ffn(name, slots, tokens, width, hidden, dtype, act, packed, ragged=False):
    return dict(name=name, op="ffn", slots=slots, tokens=tokens, width=width, hidden=hidden, dtype=dtype, act=act, packed=packed, ragged=ragged)


def _lora(name, slots, tokens, width, out_width, rank, adapters, dtype, packed, ragged=False):
    return dict(name=name, op="lora", slots=slots, tokens=tokens, width=width, out_width=out_width, rank=rank, adapters=adapters, dtype=dtype,
                packed=packed, ragged=ragged)


def listed():
    return [
        # one row, as the conditioning vector of a single sample passes it: launch latency
        _norm("norm_one", 1, 1, 1152, "f32", "bf16", "none", "layer", False),
        # configuration 4's pass: 6 slots of 4096 tokens, the stream in fp32, the branch's output gated, the next branch's input modulated
        _norm("norm_text_4096", 6, 4096, 1152, "f32", "bf16", "none", "layer", False),
        # a video latent, 16 frames of 32 x 32 tokens, the stream in bf16, RMS norms on both sides of the branch
        _norm("norm_video", 4, 16384, 1536, "bf16", "bf16", "rms", "rms", True),
        # fp32, LayerNorm on both sides, 13 slots of at most 252 tokens, a width that no vector divides
        _norm("norm_f32", 13, 252, 771, "f32", "f32", "layer", "layer", False, ragged=True),
        # one token through configuration 3's widths: the weights' bytes
        _ffn("ffn_one", 1, 1, 1152, 4608, "bf16", "silu", False),
        # configuration 2's pass: 12 slots of 256 tokens
        _ffn("ffn_dit_s", 12, 256, 384, 1536, "bf16", "silu", False),
        # configuration 5's pass: 64 slots of 1024 tokens; the largest
        _ffn("ffn_wide", 64, 1024, 1152, 4608, "bf16", "gelu", False),
        # a small fp32 model on token lists of uneven length
        _ffn("ffn_f32", 5, 331, 250, 694, "f32", "gelu", True, ragged=True),
        # the modulation Linear of 64 requests with styles of their own: one row each
        _lora("lora_rows", 64, 1, 1152, 6912, 16, 24, "bf16", False),
        # configuration 5's q | k | v of 64 slots of 1024 tokens, eight styles among them
        _lora("lora_qkv", 64, 1024, 1152, 3456, 32, 8, "bf16", False),
        # the text's keys and values, 77 tokens a slot at most, every request its own adapter
        _lora("lora_text", 19, 77, 1024, 2304, 24, 19, "bf16", True, ragged=True),
        # a small fp32 model, a rank that no vector divides
        _lora("lora_f32", 7, 250, 390, 1170, 5, 3, "f32", False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: sizes between those of the listed cases, odd ones among them, at most their largest cost for its operator."""
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), _cost(c))
    while True:
        op = rng.choice(["norm", "ffn", "lora"])
        dtype = "bf16" if rng.random() < 0.7 else "f32"
        slots, tokens = _log_int(rng, 1, 64), _log_int(rng, 1, 16384)
        packed, ragged = rng.random() < 0.5, rng.random() < 0.4
        unit = 8 if dtype == "bf16" else 1
        width = unit * _log_int(rng, 64 // unit, 2048 // unit)
        if op == "norm":
            stream = "f32" if dtype == "f32" else rng.choice(["f32", "bf16"])
            if rng.random() < 0.3:
                width = rng.randint(64, 2048)
            c = _norm("", slots, tokens, width, stream, dtype, rng.choice(["none", "rms", "layer"]), rng.choice(["rms", "layer"]), packed, ragged)
        elif op == "ffn":
            c = _ffn("", slots, tokens, width, unit * _log_int(rng, 128 // unit, 6144 // unit), dtype, rng.choice(["silu", "gelu"]), packed, ragged)
        else:
            c = _lora("", slots, tokens, width, rng.choice([8, 2]) * _log_int(rng, 32, 900), _log_int(rng, 1, 128), rng.randint(1, slots), dtype, packed, ragged)
        if _cost(c) <= most[op] and not (dtype == "f32" and work(c)["flops"] > 1e11):
            del c["name"]
            return c


def _cost(case):
    w = work(case)
    return w["bytes"] + w["flops"] / 300


def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    # (a slot's length is between half of its tokens and all of them)
    rows, d = case["slots"] * case["tokens"] * (0.75 if case["ragged"] else 1), case["width"]
    if case["op"] == "norm":
        return {"bytes": rows * d * 2 * (_size(case["stream"]) + _size(case["branch"])) + 12 * case["slots"] * d, "flops": 20 * rows * d}
    size = _size(case["dtype"])
    if case["op"] == "ffn":
        return {"bytes": size * (2 * rows * d + 3 * d * case["hidden"]), "flops": 6 * rows * d * case["hidden"]}
    used = min(case["slots"], case["adapters"])
    return {"bytes": size * (rows * (d + case["out_width"]) + d * case["out_width"] + used * case["rank"] * (d + case["out_width"])),
            "flops": 2 * rows * (d * case["out_width"] + case["rank"] * (d + case["out_width"]))}


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rows(case, x, dtype):
    """x [slots, tokens, columns] in its type: by itself, or the middle columns of wider rows."""
    if not case["packed"]:
        return x.to(dtype)
    wide = torch.zeros(x.shape[0], x.shape[1], x.shape[2] + 48, dtype=dtype, device="cuda")
    wide[..., 16:16 + x.shape[2]] = x
    return wide[..., 16:16 + x.shape[2]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    slots, tokens, d = case["slots"], case["tokens"], case["width"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s["lens"], s["out"] = None, None
    if case["ragged"]:
        s["lens"] = torch.randint((tokens + 1) // 2, tokens + 1, (slots,), generator=g, device="cuda", dtype=torch.int32)
    if case["op"] == "norm":
        # the stream grows over the blocks and has a few large columns, as trained ones do
        columns = 1 + 5 * (torch.rand(d, generator=g, device="cuda") < 0.02)
        s["x"] = _rows(case, randn(slots, tokens, d) * 3 * columns + 0.2 * randn(d), _dtype(case["stream"]))
        s["y"] = _rows(case, randn(slots, tokens, d), _dtype(case["branch"]))
        # shift, scale and gate of every slot: columns of the modulation Linear's rows
        rows = 0.3 * randn(slots, 6 * d)
        s["shift"], s["scale"], s["gate"] = rows[:, :d], rows[:, d:2 * d], rows[:, 5 * d:]
        s["after_gain"] = 1 + 0.1 * randn(d) if case["after"] != "none" else None
        s["after_bias"] = 0.1 * randn(d) if case["after"] == "layer" else None
        s["before_gain"] = 1 + 0.1 * randn(d) if case["before"] == "rms" else None
        s["h_out"] = None
        if case["ragged"]:
            # the program's own buffers: rows behind a slot's length stay what they are
            s["out"], s["h_out"] = s["x"].clone(), torch.zeros_like(s["y"])
        return s
    s["x"] = _rows(case, randn(slots, tokens, d), _dtype(case["dtype"]))
    t = _dtype(case["dtype"])
    if case["op"] == "ffn":
        f = case["hidden"]
        s["w_in"], s["b_in"] = (randn(2 * f, d) * d ** -0.5).to(t), 0.1 * randn(2 * f)      # the gate's rows, then the value's
        s["w_out"], s["b_out"] = (randn(d, f) * f ** -0.5).to(t), 0.1 * randn(d)
        n = d
    else:
        n, r = case["out_width"], case["rank"]
        s["w"], s["bias"] = (randn(n, d) * d ** -0.5).to(t), 0.1 * randn(n)
        s["a"], s["b"] = (randn(case["adapters"], r, d) * d ** -0.5).to(t), (0.3 * randn(case["adapters"], n, r)).to(t)
        s["scales"] = 0.5 + torch.rand(case["adapters"], generator=g, device="cuda")
        # some requests have no adapter
        s["which"] = torch.randint(-1, case["adapters"], (slots,), generator=g, device="cuda", dtype=torch.int32)
    if case["ragged"]:
        s["out"] = torch.zeros(slots, tokens, n, dtype=t, device="cuda")
    return s


def _inside(s, y, behind):
    """Rows behind a slot's length are left as they were."""
    if s["lens"] is None:
        return y
    keep = torch.arange(s["tokens"], device="cuda")[None] < s["lens"][:, None]
    return torch.where(keep[..., None], y, behind)


def _plain_norm(x, kind, gain, bias):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    if gain is not None:
        x = x * gain
    return x if bias is None else x + bias


def _plain_residual(s):
    y = _plain_norm(s["y"].float(), s["after"], s["after_gain"], s["after_bias"])
    z = s["x"].float() + s["gate"][:, None] * y
    h = _plain_norm(z, s["before"], s["before_gain"], None) * (1 + s["scale"][:, None]) + s["shift"][:, None]
    return _inside(s, z.to(s["x"].dtype), s["out"]), _inside(s, h.to(s["y"].dtype), s["h_out"])


def _plain_ffn(s):
    u = s["x"].float() @ s["w_in"].float().t() + s["b_in"]
    a, v = u[..., :s["hidden"]], u[..., s["hidden"]:]
    if s["act"] == "silu":
        a = a / (1 + torch.exp(-a))
    else:
        a = 0.5 * a * (1 + torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a * a * a)))
    y = (a * v) @ s["w_out"].float().t() + s["b_out"]
    return _inside(s, y.to(s["x"].dtype), s["out"])


def _plain_lora(s):
    x, some = s["x"].float(), (s["which"] >= 0)
    i = s["which"].clamp(min=0).long()
    y = x @ s["w"].float().t() + s["bias"]
    a, b = s["a"][i].float(), s["b"][i].float()
    low = (x @ a.transpose(1, 2).contiguous()) * (s["scales"][i] * some)[:, None, None]
    y = y + low @ b.transpose(1, 2).contiguous()
    return _inside(s, y.to(s["x"].dtype), s["out"])


def _own(s):
    from paper_2603_25872_amd import drf
    if s["op"] == "norm":
        return drf.residual_norm(s["x"], s["y"], gate=s["gate"], after=s["after"], after_gain=s["after_gain"], after_bias=s["after_bias"], before=s["before"],
                                 before_gain=s["before_gain"], shift=s["shift"], scale=s["scale"], eps=EPS, lens=s["lens"], out=s["out"], h_out=s["h_out"])
    if s["op"] == "ffn":
        return drf.gated_ffn(s["x"], s["w_in"], s["w_out"], b_in=s["b_in"], b_out=s["b_out"], act=s["act"], lens=s["lens"], out=s["out"])
    return drf.linear_adapters(s["x"], s["w"], s["a"], s["b"], s["which"], bias=s["bias"], scales=s["scales"], lens=s["lens"], out=s["out"])


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_residual, "ffn": _plain_ffn, "lora": _plain_lora}[state["op"]](state)


def _exact_norm(x, kind):
    if kind == "none":
        return x
    if kind == "layer":
        return (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS)
    return x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS)


def exact(case, seed):
    s = prepare(case, seed)
    slots, tokens = case["slots"], case["tokens"]
    # one slot at a time, its rows alone, in float64
    lens = [tokens] * slots if s["lens"] is None else s["lens"].tolist()
    outs = []
    for j, m in enumerate(lens):
        x = s["x"][j, :m].double()
        if case["op"] == "norm":
            y = _exact_norm(s["y"][j, :m].double(), case["after"])
            if s["after_gain"] is not None:
                y = torch.addcmul(torch.zeros_like(y) if s["after_bias"] is None else s["after_bias"].double().expand_as(y), y, s["after_gain"].double())
            z = torch.addcmul(x, y, s["gate"][j].double())
            gain = (1 + s["scale"][j].double()) * (1 if s["before_gain"] is None else s["before_gain"].double())
            parts = [z, torch.addcmul(s["shift"][j].double(), _exact_norm(z, case["before"]), gain)]
            behind = [s["x"][j, m:].double(), torch.zeros_like(s["y"][j, m:], dtype=torch.float64)]
        elif case["op"] == "ffn":
            w, b = s["w_in"].double(), s["b_in"].double()
            a, v = torch.addmm(b, x, w.t()).chunk(2, dim=-1)
            a = a * torch.sigmoid(a if case["act"] == "silu" else 2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3))
            parts = [torch.addmm(s["b_out"].double(), a * v, s["w_out"].double().t())]
            behind = [torch.zeros(tokens - m, parts[0].shape[1], dtype=torch.float64, device="cuda")]
        else:
            i = int(s["which"][j])
            w = s["w"].double()
            if i >= 0:                                  # the adapter merged into the projection
                w = w + float(s["scales"][i]) * (s["b"][i].double() @ s["a"][i].double())
            parts = [torch.addmm(s["bias"].double(), x, w.t())]
            behind = [torch.zeros(tokens - m, parts[0].shape[1], dtype=torch.float64, device="cuda")]
        outs.append([torch.cat(p) for p in zip(parts, behind)])
    outs = [torch.stack(o) for o in zip(*outs)]
    return tuple(outs) if case["op"] == "norm" else outs[0]
