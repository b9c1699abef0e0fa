"""The operators of the denoiser's attention, as timed cases: rotary positions with several axes, norms of queries and keys with the
rotation in the same pass, the choice of key blocks by a cheap score, and attention over the chosen blocks.

A case names one operator with its sizes; `prepare` makes what a program holds before the call, `run` makes one pass, in elementary torch
operations or, where `own` is true, by the public binding.  Sizes are those of the workload configurations of
`paper_2603_25872_amd/inputs.py` (6 heads of 64, 16 heads of 72; 256, 1024 and 4096 tokens; 6 to 64 slots a pass), video latents of the same
models (frames x rows x columns tokens), and shapes that no tile divides.

Tensors are [slots, tokens, heads, head width].  "packed" ones are the column ranges of a qkv Linear's output rows, the others are stored
head by head.
"""
import math

import torch

own = False
EPS = 1e-6


def _rope(name, slots, tokens, heads, d, dtype, dims, extent, layout, packed, table=False, ragged=False):
    return dict(name=name, op="rope", slots=slots, tokens=tokens, heads=heads, d=d, dtype=dtype, dim0=dims[0], dim1=dims[1], dim2=dims[2],
                ext0=extent[0], ext1=extent[1], ext2=extent[2], layout=layout, packed=packed, table=table, ragged=ragged)


def _qk(name, slots, tokens, heads, kv_heads, d, dtype, norm, dims, extent, layout, packed, ragged=False):
    return dict(_rope(name, slots, tokens, heads, d, dtype, dims, extent, layout, packed, False, ragged), op="qk", kv_heads=kv_heads, norm=norm)


def _select(name, slots, tokens, heads, kv_heads, d, dtype, q_block, kv_block, topk, packed, ragged=False):
    return dict(name=name, op="select", slots=slots, q_tokens=tokens, tokens=tokens, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype,
                q_block=q_block, kv_block=kv_block, topk=topk, packed=packed, ragged=ragged)


def _attend(name, slots, q_tokens, tokens, heads, kv_heads, d, dtype, q_block, kv_block, topk, packed, ragged=False):
    return dict(_select(name, slots, tokens, heads, kv_heads, d, dtype, q_block, kv_block, topk, packed, ragged), op="attend", q_tokens=q_tokens)


def listed():
    return [
        # one token's heads, as a caller that adds tokens one at a time rotates them: launch latency
        _rope("rope_one", 1, 1, 16, 72, "bf16", (0, 36, 36), (1, 1, 1), "pairs", False, table=True),
        # keys of a video latent, 16 frames of 32 x 32 tokens, two guided samples: bandwidth
        _rope("rope_video", 4, 16384, 16, 72, "bf16", (24, 24, 24), (16, 32, 32), "halves", True),
        # a small fp32 model on token lists of uneven length whose positions come from a table, far from zero
        _rope("rope_table_f32", 5, 1007, 4, 32, "f32", (0, 16, 12), (1, 19, 53), "pairs", False, table=True, ragged=True),
        # configuration 2's pass: 12 slots of 256 tokens, q and k inside the qkv rows
        _qk("qk_dit_s", 12, 256, 6, 6, 64, "bf16", "rms", (0, 32, 32), (1, 16, 16), "pairs", True),
        # configuration 4's pass: 6 slots of 4096 tokens, stored head by head as the attention reads them
        _qk("qk_text_4096", 6, 4096, 16, 16, 72, "bf16", "rms", (0, 36, 36), (1, 64, 64), "pairs", False),
        # LayerNorm of heads in fp32, fewer key heads than query heads, 13 slots of at most 252 tokens
        _qk("qk_layer_f32", 13, 252, 12, 4, 80, "f32", "layer", (0, 40, 40), (1, 18, 14), "halves", True, ragged=True),
        # configuration 5's pass: 64 slots of 1024 tokens, a quarter of the blocks
        _select("select_wide", 64, 1024, 16, 16, 72, "bf16", 64, 64, 4, False),
        # one long video in fp32, 24 frames of 26 x 31 tokens, uneven slots
        _select("select_video_f32", 2, 19344, 8, 8, 64, "f32", 128, 64, 37, True, ragged=True),
        # a single query over a long sequence: latency, nothing to share between queries
        _attend("attend_one", 1, 1, 4096, 16, 16, 72, "bf16", 64, 64, 16, False),
        # configuration 4's pass: 8 of 64 blocks a query block
        _attend("attend_4096", 6, 4096, 4096, 16, 16, 72, "bf16", 64, 64, 8, False),
        # a video latent of 16 frames of 32 x 32 tokens, wide heads that share keys, large blocks
        _attend("attend_video", 4, 16384, 16384, 12, 4, 128, "bf16", 128, 128, 16, True),
        # a small fp32 model, small blocks, uneven slots
        _attend("attend_f32", 7, 1000, 1000, 4, 4, 32, "f32", 32, 32, 5, False, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: sizes between those of the listed cases, odd ones among them, at most their largest cost for its operator."""
    most = {}
    for c in listed():
        w = work(c)
        most[c["op"]] = max(most.get(c["op"], 0), w["bytes"] + w["flops"] / 300)
    pairs = max(_pairs(c) for c in listed() if c["op"] == "attend")
    while True:
        op = rng.choice(["rope", "qk", "select", "attend"])
        dtype = "bf16" if rng.random() < 0.7 else "f32"
        slots, packed, ragged = _log_int(rng, 1, 64), rng.random() < 0.5, rng.random() < 0.4
        kv_heads = rng.randint(1, 16)
        heads = kv_heads * rng.choice([1, 1, 1, 2, 3])
        if op in ("rope", "qk"):
            ext = (_log_int(rng, 1, 16), _log_int(rng, 1, 64), _log_int(rng, 1, 64))
            tokens = ext[0] * ext[1] * ext[2]
            dims = tuple(2 * rng.randint(0, 20) for _ in range(3))
            d = 8 * rng.randint(max(1, -(-sum(dims) // 8)), 16) if sum(dims) <= 128 else 0
            layout = rng.choice(["pairs", "halves"])
            if sum(dims) == 0 or d == 0 or heads > 32:
                continue
            if op == "rope":
                c = _rope("", slots, tokens, heads, d, dtype, dims, ext, layout, packed, rng.random() < 0.3, ragged)
            else:
                c = _qk("", slots, tokens, heads, kv_heads, d, dtype, rng.choice(["rms", "layer"]), dims, ext, layout, packed, ragged)
        else:
            tokens = _log_int(rng, 100, 20000)
            d = 8 * rng.randint(1, 16)
            q_block, kv_block = rng.choice([32, 64, 128]), rng.choice([32, 64, 128])
            blocks = -(-tokens // kv_block)
            topk = rng.randint(1, max(1, min(blocks - 1, 40)))
            if not 2 <= blocks <= 1024 or heads > 32:
                continue
            if op == "select":
                c = _select("", slots, tokens, heads, kv_heads, d, dtype, q_block, kv_block, topk, packed, ragged)
            else:
                q_tokens = tokens if rng.random() < 0.7 else _log_int(rng, 1, 1000)
                c = _attend("", slots, q_tokens, tokens, heads, kv_heads, d, dtype, q_block, kv_block, topk, packed and q_tokens == tokens, ragged)
        w = work(c)
        if w["bytes"] + w["flops"] / 300 <= most[op] and not (op == "attend" and (_pairs(c) > pairs or dtype == "f32" and w["flops"] > 5e10)):
            del c["name"]
            return c


def _pairs(case):
    """Scores that an attention case forms."""
    return case["slots"] * case["heads"] * case["q_tokens"] * case["topk"] * case["kv_block"]


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    rows, d = case["slots"] * case["tokens"], case["d"]
    if case["op"] == "rope":
        n = rows * case["heads"] * d
        return {"bytes": 2 * n * size, "flops": 3 * n}
    if case["op"] == "qk":
        n = rows * (case["heads"] + case["kv_heads"]) * d
        return {"bytes": 2 * n * size, "flops": 7 * n}
    nq, nk = -(-case["q_tokens"] // case["q_block"]), -(-case["tokens"] // case["kv_block"])
    if case["op"] == "select":
        n = case["slots"] * d * (case["q_tokens"] * case["heads"] + case["tokens"] * case["kv_heads"])
        return {"bytes": n * size + case["slots"] * case["heads"] * nq * -(-nk // 32) * 4, "flops": n + 2 * d * case["slots"] * case["heads"] * nq * nk}
    keys = min(case["topk"] * case["kv_block"], case["tokens"])
    n = case["slots"] * d * (2 * case["q_tokens"] * case["heads"] + 2 * case["tokens"] * case["kv_heads"])
    return {"bytes": n * size, "flops": 4 * d * case["slots"] * case["heads"] * case["q_tokens"] * keys}


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _field(g, case, tokens, heads, block):
    """[slots, heads, tokens, d] that varies slowly along the tokens (what neighbouring tokens have in common) plus as much noise."""
    coarse = torch.randn(case["slots"], heads, -(-tokens // block), case["d"], generator=g, device="cuda")
    x = torch.randn(case["slots"], heads, tokens, case["d"], generator=g, device="cuda")
    x += coarse.repeat_interleave(block, dim=2)[:, :, :tokens]
    return x.to(_dtype(case))


def _lay(parts, packed):
    """Tensors [slots, heads, tokens, d] as [slots, tokens, heads, d] views: of one tensor of rows, or head by head."""
    if not packed:
        return [p.transpose(1, 2) for p in parts]
    rows = torch.cat([p.transpose(1, 2) for p in parts], dim=2)
    return list(rows.split([p.shape[1] for p in parts], dim=2))


def _lens(g, case, tokens):
    if not case["ragged"]:
        return None
    return torch.randint(tokens // 2, tokens + 1, (case["slots"],), generator=g, device="cuda", dtype=torch.int32)


def _config(case):
    """What a program sets up once: the rotation's sections, grid and base."""
    return dict(dims=(case["dim0"], case["dim1"], case["dim2"]), extents=(case["ext0"], case["ext1"], case["ext2"]), theta=10000.0, layout=case["layout"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] in ("rope", "qk"):
        s["rope"] = _config(case)
        s["plan"] = _plan(s["rope"])
        kv_heads = case.get("kv_heads", case["heads"])
        s["q"], s["k"], _ = _lay([_field(g, case, case["tokens"], n, 64) for n in (case["heads"], kv_heads, kv_heads)], case["packed"])
        s["lens"] = _lens(g, case, case["tokens"])
        if case["op"] == "qk":
            # gains near one as a trained norm has them
            s["q_gain"], s["k_gain"], s["q_bias"], s["k_bias"] = (
                m + 0.1 * torch.randn(case["d"], generator=g, device="cuda") for m in (1.0, 1.0, 0.0, 0.0))
            if case["norm"] == "rms":
                s["q_bias"] = s["k_bias"] = None
        s["positions"] = None
        if case.get("table"):
            s["positions"] = torch.randint(0, 20000, (case["slots"], case["tokens"], 3), generator=g, device="cuda").float()
        return s
    s["q"], s["k"], s["v"] = _lay([_field(g, case, t, n, case["kv_block"]) for t, n in (
        (case["q_tokens"], case["heads"]), (case["tokens"], case["kv_heads"]), (case["tokens"], case["kv_heads"]))], case["packed"])
    s["kv_lens"] = _lens(g, case, case["tokens"])
    s["q_lens"] = s["kv_lens"] if case["q_tokens"] == case["tokens"] else None
    if case["op"] == "attend":
        s["blocks"] = _plain_select(s)
    return s


def _plan(rope):
    """What a program sets up once for the plain form: axis and frequency of every pair, columns of its first and of its second member."""
    dims = torch.tensor(rope["dims"], device="cuda")
    half = dims // 2
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), half)
    i = torch.arange(axis.numel(), device="cuda") - (torch.cumsum(half, 0) - half)[axis]
    freq = torch.pow(torch.tensor(rope["theta"], dtype=torch.float64, device="cuda"), -2.0 * i.double() / dims[axis])
    start = (torch.cumsum(dims, 0) - dims)[axis]
    if rope["layout"] == "pairs":
        return axis, freq, start + 2 * i, start + 2 * i + 1
    return axis, freq, start + i, start + i + half[axis]


def _angles(s):
    """[slots or 1, tokens, pairs] in float64."""
    axis, freq = s["plan"][:2]
    pos = s["positions"]
    if pos is None:
        n, e = torch.arange(s["tokens"], device="cuda"), s["rope"]["extents"]
        pos = torch.stack([n // (e[1] * e[2]), n // e[2] % e[1], n % e[2]], dim=-1)[None]
    return pos.double()[..., axis] * freq


def _plain_rotate(s, x):
    """fp32 [slots, tokens, heads, d]; angles in 64 bits, cosines and sines rounded to 32."""
    phi = _angles(s)
    c, n = phi.cos().float()[:, :, None], phi.sin().float()[:, :, None]
    a, b = s["plan"][2:]
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * n
    y[..., b] = x[..., a] * n + x[..., b] * c
    return y


def _plain_norm(s, x, gain, bias):
    if s["norm"] == "rms":
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain + bias


def _inside(s, y):
    """Rows behind a slot's length are not part of the result."""
    if s["lens"] is None:
        return y
    keep = torch.arange(s["tokens"], device="cuda")[None] < s["lens"][:, None]
    return torch.where(keep[:, :, None, None], y, torch.zeros_like(y))


def _block_means(x, block, lens):
    """Means [slots, heads, blocks, d] in float64 over the rows inside a slot's length, and whether a block has any."""
    slots, tokens, heads, d = x.shape
    nb = -(-tokens // block)
    full = torch.zeros(slots, nb * block, heads, d, dtype=torch.float64, device="cuda")
    full[:, :tokens] = x
    lens = torch.full((slots,), tokens, device="cuda") if lens is None else lens
    keep = torch.arange(nb * block, device="cuda")[None] < lens[:, None]
    full = torch.where(keep[:, :, None, None], full, torch.zeros_like(full))
    count = keep.view(slots, nb, block).sum(-1)
    mean = full.view(slots, nb, block, heads, d).sum(2) / count.clamp(min=1)[:, :, None, None]
    return mean.transpose(1, 2).contiguous(), count > 0


def _plain_select(s):
    """Words of 32 blocks: the topk blocks of largest score, the lowest of equal ones first."""
    qm, _ = _block_means(s["q"], s["q_block"], s["q_lens"])
    km, some = _block_means(s["k"], s["kv_block"], s["kv_lens"])
    km = km.repeat_interleave(s["heads"] // s["kv_heads"], dim=1)
    score = qm @ km.transpose(2, 3).contiguous()
    score = torch.where(some[:, None, None], score, torch.full_like(score, -math.inf))
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :s["topk"]]
    chosen = torch.zeros(score.shape, dtype=torch.bool, device="cuda").scatter_(-1, order, True) & some[:, None, None]
    if s["q_lens"] is not None:
        has = torch.arange(qm.shape[2], device="cuda")[None] * s["q_block"] < s["q_lens"][:, None]
        chosen &= has[:, None, :, None]
    words = -(-score.shape[-1] // 32)
    bits = torch.zeros(*score.shape[:-1], words * 32, dtype=torch.int64, device="cuda")
    bits[..., :score.shape[-1]] = chosen
    return (bits.view(*score.shape[:-1], words, 32) << torch.arange(32, device="cuda")).sum(-1).to(torch.int32)


def _plain_attend(s):
    """Keys and values of each query block's list gathered, softmax in fp32; a query without keys gives zeros."""
    slots, nq, heads, d = s["q"].shape
    kb, qb, tokens = s["kv_block"], s["q_block"], s["tokens"]
    nkb, nqb = -(-tokens // kb), -(-nq // qb)
    bits = (s["blocks"][..., None] >> torch.arange(32, device="cuda")) & 1
    bits = bits.flatten(-2)[..., :nkb]
    most = min(s["topk"], nkb)
    order = torch.sort(bits, dim=-1, descending=True, stable=True)
    index, live = order.indices[..., :most], order.values[..., :most] > 0
    rows = (index[..., None] * kb + torch.arange(kb, device="cuda")).flatten(-2)                    # [slots, heads, nqb, most * kb]
    lens = torch.full((slots,), tokens, device="cuda") if s["kv_lens"] is None else s["kv_lens"]
    valid = live[..., None].expand(*live.shape, kb).flatten(-2) & (rows < lens[:, None, None, None])
    rows = rows.clamp(max=tokens - 1)
    at = torch.arange(slots, device="cuda")[:, None, None, None]
    h = (torch.arange(heads, device="cuda") // (heads // s["kv_heads"]))[None, :, None, None]
    k, v = s["k"][at, rows, h].float(), s["v"][at, rows, h].float()                                 # [slots, heads, nqb, keys, d]
    q = torch.zeros(slots, nqb * qb, heads, d, device="cuda")
    q[:, :nq] = s["q"]
    q = q.view(slots, nqb, qb, heads, d).permute(0, 3, 1, 2, 4).contiguous()
    score = q @ k.transpose(3, 4).contiguous() * d ** -0.5
    score = torch.where(valid[:, :, :, None], score, torch.full_like(score, -math.inf))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    y = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    y = y.permute(0, 2, 3, 1, 4).reshape(slots, nqb * qb, heads, d)[:, :nq]
    if s["q_lens"] is not None:
        keep = torch.arange(nq, device="cuda")[None] < s["q_lens"][:, None]
        y = torch.where(keep[:, :, None, None], y, torch.zeros_like(y))
    return y.to(s["q"].dtype)


def _own(s):
    from paper_2603_25872_amd import drf
    if s["op"] in ("rope", "qk"):
        if "rope_config" not in s:                      # set up once, as a program does
            s["rope_config"] = drf.rope_config(**s["rope"])
        # rows behind a slot's length are left as they were: zeros here
        new = torch.zeros if s["lens"] is not None else torch.empty
        q_out = new(s["q"].shape, dtype=s["q"].dtype, device="cuda")
        if s["op"] == "rope":
            return drf.rope(s["q"], s["rope_config"], positions=s["positions"], lens=s["lens"], out=q_out)
        k_out = new(s["k"].shape, dtype=s["k"].dtype, device="cuda")
        return drf.qk_norm_rope(s["q"], s["k"], s["norm"], s["rope_config"], q_gain=s["q_gain"], k_gain=s["k_gain"], q_bias=s["q_bias"],
                                k_bias=s["k_bias"], eps=EPS, lens=s["lens"], q_out=q_out, k_out=k_out)
    if s["op"] == "select":
        return drf.block_select(s["q"], s["k"], s["q_block"], s["kv_block"], s["topk"], q_lens=s["q_lens"], kv_lens=s["kv_lens"])
    return drf.block_attention(s["q"], s["k"], s["v"], s["blocks"], s["q_block"], s["kv_block"], q_lens=s["q_lens"], kv_lens=s["kv_lens"])


def run(state):
    s = state
    if own:
        return _own(s)
    if s["op"] == "rope":
        return _inside(s, _plain_rotate(s, s["q"].float()).to(s["q"].dtype))
    if s["op"] == "qk":
        q = _plain_rotate(s, _plain_norm(s, s["q"].float(), s["q_gain"], s["q_bias"]))
        k = _plain_rotate(s, _plain_norm(s, s["k"].float(), s["k_gain"], s["k_bias"]))
        return _inside(s, q.to(s["q"].dtype)), _inside(s, k.to(s["k"].dtype))
    if s["op"] == "select":
        return _plain_select(s)
    return _plain_attend(s)


def _exact_heads(s, x, gain=None, bias=None):
    """Norm and rotation from their definitions, the rotation as a product of complex numbers."""
    x = x.double()
    if gain is not None:
        if s["norm"] == "layer":
            x = x - x.sum(-1, keepdim=True) / s["d"]
        x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / s["d"] + EPS) * gain.double()
        if bias is not None:
            x = x + bias.double()
    n = torch.arange(s["tokens"], device="cuda")
    out, at = [], 0
    for axis, dim in enumerate(s["rope"]["dims"]):
        part, at = x[..., at:at + dim], at + dim
        if dim == 0:
            continue
        below = math.prod(s["rope"]["extents"][axis + 1:])
        pos = (n // below % s["rope"]["extents"][axis])[None].double() if s["positions"] is None else s["positions"][..., axis].double()
        if axis == 0 and s["positions"] is None:
            pos = (n // below)[None].double()
        freq = torch.tensor([s["rope"]["theta"] ** (-2.0 * i / dim) for i in range(dim // 2)], dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[..., None] * freq)[:, :, None]
        if s["rope"]["layout"] == "pairs":
            z = torch.view_as_complex(part.unflatten(-1, (dim // 2, 2)).contiguous()) * turn
            out.append(torch.view_as_real(z).flatten(-2))
        else:
            z = torch.complex(part[..., :dim // 2].contiguous(), part[..., dim // 2:].contiguous()) * turn
            out += [z.real, z.imag]
    y = torch.cat(out + [x[..., at:]], dim=-1)
    if s["lens"] is not None:
        for j, m in enumerate(s["lens"].tolist()):
            y[j, m:] = 0
    return y


def exact(case, seed):
    if case["op"] == "select":
        return None                                     # whole numbers
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_heads(s, s["q"])
    if case["op"] == "qk":
        return _exact_heads(s, s["q"], s["q_gain"], s["q_bias"]), _exact_heads(s, s["k"], s["k_gain"], s["k_bias"])
    # one (slot, head) at a time over all keys, in float64
    slots, nq, heads, d = s["q"].shape
    out = torch.zeros(slots, nq, heads, d, dtype=torch.float64, device="cuda")
    key_block = torch.arange(s["tokens"], device="cuda") // s["kv_block"]
    query_block = torch.arange(nq, device="cuda") // s["q_block"]
    for j in range(slots):
        m = s["tokens"] if s["kv_lens"] is None else int(s["kv_lens"][j])
        mq = nq if s["q_lens"] is None else int(s["q_lens"][j])
        for h in range(heads):
            g = h // (heads // s["kv_heads"])
            seen = (s["blocks"][j, h][:, key_block[:m] // 32] >> (key_block[:m] % 32)) & 1
            score = s["q"][j, :mq, h].double() @ s["k"][j, :m, g].double().t().contiguous() / math.sqrt(d)
            score.masked_fill_(seen[query_block[:mq]] == 0, -math.inf)
            y = torch.softmax(score, dim=-1) @ s["v"][j, :m, g].double()
            out[j, :mq, h] = torch.where(torch.isnan(y), torch.zeros_like(y), y)
    return out
