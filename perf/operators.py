"""Timed cases of the operators around an 8-bit K/V cache: rotary positions, the quantising append, reading back, and
attention over the cache (one new token over a page list; verification of several with page scores).

The cache holds one-byte codes (e4m3, or int8) in the layout of the bf16 caches, [pages, 16, KV heads, head dim], and one
fp32 scale per token, KV head and tensor in `scales` [pages, KV heads, 2 (K, V), 16].  A case is one call of one operator:

  rotate   rotary positions of a tensor's heads
  append   new tokens' K (rotated) and V quantised into the cache, their queries rotated beside them
  read     a list of tokens read back as bf16
  draft    attention of one new token per sequence over a page list (a selection, or the whole block table)
  verify   attention of several new tokens per sequence, causal, with the criticality of every page

`own` decides what run() calls: the plain forms in elementary torch operations, or the package's entry points.
"""
from __future__ import annotations

import math
from typing import Dict, List

import torch

own = False

PAGE = 16
DEVICE = "cuda:0"
TOP = {"e4m3": 448.0, "int8": 127.0}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TINY = 2.0 ** -110            # rows below it are stored as zeros
ORIGINAL = 32768              # positions the unscaled frequencies were made for


def _case(name: str, kind: str, **sizes) -> Dict[str, object]:
    base = dict(name=name, kind=kind, batch=1, heads=32, kv_heads=8, dim=128, queries=1, lo=0, hi=0, tokens=0, page=PAGE,
                format="e4m3", rot=0, layout="half", scaling="none", collect=0)
    base.update(sizes)
    return base


def listed() -> List[Dict[str, object]]:
    return [
        # The verification rows of a serving batch: 16 sequences x 5 tokens, 64 heads.  All latency.
        _case("rotate_rows_16x5", "rotate", batch=16, tokens=5, heads=64, kv_heads=0, lo=8192, hi=65536, rot=128),
        # A prompt's queries and keys (one projection's 32 + 8 heads), half of every head rotated, pairs interleaved,
        # positions far beyond the trained length.
        _case("rotate_prompt_8k", "rotate", batch=1, tokens=8191, heads=40, kv_heads=0, lo=122000, hi=122000, rot=64,
              layout="interleaved", scaling="linear"),
        # A decoding step of a batch in flight: one token per sequence into the cache, its queries rotated.
        _case("append_step_batch24", "append", batch=24, tokens=1, lo=1001, hi=20011, rot=128),
        # Four prompts of up to 4096 tokens, padded to the longest, context extended by four.
        _case("append_prompt_4x4096", "append", batch=4, tokens=4096, lo=0, hi=32000, rot=128, scaling="yarn"),
        # int8 codes of K and V alone (keys that came rotated), the 64-dimensional head shape, an odd prompt length.
        _case("append_int8_hd64", "append", batch=8, tokens=1011, lo=0, hi=500, dim=64, heads=64, format="int8"),
        # A selection of 130 pages read back, as a check against an exact pass would.
        _case("read_selection_8x2080", "read", batch=8, lo=2080, hi=2080, tokens=2080, format="int8"),
        # Whole sequences back to bf16, ragged.
        _case("read_batch4_64k", "read", batch=4, lo=20000, hi=65521, tokens=65521),
        # A draft call at 32K tokens of context: 130 selected pages of one sequence.  Launches and round trips.
        _case("draft_32k", "draft", batch=1, lo=2080, hi=2080),
        # Sixteen requests of 8192 tokens at random positions, one-token pages.
        _case("draft_tokens_16x8k", "draft", batch=16, lo=8192, hi=8192, page=1),
        # Plain decoding of a ragged batch: one new token over each whole sequence, int8 codes.
        _case("decode_batch12_1k_48k", "draft", batch=12, heads=64, lo=1001, hi=48013, format="int8"),
        # The headline verification: 32K tokens, five rows per head, every page scored.
        _case("verify_32k", "verify", batch=1, queries=5, lo=32768, hi=32768, collect=1),
        # Verification of a ragged serving batch, 40 rows per KV head, every page scored.
        _case("verify_ragged16_8k_64k", "verify", batch=16, heads=64, queries=5, lo=8192, hi=65536, collect=1),
    ]


def _lengths(case) -> List[int]:
    """Lengths of the batch: spread over [lo, hi] in an order without pattern, fixed by the case alone."""
    lo, hi, n = case["lo"], case["hi"], case["batch"]
    return [lo + int((hi - lo) * math.fmod((i + 1) * 0.6180339887498949, 1.0)) for i in range(n)]


def _counts(case) -> List[int]:
    """New tokens of each sequence of an append: the first has all of them, the others fewer where there are many."""
    t, n = case["tokens"], case["batch"]
    return [t if i == 0 or t < 8 else t - int(0.4 * t * math.fmod(i * 0.7548776662466927, 1.0)) for i in range(n)]


def work(case) -> Dict[str, float]:
    """Each input once, each output once."""
    B, Hq, Hkv, D, G = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["queries"]
    cached = Hkv * (2 * D + 8)                                   # a token's K and V codes and scales
    if case["kind"] == "rotate":
        tokens = B * case["tokens"]
        return {"bytes": tokens * (4.0 * Hq * D + 4), "flops": 3.0 * tokens * Hq * case["rot"]}
    if case["kind"] == "append":
        tokens = sum(_counts(case))
        q = 4.0 * Hq * D if case["rot"] else 0.0
        return {"bytes": tokens * (4.0 * Hkv * D + cached + q), "flops": tokens * (6.0 * Hkv * D + 3.0 * (Hkv + Hq) * case["rot"])}
    lens = _lengths(case)
    total = sum(lens)
    if case["kind"] == "read":
        return {"bytes": total * (cached + 4.0 * Hkv * D), "flops": 2.0 * total * Hkv * D}
    nbytes = total * cached + 4.0 * B * G * Hq * D + sum(4 * -(-n // case["page"]) for n in lens)
    if case["collect"]:
        nbytes += sum(4 * -(-n // PAGE) for n in lens)
    return {"bytes": nbytes, "flops": 4.0 * total * G * Hq * D}


def draw(rng) -> Dict[str, object]:
    """Another case of the same ranges: 1 to 32 sequences, 1 to 131072 tokens, both head dimensions and formats, groups of 1
    to 8 heads, 1 to 12 verification rows, page lists of 1 to 16 tokens per page."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(work(c)["bytes"] for c in listed())
    most_flops = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["rotate", "append", "read", "draft", "draft", "verify", "verify"])
        heads, kv_heads = rng.choice([(32, 8), (32, 8), (64, 8), (16, 8), (28, 4), (40, 8), (8, 8)])
        dim = rng.choice([128, 128, 64])
        c = _case("", kind, heads=heads, kv_heads=kv_heads, dim=dim, format=rng.choice(["e4m3", "int8"]), batch=log_int(1, 32))
        del c["name"]
        if kind in ("rotate", "append"):
            c["tokens"] = log_int(1, 8192 if kind == "rotate" else 4096)
            c["hi"] = log_int(16, 131072)
            c["lo"] = int(c["hi"] * rng.choice([1.0, 0.5, 0.0]))
            c["rot"] = rng.choice([dim, dim, dim // 2, dim // 4, 16, dim - 16])
            c["layout"] = rng.choice(["half", "interleaved"])
            c["scaling"] = rng.choice(["none", "linear", "ntk", "yarn"])
            if kind == "rotate":
                c["kv_heads"] = 0
            elif c["format"] == "int8":
                c["rot"] = 0                                     # (keys that came rotated)
            if c["batch"] * c["tokens"] > 32768 or c["batch"] * (c["hi"] + c["tokens"]) > 600000:
                continue
        else:
            c["hi"] = log_int(40, 131072)
            c["lo"] = max(1, int(c["hi"] * rng.choice([1.0, 0.7, 0.25, 0.1])))
            if kind == "read":
                c["tokens"] = c["hi"]
            elif kind == "draft":
                c["page"] = rng.choice([1, 2, 4, 8, 16, 16, 16])
            else:
                c["queries"] = rng.randint(1, 12)
                c["collect"] = rng.choice([0, 1, 1, 2])
                if c["queries"] * (heads // kv_heads) > 96:
                    continue
        if work(c)["bytes"] > most or work(c)["flops"] > most_flops:
            continue
        if c["kind"] in ("draft", "read", "verify") and c["batch"] * c["hi"] > 1100000:
            continue
        return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------

def _normal(shape, gen) -> torch.Tensor:
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)


def _frequencies(case):
    """(radians per position float64 [rot / 2], magnitude): base 1e6; linear, NTK-aware and YaRN scaling by four."""
    rot, base, factor = case["rot"], 1.0e6, 4.0
    if rot == 0:
        return None, 1.0
    if case["scaling"] == "ntk" and rot > 2:
        base *= factor ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if case["scaling"] == "linear":
        return (f / factor).to(DEVICE), 1.0
    if case["scaling"] == "yarn":
        # dims that turn more than 32 times over the original length keep their frequency, those below once are interpolated
        def dim_of(turns):
            return rot * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(math.floor(dim_of(32.0)), 0), min(math.ceil(dim_of(1.0)), rot - 1)
        ramp = ((torch.arange(rot // 2, dtype=torch.float64) - low) / max(high - low, 0.001)).clamp(0, 1)
        return (f / factor * ramp + f * (1 - ramp)).to(DEVICE), 0.1 * math.log(factor) + 1.0
    return f.to(DEVICE), 1.0


def _quantise(x, fmt):
    """(codes, scales) of fp32 rows x [..., D]: the row's largest magnitude becomes the format's."""
    top = TOP[fmt]
    a = x.abs().amax(-1)
    live = a >= TINY
    scale = torch.where(live, a / top, torch.zeros_like(a))
    inv = torch.where(live, top / a, torch.zeros_like(a))
    y = x * inv[..., None]
    return (torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)), scale


def _cache(case, pages, gen, direction=None):
    """K and V codes and scales of a pool of unit normals; every page's keys shifted along `direction` by an importance of its
    own, so that some pages carry most of the weight."""
    Hkv, D, fmt = case["kv_heads"], case["dim"], case["format"]
    k = torch.empty((pages, PAGE, Hkv, D), dtype=CODES[fmt], device=DEVICE)
    v = torch.empty_like(k)
    scales = torch.empty((pages, Hkv, 2, PAGE), dtype=torch.float32, device=DEVICE)
    step = max(1, (1 << 26) // (PAGE * Hkv * D))
    for p0 in range(0, pages, step):
        count = min(step, pages - p0)
        for w, codes in enumerate((k, v)):
            x = _normal((count, PAGE, Hkv, D), gen)
            if w == 0 and direction is not None:
                x += 4.0 * _normal((count, 1, 1, 1), gen) * direction
            c, s = _quantise(x, fmt)
            codes[p0:p0 + count] = c
            scales[p0:p0 + count, :, w] = s.transpose(1, 2)
    return k, v, scales


def _tables(counts, gen):
    """Pages handed out in random order (the last page of the pool belongs to nobody), rows padded with -1."""
    pages = sum(counts)
    order = torch.randperm(pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.full((len(counts), max(max(counts), 1)), -1, dtype=torch.int32, device=DEVICE)
    first = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[first:first + c]
        first += c
    return table, pages + 1


def prepare(case, seed: int):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    kind = case["kind"]
    B, Hq, Hkv, D, G, T = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["queries"], case["tokens"]
    lens = _lengths(case)
    s = dict(case=dict(case), scale=1.0 / math.sqrt(D))
    s["freq"], s["magnitude"] = _frequencies(case)
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEVICE)
    if kind == "rotate":
        s["x"] = _normal((B * T, Hq, D), gen).to(torch.bfloat16)
        s["positions"] = (lens_t[:, None] + torch.arange(T, dtype=torch.int32, device=DEVICE)).reshape(-1).contiguous()
    elif kind == "append":
        counts = _counts(case)
        s["table"], pages = _tables([-(-(n + t) // PAGE) for n, t in zip(lens, counts)], gen)
        s["k"], s["v"], s["scales"] = _cache(case, pages, gen)
        s["k_new"], s["v_new"] = (_normal((B, T, Hkv, D), gen).to(torch.bfloat16) for _ in range(2))
        s["q"] = _normal((B, T, Hq, D), gen).to(torch.bfloat16) if case["rot"] else None
        s["lens"], s["counts"] = lens_t, torch.tensor(counts, dtype=torch.int32, device=DEVICE)
    else:
        direction = _normal((max(Hkv, 1), D), gen)
        direction /= direction.norm(dim=-1, keepdim=True)
        # verification reads a whole sequence, a draft call or a read a list of pages out of a pool twice as large
        ps = case["page"]
        table, pages = _tables([-(-n // PAGE) for n in lens], gen)
        s["k"], s["v"], s["scales"] = _cache(case, pages, gen, direction)
        if ps < PAGE:
            per = PAGE // ps                                     # small pages of a sequence's own, in random order
            small = table[:, :, None] * per + torch.arange(per, dtype=torch.int32, device=DEVICE)
            key = torch.rand(small.shape, generator=gen, device=DEVICE)
            valid = torch.arange(table.shape[1] * PAGE, device=DEVICE).view(1, -1, per, ps)[..., 0] < lens_t.view(-1, 1, 1)
            key = torch.where(valid, key, torch.full_like(key, 2.0)).reshape(B, -1)
            table = small.reshape(B, -1).gather(1, key.argsort(dim=1))
            table = table[:, :-(-max(lens) // ps)].contiguous()
        s["table"], s["lens"] = table, lens_t
        along = 0.25 * math.sqrt(D) * direction.repeat_interleave(max(Hq // max(Hkv, 1), 1), dim=0)
        s["q"] = (_normal((B, G, Hq, D), gen) + along).to(torch.bfloat16)
        if kind == "draft":
            s["q"] = s["q"][:, 0].contiguous()
    if own:
        _handles(s)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the package's calls
# ---------------------------------------------------------------------------------------------------------------------

def _handles(s):
    """Descriptors, outputs and workspace, as a program that calls the package keeps them."""
    from paper_2602_07223_amd import binding as vb
    c = s["case"]
    B, Hq, Hkv, D, G, T = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["queries"], c["tokens"]
    kind, dev = c["kind"], s["freq"].device if s["freq"] is not None else s["lens"].device
    s["vb"], s["stream"] = vb, torch.cuda.current_stream().cuda_stream
    bf16 = dict(dtype=torch.bfloat16, device=dev)
    if s["freq"] is not None:
        s["rope"] = vb.make_rope(s["freq"], c["rot"], vb.ROPE_HALF if c["layout"] == "half" else vb.ROPE_INTERLEAVED, s["magnitude"])
    else:
        s["rope"] = None
    if kind == "rotate":
        s["out"] = torch.empty_like(s["x"])
        return
    s["quant"] = vb.make_quant(s["k"], s["v"], s["scales"], vb.QUANT_E4M3 if c["format"] == "e4m3" else vb.QUANT_INT8)
    width = s["table"].shape[1]
    room = dict(batch=B, num_q_heads=Hq, num_kv_heads=Hkv, num_queries=G, max_blocks=width, max_sel_blocks=width, head_dim=D,
                softmax_scale=s["scale"])
    pages = s["k"].shape[0]
    if kind == "append":
        s["desc"] = vb.make_desc(max_seq_len=width * PAGE, num_pages=pages, **room)
        s["q_out"] = torch.zeros_like(s["q"]) if s["q"] is not None else None
        s["after"] = torch.empty_like(s["lens"])
        s["new"] = vb.make_new_tokens(s["k_new"], s["v_new"], T, new_lens=s["counts"], q=s["q"], q_out=s["q_out"])
        return
    s["desc"] = vb.make_desc(max_seq_len=max(_lengths(c)), num_pages=pages * (PAGE // c["page"]), page_size=c["page"],
                             collect_rows=c["collect"], **room)
    if kind == "read":
        s["k_out"], s["v_out"] = (torch.zeros((B, T, Hkv, D), **bf16) for _ in range(2))
        return
    s["workspace"] = torch.empty(vb.vegas_quant_workspace_bytes(s["desc"]), dtype=torch.uint8, device=dev)
    s["out"] = torch.empty(s["q"].shape, **bf16)
    s["scores"] = torch.empty((B, width), dtype=torch.float32, device=dev) if c["collect"] else None


def _run_own(s):
    c, vb = s["case"], s["vb"]
    kind = c["kind"]
    if kind == "rotate":
        vb.vegas_rotate(s["rope"], c["dim"], s["x"].shape[0], c["heads"], s["positions"], s["x"], s["out"], stream=s["stream"])
        return s["out"]
    if kind == "append":
        vb.vegas_append_quant(s["desc"], s["quant"], s["rope"], s["new"], s["table"], s["lens"], s["after"], stream=s["stream"])
        return s["k"], s["v"], s["scales"], s["after"], s["q_out"]
    if kind == "read":
        vb.vegas_read_quant(s["desc"], s["quant"], s["table"], s["lens"], None, c["tokens"], s["k_out"], s["v_out"], stream=s["stream"])
        return s["k_out"], s["v_out"]
    if kind == "draft":
        vb.vegas_draft_attention_quant(s["desc"], s["quant"], s["q"], s["table"], s["lens"], s["out"], s["workspace"], stream=s["stream"])
        return s["out"]
    vb.vegas_verify_attention_quant(s["desc"], s["quant"], s["q"], s["table"], s["lens"], s["out"], s["scores"], s["workspace"],
                                    stream=s["stream"])
    return s["out"], s["scores"]


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------

def _turned(x, positions, s):
    """x [N, H, D] (fp32) rotated by positions [N]: angles in 64 bits, the rotation in 32."""
    c = s["case"]
    rot = c["rot"]
    angle = positions.double()[:, None] * s["freq"]
    cos = (angle.cos().float() * s["magnitude"])[:, None]
    sin = (angle.sin().float() * s["magnitude"])[:, None]
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat((a * cos - b * sin, a * sin + b * cos, x[..., rot:]), -1)
    a, b = x[..., :rot:2], x[..., 1:rot:2]
    return torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2), x[..., rot:]), -1)


def _slots(s, count):
    """Cache slots [B, count] of the listed tokens (those past a row's length: slot 0)."""
    ps = s["case"]["page"]
    at = torch.arange(count, device=s["table"].device)
    slots = s["table"].long()[:, (at // ps).clamp(max=s["table"].shape[1] - 1)] * ps + at % ps
    return torch.where(at < s["lens"].long()[:, None], slots, torch.zeros_like(slots))


def _gather(s, which, slots):
    """fp32 [B, count, Hkv, D]: the values that the cached codes stand for."""
    codes = s["k"] if which == 0 else s["v"]
    flat = codes.view(-1, *codes.shape[2:])
    scale = s["scales"][:, :, which].transpose(1, 2).reshape(-1, codes.shape[2])
    return flat.view(torch.uint8)[slots].view(codes.dtype).float() * scale[slots][..., None]


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    B, Hq, Hkv, D, G, T = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["queries"], c["tokens"]
    if kind == "rotate":
        return _turned(s["x"].float(), s["positions"], s).to(torch.bfloat16)
    if kind == "append":
        t = torch.arange(T, device=s["lens"].device)
        pos = s["lens"][:, None] + t
        k, v = s["k_new"].float(), s["v_new"].float()
        q_out = None
        live = t < s["counts"][:, None]
        if c["rot"]:
            k = _turned(k.view(B * T, Hkv, D), pos.reshape(-1), s).view(B, T, Hkv, D)
            q_out = _turned(s["q"].float().view(B * T, Hq, D), pos.reshape(-1), s).view(B, T, Hq, D).to(torch.bfloat16)
            q_out = torch.where(live[..., None, None], q_out, torch.zeros_like(q_out))
        spare = s["k"].shape[0] - 1                              # rows past a sequence's own go where they were read
        page = torch.gather(s["table"], 1, (pos // PAGE).clamp(max=s["table"].shape[1] - 1).long()).long()
        page = torch.where(live, page, torch.full_like(page, spare))
        slot = torch.where(live, pos % PAGE, torch.zeros_like(pos)).long()
        for which, (x, cache) in enumerate(((k, s["k"]), (v, s["v"]))):
            codes, scale = _quantise(x, c["format"])
            old, kept = cache.view(torch.uint8)[page, slot], s["scales"][page, :, which, slot]
            cache.view(torch.uint8)[page, slot] = torch.where(live[..., None, None], codes.view(torch.uint8), old)
            s["scales"][page, :, which, slot] = torch.where(live[..., None], scale, kept)
        return s["k"], s["v"], s["scales"], s["lens"] + s["counts"], q_out
    if kind == "read":
        slots = _slots(s, T)
        live = (torch.arange(T, device=slots.device) < s["lens"][:, None])[..., None, None]
        return tuple(torch.where(live, x, torch.zeros_like(x)).to(torch.bfloat16)
                     for x in (_gather(s, 0, slots), _gather(s, 1, slots)))
    n = max(_lengths(c))
    slots = _slots(s, n)
    q = s["q"].float().view(B, G, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(B, Hkv, -1, D)        # rows (t, head of the group)
    k = _gather(s, 0, slots).permute(0, 2, 3, 1).contiguous()
    logits = torch.matmul(q, k) * s["scale"]
    del k
    at = torch.arange(n, device=q.device)
    row = torch.arange(G, device=q.device).repeat_interleave(Hq // Hkv)
    seen = at <= (s["lens"][:, None, None] - G + row[:, None])                                     # [B, rows, n]
    logits = logits.masked_fill(~seen[:, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    w = torch.exp(logits - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    del logits
    total = w.sum(-1, keepdim=True)
    w /= torch.where(total > 0, total, torch.ones_like(total))
    out = torch.matmul(w, _gather(s, 1, slots).transpose(1, 2).contiguous())
    out = out.view(B, Hkv, G, -1, D).transpose(1, 2).reshape(s["q"].shape).to(torch.bfloat16)
    if kind == "draft":
        return out
    if not c["collect"]:
        return out, None
    picked = w.view(B, Hkv, G, -1, n)
    rows = G if c["collect"] == 1 else min(G, 2)
    if c["collect"] == 2 and G > 2:
        picked = picked[:, :, ::G - 1]
    per_token = picked.sum((1, 2, 3))
    per_token = torch.nn.functional.pad(per_token, (0, s["table"].shape[1] * PAGE - n))
    return out, per_token.view(B, -1, PAGE).sum(-1) / (rows * Hq)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------------------------------
# the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------------------------------

def _exact_turn(x, pos, freq, magnitude, rot, layout):
    """x [N, H, D] float64, as multiplication by unit complex numbers."""
    z = torch.polar(torch.full((len(pos), rot // 2), magnitude, dtype=torch.float64, device=x.device), pos.double()[:, None] * freq)[:, None]
    y = x.clone()
    first = slice(0, rot // 2) if layout == "half" else slice(0, rot, 2)
    second = slice(rot // 2, rot) if layout == "half" else slice(1, rot, 2)
    turned = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z
    y[..., first], y[..., second] = turned.real, turned.imag
    return y


def _e4m3(y):
    """float64 to the nearest value of 4 significant bits (exponents from -6 on, multiples of 2^-9 below), ties to even."""
    exponent = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    return torch.round(y / step) * step


def exact(case, seed: int):
    s = prepare(case, seed)
    B, Hq, Hkv, D, G, T = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["queries"], case["tokens"]
    kind, lens, ps = case["kind"], _lengths(case), case["page"]
    if kind == "rotate":
        return _exact_turn(s["x"].double(), s["positions"], s["freq"], s["magnitude"], case["rot"], case["layout"])
    if kind == "append":
        k, v, scales = s["k"].double(), s["v"].double(), s["scales"].double()
        counts, table = _counts(case), s["table"].long()
        q_out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE) if s["q"] is not None else None
        for b, (n, t) in enumerate(zip(lens, counts)):
            pos = torch.arange(n, n + t, device=DEVICE)
            page, slot = table[b, pos // PAGE], pos % PAGE
            for which, (new, cache) in enumerate(((s["k_new"], k), (s["v_new"], v))):
                x = new[b, :t].double()
                if which == 0 and case["rot"]:
                    x = _exact_turn(x, pos, s["freq"], s["magnitude"], case["rot"], case["layout"])
                scale = x.abs().amax(-1) / TOP[case["format"]]
                y = x / scale.clamp(min=1e-300)[..., None]
                cache[page, slot] = _e4m3(y) if case["format"] == "e4m3" else torch.round(y)
                scales[page, :, which, slot] = scale
            if q_out is not None:
                q_out[b, :t] = _exact_turn(s["q"][b, :t].double(), pos, s["freq"], s["magnitude"], case["rot"], case["layout"])
        after = torch.tensor([n + t for n, t in zip(lens, counts)], device=DEVICE)
        if case["format"] == "int8":
            k, v = k.to(torch.int8), v.to(torch.int8)
        return k, v, scales, after, q_out

    def values(b, which, first, count):
        pos = torch.arange(first, first + count, device=DEVICE)
        slot = s["table"].long()[b, pos // ps] * ps + pos % ps
        codes = (s["k"], s["v"])[which].view(-1, Hkv, D).view(torch.uint8)[slot].view(s["k"].dtype)
        return codes.double() * s["scales"][slot // PAGE, :, which, slot % PAGE].double()[..., None]

    if kind == "read":
        out = [torch.zeros((B, T, Hkv, D), dtype=torch.float64, device=DEVICE) for _ in range(2)]
        for b, n in enumerate(lens):
            for which in range(2):
                out[which][b, :n] = values(b, which, 0, n)
        return tuple(out)
    if work(case)["flops"] > 1.2e11:                             # (seconds in 64 bits)
        heads_at_once = 2
    else:
        heads_at_once = Hkv
    g = Hq // Hkv
    out = torch.zeros((B, G, Hq, D), dtype=torch.float64, device=DEVICE)
    scores = torch.zeros((B, s["table"].shape[1]), dtype=torch.float64, device=DEVICE)
    rows = [t for t in range(G)] if case["collect"] == 1 else sorted({0, G - 1})
    for b, n in enumerate(lens):
        kb, vb_ = values(b, 0, 0, n), values(b, 1, 0, n)
        per_token = torch.zeros(n, dtype=torch.float64, device=DEVICE)
        for h in range(0, Hkv, heads_at_once):
            hs = slice(h, min(h + heads_at_once, Hkv))
            q = s["q"].view(B, G, Hkv, g, D)[b][:, hs].double()                                   # [G, heads, g, D]
            logits = torch.einsum("thgd,nhd->thgn", q, kb[:, hs]) * s["scale"]
            seen = torch.arange(n, device=DEVICE) <= (n - G + torch.arange(G, device=DEVICE))[:, None]
            logits = torch.where(seen[:, None, None], logits, torch.full_like(logits, -math.inf))
            w = torch.nan_to_num(torch.softmax(logits, -1), nan=0.0)
            out.view(B, G, Hkv, g, D)[b][:, hs] = torch.einsum("thgn,nhd->thgd", w, vb_[:, hs])
            per_token += w[rows].sum((0, 1, 2))
        pages = -(-n // PAGE)
        scores[b, :pages] = torch.nn.functional.pad(per_token, (0, pages * PAGE - n)).view(pages, PAGE).sum(-1) / (len(rows) * Hq)
    if kind == "draft":
        return out[:, 0]
    return out, scores if case["collect"] else None
