"""Rotary positions, the quantising append and reading back on the GPU, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_07223_amd import binding as vb
from tests import quant_ref as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FMT = {"e4m3": vb.QUANT_E4M3, "int8": vb.QUANT_INT8}
LAYOUT = {"half": vb.ROPE_HALF, "interleaved": vb.ROPE_INTERLEAVED}


def stream():
    return torch.cuda.current_stream().cuda_stream


def make_rope(rot, layout, scaling=vb.ROPE_SCALE_NONE):
    freq, magnitude = vb.vegas_rope_frequencies(rot, 1e6, scaling, 4.0, 32768)
    return vb.make_rope(torch.tensor(freq, dtype=torch.float64, device=DEV), rot, LAYOUT[layout], magnitude), freq, magnitude


def f64(t):
    return t.detach().cpu().float().numpy().astype(np.float64)


@pytest.mark.parametrize("tokens,heads,dim,rot,layout,scaling,far", [
    (1, 1, 128, 128, "half", vb.ROPE_SCALE_NONE, 100),
    (1, 1, 64, 16, "interleaved", vb.ROPE_SCALE_NONE, 100),
    (5, 32, 128, 128, "half", vb.ROPE_SCALE_YARN, 131072),
    (80, 64, 128, 64, "interleaved", vb.ROPE_SCALE_LINEAR, 131072),
    (7, 40, 128, 112, "half", vb.ROPE_SCALE_NTK, 1 << 20),
    (3, 9, 64, 64, "half", vb.ROPE_SCALE_NONE, 1 << 20),
    (333, 17, 64, 48, "interleaved", vb.ROPE_SCALE_YARN, 65536),
    (1021, 33, 128, 128, "interleaved", vb.ROPE_SCALE_NONE, 1 << 27),
    (4099, 10, 128, 96, "half", vb.ROPE_SCALE_NONE, 32768),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_rotate(tokens, heads, dim, rot, layout, scaling, far, in_place):
    g = torch.Generator().manual_seed(tokens + heads)
    x = torch.randn((tokens, heads, dim), generator=g).to(torch.bfloat16)
    pos = torch.randint(0, far, (tokens,), generator=g, dtype=torch.int32)
    rope, freq, magnitude = make_rope(rot, layout, scaling)
    xd = x.to(DEV)
    out = xd if in_place else torch.full_like(xd, 7.0)
    vb.vegas_rotate(rope, dim, tokens, heads, pos.to(DEV), xd, out, stream=stream())
    ref = Q.rotated(f64(x), pos.numpy(), freq, magnitude, layout)
    err = np.abs(f64(out) - ref)
    # bf16: half a step; pairs: fp32 rotation
    assert (err <= 2.0 ** -8 * np.abs(ref) + Q.turn_slack(f64(x), freq, magnitude, layout)).all(), err.max()
    assert torch.equal(out.cpu()[..., rot:], x[..., rot:])


def test_rotate_heads_inside_a_projection_row():
    """Queries and keys of one fused projection [tokens, (Hq + 2 Hkv) * D], rotated where they lie: values and neighbours stay."""
    tokens, hq, hkv, dim = 37, 8, 2, 128
    rows = torch.randn((tokens, hq + 2 * hkv, dim), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    pad = torch.full((tokens, hq + 2 * hkv + 1, dim), 3.0, dtype=torch.bfloat16, device=DEV)
    pad[:, :-1] = rows.to(DEV)
    pos = torch.arange(tokens, dtype=torch.int32) * 11
    rope, freq, magnitude = make_rope(128, "half")
    part = pad[:, :hq + hkv]
    vb.vegas_rotate(rope, dim, tokens, hq + hkv, pos.to(DEV), part, part, stream=stream())
    ref = Q.rotated(f64(rows[:, :hq + hkv]), pos.numpy(), freq, magnitude, "half")
    err = np.abs(f64(pad[:, :hq + hkv]) - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + Q.turn_slack(f64(rows[:, :hq + hkv]), freq, magnitude, "half")).all()
    assert torch.equal(pad[:, hq + hkv:-1].cpu(), rows[:, hq + hkv:]) and (pad[:, -1] == 3.0).all()


def test_rotate_of_no_tokens_and_of_position_zero():
    rope, freq, magnitude = make_rope(64, "half")
    x = torch.randn((4, 3, 64), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    out = torch.full_like(x, 5.0)
    vb.vegas_rotate(rope, 64, 0, 3, torch.zeros(4, dtype=torch.int32, device=DEV), x, out, stream=stream())
    assert (out == 5.0).all()
    vb.vegas_rotate(rope, 64, 4, 3, torch.zeros(4, dtype=torch.int32, device=DEV), x, out, stream=stream())
    assert torch.equal(out, x)


class Pool:
    """A pool of 8-bit pages whose contents are known, with tables of pages in random order."""

    def __init__(self, lens, room, hkv, dim, fmt, seed, hnd=False):
        self.g = torch.Generator().manual_seed(seed)
        self.hkv, self.dim, self.fmt = hkv, dim, fmt
        counts = [-(-r // 16) for r in room]
        self.pages = sum(counts) + 2
        self.max_blocks = max(max(counts), 1) + 1
        order = torch.randperm(self.pages - 2, generator=self.g).to(torch.int32)
        self.table = torch.full((len(lens), self.max_blocks), -1, dtype=torch.int32)
        first = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = order[first:first + c]
            first += c
        self.lens = torch.tensor(lens, dtype=torch.int32)
        shape = (self.pages, 16, hkv, dim)
        raw = [torch.randint(-127, 127, shape, generator=self.g, dtype=torch.int8) for _ in range(2)]
        if fmt == "e4m3":
            raw = [(r.float() * 3).to(torch.float8_e4m3fn) for r in raw]
        self.host = raw
        self.scales = torch.rand((self.pages, hkv, 2, 16), generator=self.g) + 0.5
        self.hnd = hnd
        dev = [r.view(torch.uint8).to(DEV) for r in raw]
        if hnd:                                             # [page, head, slot, dim] in memory
            dev = [d.transpose(1, 2).contiguous().transpose(1, 2) for d in dev]
        self.k, self.v = dev
        self.dscales = self.scales.to(DEV)
        self.quant = vb.make_quant(self.k, self.v, self.dscales, FMT[fmt])

    def desc(self, hq, **over):
        kw = dict(batch=len(self.lens), num_q_heads=hq, num_kv_heads=self.hkv, num_queries=1, max_blocks=self.max_blocks,
                  max_sel_blocks=self.max_blocks, max_seq_len=self.max_blocks * 16, num_pages=self.pages, head_dim=self.dim, softmax_scale=0.1)
        if self.hnd:
            kw.update(kv_page_stride=16 * self.hkv * self.dim, kv_token_stride=self.dim, kv_head_stride=16 * self.dim)
        kw.update(over)
        return vb.make_desc(**kw)

    def codes(self, which):
        return (self.k, self.v)[which].cpu().contiguous().view(Q.DTYPE[self.fmt])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,new,counts,hq,hkv,dim,hnd", [
    ([0], 1, None, 8, 8, 128, False),
    ([15, 16, 17, 0], 1, None, 32, 8, 128, False),
    ([5, 31], 3, [3, 0], 28, 4, 128, False),
    ([7, 0, 33], 40, [40, 1, 17], 10, 5, 64, False),
    ([3], 130, None, 1, 1, 64, True),
    ([100, 9], 77, [76, 77], 64, 8, 128, True),
    ([0, 12], 515, [500, 515], 24, 12, 128, False),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_keys_that_come_rotated(fmt, lens, new, counts, hq, hkv, dim, hnd, in_place):
    """Codes, scales and lengths bit for bit; everything else in the cache as it was."""
    took = counts or [new] * len(lens)
    pool = Pool(lens, [n + c for n, c in zip(lens, took)], hkv, dim, fmt, seed=new + hkv, hnd=hnd)
    k, v = (torch.randn((len(lens), new, hkv, dim), generator=pool.g).to(torch.bfloat16) for _ in range(2))
    k[0, 0, 0] = 0.0                                        # a row of zeros, one below the smallest scale, one whose largest stands alone
    if took[0] > 1:
        k[0, 1, 0] = 2.0 ** -115
        v[0, 1, 0] = 0.0
        v[0, 1, 0, 5] = -3.0
    lens_d = pool.lens.to(DEV)
    after = lens_d if in_place else torch.full_like(lens_d, -7)
    tokens = vb.make_new_tokens(k.to(DEV), v.to(DEV), new, new_lens=None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV))
    vb.vegas_append_quant(pool.desc(hq), pool.quant, None, tokens, pool.table.to(DEV), lens_d, after, stream=stream())
    assert after.cpu().tolist() == [n + c for n, c in zip(lens, took)]
    want = [pool.host[0].clone(), pool.host[1].clone()]
    scales = pool.scales.clone()
    for b, (n, c) in enumerate(zip(lens, took)):
        for which, x in enumerate((k, v)):
            codes, sc = Q.quantise(x[b, :c].float().numpy(), fmt)
            for t in range(c):
                page, slot = int(pool.table[b, (n + t) // 16]), (n + t) % 16
                want[which].view(torch.uint8)[page, slot] = codes[t].view(torch.uint8)
                scales[page, :, which, slot] = torch.from_numpy(sc[t])
    for which in range(2):
        assert torch.equal(pool.codes(which).view(torch.uint8), want[which].view(torch.uint8)), which
    assert torch.equal(pool.dscales.cpu(), scales)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,new,counts,hq,hkv,dim,rot,layout,in_place", [
    ([1000], 1, None, 32, 8, 128, 128, "half", True),
    ([100000, 5, 77], 1, None, 64, 8, 128, 64, "interleaved", False),
    ([3, 60], 21, [21, 4], 9, 3, 64, 48, "half", True),
    ([0, 900], 130, [100, 130], 16, 4, 64, 64, "interleaved", False),
    ([50], 300, None, 40, 8, 128, 112, "half", True),
])
def test_append_with_rotation(fmt, lens, new, counts, hq, hkv, dim, rot, layout, in_place):
    """Keys within half a step of the rotated ones (codes are rounded once, from fp32), queries as vegas_rotate's, values untouched by
    the rotation; padding rows of q_out left alone."""
    took = counts or [new] * len(lens)
    pool = Pool(lens, [n + c for n, c in zip(lens, took)], hkv, dim, fmt, seed=new + dim)
    k, v = (torch.randn((len(lens), new, hkv, dim), generator=pool.g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((len(lens), new, hq, dim), generator=pool.g).to(torch.bfloat16)
    rope, freq, magnitude = make_rope(rot, layout, vb.ROPE_SCALE_YARN)
    lens_d, q_out = pool.lens.to(DEV), torch.full(q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
    after = lens_d if in_place else torch.full_like(lens_d, -7)
    tokens = vb.make_new_tokens(k.to(DEV), v.to(DEV), new, q=q.to(DEV), q_out=q_out,
                                new_lens=None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV))
    vb.vegas_append_quant(pool.desc(hq), pool.quant, rope, tokens, pool.table.to(DEV), lens_d, after, stream=stream())
    assert after.cpu().tolist() == [n + c for n, c in zip(lens, took)]
    got_scales = pool.dscales.cpu().numpy().astype(np.float64)
    for b, (n, c) in enumerate(zip(lens, took)):
        pos = np.arange(n, n + c)
        ref = Q.rotated(f64(k[b, :c]), pos, freq, magnitude, layout)
        slack = Q.turn_slack(f64(k[b, :c]), freq, magnitude, layout)
        page, slot = pool.table[b, pos // 16].long(), torch.from_numpy(pos % 16)
        codes = pool.codes(0).float()[page, slot].numpy().astype(np.float64)
        scale = got_scales[page, :, 0, slot][..., None]
        top = np.abs(ref).max(-1, keepdims=True)
        assert (np.abs(scale * Q.TOP[fmt] - top) <= 2.0 ** -22 * top + slack.max(-1, keepdims=True)).all()
        # half a step of the code: e4m3 2^-4 of the value, 2^-10 below its normal range; int8 1/2; and fp32 roundings of the product and scale
        half = np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * scale) if fmt == "e4m3" else 0.5 * scale
        assert (np.abs(codes * scale - ref) <= half + 2 * slack + 2.0 ** -21 * top).all()
        want, sc = Q.quantise(v[b, :c].float().numpy(), fmt)
        assert torch.equal(pool.codes(1)[page, slot].view(torch.uint8), want.view(torch.uint8))
        rq = Q.rotated(f64(q[b, :c]), pos, freq, magnitude, layout)
        assert (np.abs(f64(q_out[b, :c]) - rq) <= 2.0 ** -8 * np.abs(rq) + Q.turn_slack(f64(q[b, :c]), freq, magnitude, layout)).all()
        assert (q_out[b, c:] == 9.0).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_rows_that_are_not_finite_are_marked_and_their_codes_are_zero(fmt):
    pool = Pool([2], [20], 2, 128, fmt, seed=3)
    k, v = (torch.randn((1, 3, 2, 128), generator=pool.g).to(torch.bfloat16) for _ in range(2))
    k[0, 0, 1, 100] = float("inf")
    k[0, 1, 0, 3] = float("nan")
    v[0, 2, 1, 127] = -float("inf")
    after = torch.empty(1, dtype=torch.int32, device=DEV)
    vb.vegas_append_quant(pool.desc(4), pool.quant, None, vb.make_new_tokens(k.to(DEV), v.to(DEV), 3), pool.table.to(DEV), pool.lens.to(DEV), after,
                          stream=stream())
    page = int(pool.table[0, 0])
    sc = pool.dscales.cpu()[page]                           # [head, K or V, slot]
    bad = {(1, 0, 2), (0, 0, 3), (1, 1, 4)}
    for h in range(2):
        for w in range(2):
            for s in range(2, 5):
                assert torch.isnan(sc[h, w, s]).item() == ((h, w, s) in bad)
                if (h, w, s) in bad:
                    assert (pool.codes(w).view(torch.uint8)[page, s, h] == 0).all()
    ko, vo = (torch.zeros((1, 5, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    vb.vegas_read_quant(pool.desc(4), pool.quant, pool.table.to(DEV), after, None, 5, ko, vo, stream=stream())
    assert torch.isnan(ko[0, 2, 1]).all() and torch.isnan(ko[0, 3, 0]).all() and torch.isnan(vo[0, 4, 1]).all()
    assert torch.isfinite(ko[0, 2, 0]).all() and torch.isfinite(vo[0, 4, 0]).all()


@pytest.mark.parametrize("in_place,new", [(True, 2), (True, 70), (False, 2)])
def test_a_sequence_without_room_takes_nothing(in_place, new):
    """Room by the table row and by the descriptor's bound; the other sequences are served, and a count of zero needs no room."""
    lens = [10, 48 - new + 1, 40 if new == 2 else 0, 48]
    room = [128, 48, 128, 48]
    pool = Pool(lens, room, 2, 64, "int8", seed=8)
    table = pool.table[:, :8].contiguous()
    counts = torch.tensor([new, new, new, 0], dtype=torch.int32)
    desc = pool.desc(2, max_blocks=8, max_seq_len=10 + new if new == 70 else 41)
    k, v = (torch.randn((4, new, 2, 64), generator=pool.g).to(torch.bfloat16).to(DEV) for _ in range(2))
    lens_d = pool.lens.to(DEV)
    after = lens_d if in_place else torch.full_like(lens_d, -7)
    vb.vegas_append_quant(desc, pool.quant, None, vb.make_new_tokens(k, v, new, new_lens=counts.to(DEV)), table.to(DEV), lens_d, after, stream=stream())
    cap = min(desc.max_seq_len, 128)
    want = [n + c if n >= 0 and n + c <= cap else n for n, c in zip(lens, counts.tolist())]      # (a negative length has no room either)
    assert after.cpu().tolist() == want
    for b, n in enumerate(lens):
        if want[b] == n:
            for page in table[b][table[b] >= 0].tolist():
                assert torch.equal(pool.codes(0)[page], pool.host[0][page]) and torch.equal(pool.dscales.cpu()[page], pool.scales[page])


@pytest.mark.parametrize("sel_page", [16, 1])
@pytest.mark.parametrize("in_place", [True, False])
def test_append_grows_the_selection_as_extend_selection_does(sel_page, in_place):
    lens, new = [30, 5, 64, 16], 3
    pool = Pool(lens, [n + new for n in lens], 2, 64, "e4m3", seed=5)
    k, v = (torch.randn((4, new, 2, 64), generator=pool.g).to(torch.bfloat16).to(DEV) for _ in range(2))
    counts = torch.tensor([3, 0, 2, 3], dtype=torch.int32, device=DEV)
    width = 12 if sel_page == 16 else 40
    sel = torch.full((4, width), -1, dtype=torch.int32)
    sel_lens = torch.tensor([30, 5, 0, 16], dtype=torch.int32)
    for b, n in enumerate([30, 5, 0, 16]):
        for i in range(-(-n // sel_page)):
            sel[b, i] = pool.table[b, i] if sel_page == 16 else pool.table[b, i // 16] * 16 + i % 16
    desc = pool.desc(2, max_sel_blocks=width)
    sel_d, sel_lens_d, lens_d = sel.to(DEV), sel_lens.to(DEV), pool.lens.to(DEV)
    after = lens_d if in_place else torch.full_like(lens_d, -7)
    vb.vegas_append_quant(desc, pool.quant, None, vb.make_new_tokens(k, v, new, new_lens=counts), pool.table.to(DEV), lens_d, after, sel_d, sel_lens_d,
                          sel_page, stream=stream())
    want, want_lens = sel.clone(), sel_lens.clone()
    for b, (n, c) in enumerate(zip(lens, [3, 0, 2, 3])):
        if want_lens[b] == 0 or c == 0:
            continue
        count = (int(want_lens[b]) - 1) // sel_page + 1
        for i in range(n, n + c):
            if i % sel_page == 0:
                want[b, count] = pool.table[b, i // 16] * (16 // sel_page) + (i % 16) // sel_page
                count += 1
        want_lens[b] += c
    assert torch.equal(sel_d.cpu(), want) and torch.equal(sel_lens_d.cpu(), want_lens)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,first,tokens,hkv,dim,page,hnd", [
    ([1], None, 1, 8, 128, 16, False),
    ([0, 33], None, 40, 8, 128, 16, False),
    ([100, 17, 64], [0, 16, 70], 50, 3, 64, 16, False),
    ([100, 17], [95, -3], 20, 5, 128, 16, True),
    ([37, 50], None, 50, 2, 128, 1, False),
    ([37, 50, 9], [1, 0, 8], 45, 8, 64, 2, False),
    ([61], None, 61, 4, 128, 8, False),
])
def test_read(fmt, lens, first, tokens, hkv, dim, page, hnd):
    """Bit for bit: code * scale in fp32, rounded to bf16; rows past a list's end are left alone."""
    pool = Pool(lens, [max(n, 1) for n in lens], hkv, dim, fmt, seed=dim + page, hnd=hnd)
    if page == 16:
        table = pool.table
    else:                                                   # pages of a sequence in random order
        width = -(-max(lens) // page) + 2
        table = torch.full((len(lens), width), -1, dtype=torch.int32)
        per = 16 // page
        for b, n in enumerate(lens):
            pages = pool.table[b][pool.table[b] >= 0]
            small = (pages[:, None] * per + torch.arange(per, dtype=torch.int32)).reshape(-1)
            small = small[torch.randperm(len(small), generator=pool.g)]
            table[b, :min(width, len(small))] = small[:width]
    width = table.shape[1]
    small = dict(page_size=page, num_pages=pool.pages * (16 // page), kv_page_stride=page * hkv * dim) if page != 16 else {}
    desc = pool.desc(hkv, max_sel_blocks=width, max_seq_len=max(max(lens), 1), **small)
    out = [torch.full((len(lens), tokens, hkv, dim), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    vb.vegas_read_quant(desc, pool.quant, table.to(DEV), pool.lens.to(DEV), None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV),
                        tokens, out[0], out[1], stream=stream())
    for which in range(2):
        want = torch.full(out[0].shape, 9.0, dtype=torch.bfloat16)
        for b, n in enumerate(lens):
            f = max(first[b], 0) if first else 0
            for t in range(max(min(tokens, n - f), 0)):
                slot = int(table[b, (f + t) // page]) * page + (f + t) % page
                want[b, t] = (pool.host[which].float()[slot // 16, slot % 16] * pool.scales[slot // 16, :, which, slot % 16, None]).to(torch.bfloat16)
        assert torch.equal(out[which].cpu(), want), which


def test_strided_rows_of_a_fused_projection():
    """k, v and q as slices of one [tokens, (Hq + 2 Hkv) D] matrix; queries rotated where they lie."""
    lens, new, hq, hkv, dim = [4, 11], 5, 8, 2, 64
    pool = Pool(lens, [n + new for n in lens], hkv, dim, "int8", seed=4)
    width = (hq + 2 * hkv) * dim
    rows = torch.randn((2 * new, width), generator=pool.g).to(torch.bfloat16)
    dev = rows.to(DEV)
    rope, freq, magnitude = make_rope(64, "half")
    q, k, v = dev[:, :hq * dim], dev[:, hq * dim:(hq + hkv) * dim], dev[:, (hq + hkv) * dim:]
    tokens = vb.make_new_tokens(k, v, new, q=q, q_out=q, kv_token_stride=width, q_token_stride=width, q_out_token_stride=width)
    after = torch.empty(2, dtype=torch.int32, device=DEV)
    vb.vegas_append_quant(pool.desc(hq), pool.quant, rope, tokens, pool.table.to(DEV), pool.lens.to(DEV), after, stream=stream())
    pos = np.concatenate([np.arange(n, n + new) for n in lens])
    ref = Q.rotated(f64(rows[:, :hq * dim]).reshape(-1, hq, dim), pos, freq, magnitude, "half")
    slack = Q.turn_slack(f64(rows[:, :hq * dim]).reshape(-1, hq, dim), freq, magnitude, "half")
    assert (np.abs(f64(dev[:, :hq * dim]).reshape(-1, hq, dim) - ref) <= 2.0 ** -8 * np.abs(ref) + slack).all()
    assert torch.equal(dev[:, hq * dim:].cpu(), rows[:, hq * dim:])
    want, _ = Q.quantise(rows[:, (hq + hkv) * dim:].float().numpy().reshape(2, new, hkv, dim), "int8")
    for b, n in enumerate(lens):
        p = torch.arange(n, n + new)
        assert torch.equal(pool.codes(1)[pool.table[b, p // 16].long(), p % 16], want[b])


def test_a_corrupt_table_is_clamped_into_the_pool():
    """Page ids outside the pool: no fault, neighbours of the pool untouched (results are unspecified)."""
    pool = Pool([0], [32], 2, 64, "e4m3", seed=6)
    guard = torch.full((4096 + pool.k.numel() + 4096,), 0x55, dtype=torch.uint8, device=DEV)
    inner = guard[4096:4096 + pool.k.numel()].view(pool.k.shape)
    quant = vb.make_quant(inner, pool.v, pool.dscales, vb.QUANT_E4M3)
    table = torch.tensor([[1 << 30, -5, 0]], dtype=torch.int32, device=DEV)
    k, v = (torch.randn((1, 32, 2, 64), generator=pool.g).to(torch.bfloat16).to(DEV) for _ in range(2))
    after = torch.empty(1, dtype=torch.int32, device=DEV)
    vb.vegas_append_quant(pool.desc(2), quant, None, vb.make_new_tokens(k, v, 32), table, pool.lens.to(DEV), after, stream=stream())
    ko, vo = (torch.zeros((1, 32, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    vb.vegas_read_quant(pool.desc(2), quant, table, after, None, 32, ko, vo, stream=stream())
    torch.cuda.synchronize()
    assert (guard[:4096] == 0x55).all() and (guard[-4096:] == 0x55).all()
