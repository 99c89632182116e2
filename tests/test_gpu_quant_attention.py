"""Attention over an 8-bit cache on the GPU (verification with page scores, draft and decode calls) against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_07223_amd import binding as vb
from tests import quant_ref as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FMT = {"e4m3": vb.QUANT_E4M3, "int8": vb.QUANT_INT8}


def stream():
    return torch.cuda.current_stream().cuda_stream


def f64(t):
    return t.detach().cpu().float().numpy().astype(np.float64)


class Case:
    """A batch over a pool of random rows; what no sequence's list covers holds NaN codes (e4m3) and NaN scales."""

    def __init__(self, lens, hq, hkv, dim, fmt, G=1, page=16, seed=0, sharp=False, hnd=False, spare_width=1, max_len=0, spread=1.0):
        g = self.g = torch.Generator().manual_seed(1000 * seed + sum(lens) + hq + dim)
        self.lens, self.hq, self.hkv, self.dim, self.fmt, self.G, self.page = lens, hq, hkv, dim, fmt, G, page
        B = len(lens)
        pages16 = [-(-n // 16) for n in lens]
        self.pages = sum(pages16) + 1
        order = torch.randperm(self.pages - 1, generator=g).tolist()
        kf, vf = (torch.randn((self.pages, 16, hkv, dim), generator=g) * spread for _ in range(2))
        self.codes, self.scales = [], torch.empty((self.pages, hkv, 2, 16))
        for w, x in enumerate((kf, vf)):
            x = x * torch.exp(0.5 * torch.randn((self.pages, 16, hkv, 1), generator=g))       # scales of their own
            codes, sc = Q.quantise(x.numpy(), fmt)
            self.codes.append(codes)
            self.scales[:, :, w] = torch.from_numpy(sc).transpose(1, 2)
        per = 16 // page
        first, lists = 0, []
        for n, c in zip(lens, pages16):
            mine = order[first:first + c]
            first += c
            small = [p * per + i for p in mine for i in range(per)]
            if page != 16:
                small = [small[i] for i in torch.randperm(len(small), generator=g).tolist()]
            lists.append(small[:-(-n // page)])
        self.width = max(max(len(s) for s in lists), 1) + spare_width
        self.table = torch.full((B, self.width), -1, dtype=torch.int32)
        for b, s in enumerate(lists):
            self.table[b, :len(s)] = torch.tensor(s, dtype=torch.int32)
        self.q = (torch.randn((B, G, hq, dim), generator=g) * (4.0 if sharp else 1.0)).to(torch.bfloat16)
        self.scale = dim ** -0.5
        self.max_len = max_len or max(max(lens), 1)
        # poison
        used = torch.zeros((self.pages * 16,), dtype=torch.bool)
        self.slots = []
        for b, n in enumerate(lens):
            pos = torch.arange(n)
            s = self.table[b].long()[pos // page] * page + pos % page
            self.slots.append(s.numpy())
            used[s] = True
        bad = ~used.view(self.pages, 16)
        self.values = [Q.code_values(c) * self.scales[:, :, w].transpose(1, 2).numpy().astype(np.float64)[..., None] for w, c in enumerate(self.codes)]
        for c in self.codes:
            c.view(torch.uint8)[bad] = 0x7f                 # e4m3: NaN
        self.scales.permute(0, 3, 1, 2)[bad] = float("nan")
        dev = [c.view(torch.uint8).to(DEV) for c in self.codes]
        self.strides = {}
        if hnd:
            dev = [d.transpose(1, 2).contiguous().transpose(1, 2) for d in dev]
            self.strides = dict(kv_page_stride=16 * hkv * dim, kv_token_stride=dim, kv_head_stride=16 * dim)
        elif page != 16:
            self.strides = dict(kv_page_stride=page * hkv * dim)
        self.k, self.v = dev
        self.dscales = self.scales.to(DEV)
        self.quant = vb.make_quant(self.k, self.v, self.dscales, FMT[fmt])
        self.q_d, self.table_d = self.q.to(DEV), self.table.to(DEV)
        self.lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)

    def desc(self, **over):
        kw = dict(batch=len(self.lens), num_q_heads=self.hq, num_kv_heads=self.hkv, num_queries=self.G, max_blocks=self.width,
                  max_sel_blocks=self.width, max_seq_len=self.max_len, num_pages=self.pages * (16 // self.page), head_dim=self.dim,
                  page_size=self.page, softmax_scale=self.scale, collect_rows=vb.COLLECT_NONE, **self.strides)
        kw.update(over)
        return vb.make_desc(**kw)

    def check(self, out, scores=None, collect=0):
        got = f64(out).reshape(self.q.shape)
        for b, n in enumerate(self.lens):
            s = self.slots[b]
            k, v = (self.values[w].reshape(-1, self.hkv, self.dim)[s] for w in range(2))
            rows = list(range(self.G)) if collect == 1 else sorted({0, self.G - 1})
            ref, spread, l1, pages = Q.attention(f64(self.q[b]), k, v, n, self.G, self.scale, scores is not None, rows)
            err = np.abs(got[b] - ref)
            tol = Q.out_tolerance(ref, spread, l1, self.dim)
            assert (err <= tol).all(), (b, n, float(err.max()), float((err / tol).max()))
            if scores is not None:
                sc = scores[b].cpu().numpy().astype(np.float64)
                count = -(-n // 16)
                assert (sc[count:] == 0).all()
                if count:
                    rel = 2 * Q.weight_slack(l1, self.dim) + 1e-5       # numerator and log-sum-exp, fp32 sums of up to 10^4 terms
                    assert (np.abs(sc[:count] - pages) <= rel * pages + 1e-12).all(), (b, n, float((np.abs(sc[:count] - pages) / pages.clip(1e-30)).max()))

    def verify(self, collect=0, **over):
        desc = self.desc(collect_rows=collect, **over)
        out = torch.full(self.q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
        scores = torch.full((len(self.lens), self.width), 9.0, dtype=torch.float32, device=DEV) if collect else None
        ws = torch.full((vb.vegas_quant_workspace_bytes(desc),), 0xff, dtype=torch.uint8, device=DEV)
        vb.vegas_verify_attention_quant(desc, self.quant, self.q_d, self.table_d, self.lens_d, out, scores, ws, stream=stream())
        return out, scores

    def draft(self, **over):
        desc = self.desc(**over)
        out = torch.full((len(self.lens), self.hq, self.dim), 9.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.full((vb.vegas_quant_workspace_bytes(desc),), 0xff, dtype=torch.uint8, device=DEV)
        vb.vegas_draft_attention_quant(desc, self.quant, self.q_d, self.table_d, self.lens_d, out, ws, stream=stream())
        return out


LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1023, 4099]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("n", LENGTHS)
def test_draft_lengths(fmt, dim, n):
    c = Case([n], 8, 2, dim, fmt, seed=n)
    c.check(c.draft())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("n", LENGTHS)
def test_verify_lengths(fmt, dim, n):
    c = Case([n], 8, 2, dim, fmt, G=5, seed=n)
    out, scores = c.verify(collect=1)
    c.check(out, scores, 1)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (10, 5), (24, 8), (28, 4), (64, 8), (16, 1), (17, 1), (32, 1), (33, 1), (100, 1), (128, 1)])
@pytest.mark.parametrize("dim", [128, 64])
def test_draft_groups(fmt, hq, hkv, dim):
    """Groups of 1 to 128 heads: one or two 16-row tiles a workgroup, up to four of them."""
    c = Case([700, 0, 33], hq, hkv, dim, fmt, seed=hq)
    c.check(c.draft())
    c.check(c.draft(kv_chunk_tokens=128))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hkv,G,collect", [
    (8, 8, 1, 1), (8, 8, 16, 2), (32, 8, 5, 1), (32, 8, 5, 2), (64, 8, 5, 1), (28, 4, 7, 2), (16, 2, 12, 1), (40, 8, 12, 0), (12, 2, 8, 1),
    (8, 1, 16, 1), (8, 1, 16, 2), (4, 1, 32, 0), (10, 5, 2, 2), (2, 1, 33, 1), (7, 1, 17, 1)])
@pytest.mark.parametrize("dim", [128, 64])
def test_verify_rows(fmt, hq, hkv, G, collect, dim):
    """1 to 128 rows per KV head: one to three 16-row tiles a workgroup, sibling workgroups beyond; a ragged batch with an empty sequence and
    ones shorter than their rows (whose first rows see nothing)."""
    c = Case([900, 0, 33, 3, 1500], hq, hkv, dim, fmt, G=G, seed=G)
    out, scores = c.verify(collect=collect)
    c.check(out, scores, collect)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("page", [1, 2, 4, 8])
@pytest.mark.parametrize("lens,hq,hkv,dim", [([1], 8, 2, 128), ([45, 0, 700], 32, 8, 128), ([2049, 311], 28, 4, 64), ([33, 130], 20, 1, 128), ([640], 8, 8, 64)])
def test_draft_small_pages(fmt, page, lens, hq, hkv, dim):
    c = Case(lens, hq, hkv, dim, fmt, page=page, seed=page)
    c.check(c.draft())
    c.check(c.draft(kv_chunk_tokens=96))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("chunk", [32, 64, 96, 256, 1024, 4096])
def test_chunk_lengths_of_the_callers(fmt, chunk):
    c = Case([2500, 1, 0, 96, 1024], 20, 4, 128, fmt, G=3, seed=chunk)
    out, scores = c.verify(collect=1, kv_chunk_tokens=chunk)
    c.check(out, scores, 1)
    d = Case([2500, 1, 0, 96, 1024], 20, 4, 128, fmt, seed=chunk)
    d.check(d.draft(kv_chunk_tokens=chunk))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,hq,hkv,dim,G,loose", [
    ([8192], 32, 8, 128, 5, 0),
    ([20011, 1001, 9000, 15], 32, 8, 128, 5, 0),
    ([300] * 70, 8, 2, 64, 4, 0),                           # more sequences than are planned for
    ([5000, 70, 2000], 32, 8, 64, 6, 60000),                # a bound far above the lengths
    ([12345], 64, 8, 64, 5, 0),
    ([100 * (i % 7) for i in range(40)], 16, 4, 128, 3, 4000),
])
def test_batches(fmt, lens, hq, hkv, dim, G, loose):
    spare = max(-(-max(loose, 1) // 16) - -(-max(lens) // 16), 0) + 1
    c = Case(lens, hq, hkv, dim, fmt, G=G, seed=len(lens), spare_width=spare, max_len=loose)
    out, scores = c.verify(collect=1)
    c.check(out, scores, 1)
    out, _ = c.verify(collect=0)
    c.check(out)
    d = Case(lens, hq, hkv, dim, fmt, seed=len(lens), spare_width=spare, max_len=loose)
    d.check(d.draft())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [128, 64])
def test_sharp_weights_rising_maxima_and_large_values(fmt, dim):
    """Logits of standard deviation 4 with keys sorted so that a row's maximum rises all along, values of scale 100."""
    c = Case([1500, 257], 16, 4, dim, fmt, G=4, seed=3, sharp=True, spread=1.0)
    out, scores = c.verify(collect=1)
    c.check(out, scores, 1)
    c = Case([1500, 257], 16, 4, dim, fmt, seed=4, sharp=True, spread=10.0)
    # one query for all heads, keys in the order of its logits
    c.q[:] = c.q[:, :, :1]
    c.q_d = c.q.to(DEV)
    kv = c.values[0].reshape(-1, 4, dim)
    logits = kv[c.slots[0], 0] @ f64(c.q[0, 0, 0])
    order = np.argsort(logits)
    codes, scales = [x.clone() for x in c.codes], c.scales.clone()
    s = c.slots[0]
    for w in range(2):
        flat, sc = codes[w].view(torch.uint8).view(-1, 4, dim), scales[:, :, w].transpose(1, 2).reshape(-1, 4)
        flat[torch.from_numpy(s)], sc[torch.from_numpy(s)] = flat[torch.from_numpy(s[order])].clone(), sc[torch.from_numpy(s[order])].clone()
        scales[:, :, w] = sc.view(c.pages, 16, 4).transpose(1, 2)
        c.values[w].reshape(-1, 4, dim)[s] = c.values[w].reshape(-1, 4, dim)[s[order]].copy()
        (c.k, c.v)[w].copy_(codes[w].view(torch.uint8).to(DEV))
    c.dscales.copy_(scales.to(DEV))
    c.check(c.draft())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_head_major_pages_and_other_strides(fmt):
    c = Case([1000, 17], 16, 4, 128, fmt, G=3, seed=9, hnd=True)
    out, scores = c.verify(collect=1)
    c.check(out, scores, 1)
    d = Case([1000, 17], 16, 4, 64, fmt, seed=9, hnd=True)
    d.check(d.draft())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_later_token_that_is_not_finite_leaves_earlier_rows_alone(fmt):
    """The last of four verification tokens has K and V rows marked NaN: rows 0 .. 2 do not see them."""
    c = Case([200], 8, 2, 128, fmt, G=4, seed=11)
    slot = int(c.slots[0][-1])
    c.dscales[slot // 16, :, :, slot % 16] = float("nan")
    c.k.view(-1, 2, 128)[slot] = 0
    c.v.view(-1, 2, 128)[slot] = 0
    out, _ = c.verify()
    got = f64(out)[0, :3]
    k, v = (c.values[w].reshape(-1, 2, 128)[c.slots[0][:-1]] for w in range(2))
    ref, spread, l1, _ = Q.attention(f64(c.q[0, :3]), k, v, 199, 3, c.scale)
    assert (np.abs(got - ref) <= Q.out_tolerance(ref, spread, l1, 128)).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_repeated_pages_and_runs_are_the_same_bit_for_bit(fmt):
    c = Case([900, 40], 32, 8, 128, fmt, G=5, seed=12)
    first = c.verify(collect=1)
    again = c.verify(collect=1)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    # the same page listed twice counts twice
    d = Case([64], 8, 2, 128, fmt, seed=13)
    d.table[0, 1] = d.table[0, 0]
    d.table_d = d.table.to(DEV)
    pos = torch.arange(64)
    d.slots[0] = (d.table[0].long()[pos // 16] * 16 + pos % 16).numpy()
    d.check(d.draft())


def test_lengths_and_page_ids_out_of_range_are_clamped():
    """No fault; a length above the bound counts as the bound (page ids: results unspecified)."""
    c = Case([96], 8, 2, 128, "int8", seed=14)
    want = c.draft()
    c.lens_d = torch.tensor([1 << 29], dtype=torch.int32, device=DEV)
    assert torch.equal(c.draft(), want)
    c.lens_d = torch.tensor([-4], dtype=torch.int32, device=DEV)
    assert (c.draft() == 0).all()
    c.lens_d = torch.tensor([96], dtype=torch.int32, device=DEV)
    c.table_d = torch.tensor([[1 << 30, -9, 0, 0, 1, 2, 3]], dtype=torch.int32, device=DEV)[:, :c.width].contiguous()
    c.draft()
    c.verify(collect=1)
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,hq,hkv,dim,G,collect,chunk", [
    ([12300, 40], 10, 2, 128, 4, 1, 12320), ([9000], 6, 1, 64, 4, 2, 9024), ([20000, 19000, 33], 6, 2, 128, 15, 1, 0), ([17001], 10, 2, 64, 5, 2, 17024)])
def test_long_chunks(fmt, lens, hq, hkv, dim, G, collect, chunk):
    """Chunks of more tiles per wave than it has page ids and log-sum-exps at hand."""
    c = Case(lens, hq, hkv, dim, fmt, G=G, seed=21)
    out, scores = c.verify(collect=collect, kv_chunk_tokens=chunk)
    c.check(out, scores, collect)
    d = Case(lens, hq, hkv, dim, fmt, seed=22)
    d.check(d.draft(kv_chunk_tokens=chunk))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("lens,hq,hkv,page", [
    ([1000, 0, 37, 513], 8, 8, 16), ([3000, 1, 64, 0, 700, 128, 33, 2001, 90], 16, 8, 16), ([100, 2222, 5, 0, 257, 1000, 31, 64], 6, 6, 16),
    ([800, 4000], 10, 1, 16), ([1800, 500], 34, 2, 16), ([2500], 16, 4, 16), ([17 * i % 301 for i in range(70)], 8, 4, 16),
    ([3000, 1, 64, 0, 700, 128, 33, 2001, 90], 16, 8, 1), ([100, 2222, 5, 0, 257, 1000, 31, 64], 6, 2, 4), ([2500], 16, 4, 8),
    ([17 * i % 301 for i in range(70)], 4, 2, 2), ([900, 333], 100, 1, 1)])
def test_bounds_of_large_draft_calls(fmt, dim, lens, hq, hkv, page):
    """The lengths may lie far below the call's bound, which is what its workgroups and its plan are chosen by."""
    units = torch.cuda.get_device_properties(0).multi_processor_count
    bound = max(2048 * units // (len(lens) * hkv) + 77, max(lens) + 1, 1600)
    c = Case(lens, hq, hkv, dim, fmt, page=page, seed=31, spare_width=bound // page + 1, max_len=bound)
    c.check(c.draft())
    c.check(c.draft(kv_chunk_tokens=256))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("lens,hq,hkv,G", [
    ([1000, 0, 37, 513], 8, 8, 5), ([3000, 1, 64, 0, 700, 128, 33, 2001, 90], 64, 8, 5), ([100, 2222, 5, 0, 257, 1000, 31, 64], 18, 6, 6),
    ([800, 4000], 10, 1, 4), ([2500], 16, 4, 11), ([17 * i % 301 for i in range(70)], 8, 4, 3)])
def test_bounds_of_large_verification_calls(fmt, dim, lens, hq, hkv, G):
    units = torch.cuda.get_device_properties(0).multi_processor_count
    bound = max(2048 * units // (len(lens) * hkv) + 77, max(lens) + 1)
    c = Case(lens, hq, hkv, dim, fmt, G=G, seed=32, spare_width=bound // 16 + 1, max_len=bound)
    for collect in (0, 1, 2):
        out, scores = c.verify(collect=collect)
        c.check(out, scores, collect)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,hq,hkv,dim,G", [
    ([700, 0, 37, 513, 64, 1500, 9, 128, 333], 64, 8, 128, 7), ([700, 0, 37, 513, 64, 1500, 9, 128, 333], 32, 4, 64, 16), ([1200], 64, 8, 128, 16),
    ([900, 130], 16, 2, 128, 15), ([11 * i % 257 for i in range(66)], 28, 4, 64, 9)])
def test_row_blocks_of_large_verification_calls(fmt, lens, hq, hkv, dim, G):
    """More rows than a workgroup has, beside neighbouring heads in it."""
    units = torch.cuda.get_device_properties(0).multi_processor_count
    bound = max(2048 * units // (len(lens) * hkv) + 77, max(lens) + 1)
    c = Case(lens, hq, hkv, dim, fmt, G=G, seed=33, spare_width=bound // 16 + 1, max_len=bound)
    for collect in (0, 1, 2):
        out, scores = c.verify(collect=collect)
        c.check(out, scores, collect)
    out, scores = c.verify(collect=1, kv_chunk_tokens=512)
    c.check(out, scores, 1)
