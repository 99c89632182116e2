"""Host-side checks of the calls around an 8-bit cache and of the rotary frequencies, without a GPU: every refusal comes before a launch."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from paper_2602_07223_amd import binding as vb

A = 4096      # an aligned fake device address, never dereferenced
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def desc(**over):
    kw = dict(batch=2, num_q_heads=32, num_kv_heads=8, num_queries=5, max_blocks=2048, max_sel_blocks=2048, max_seq_len=32768,
              num_pages=4096, softmax_scale=0.1)
    kw.update(over)
    extra = {k: kw.pop(k) for k in ("reserved",) if k in kw}
    d = vb.make_desc(**kw)
    for k, v in extra.items():
        setattr(d, k, v)
    return d


def quant(k=A, v=A, scales=A, fmt=vb.QUANT_E4M3, reserved=0):
    c = vb.make_quant(k, v, scales, fmt)
    c.reserved = reserved
    return c


def rope(freq=A, rot=128, layout=vb.ROPE_HALF, magnitude=1.0, reserved=0):
    r = vb.make_rope(freq, rot, layout, magnitude)
    r.reserved = reserved
    return r


def tokens(k=A, v=A, num_new=1, reserved=0, **kw):
    n = vb.make_new_tokens(k, v, num_new, **kw)
    n.reserved = reserved
    return n


def refused(call, status):
    with pytest.raises(vb.VegasError) as e:
        call()
    assert e.value.status == status


BAD_CACHES = [
    (dict(k=None), vb.VEGAS_ERR_NULL), (dict(v=None), vb.VEGAS_ERR_NULL), (dict(scales=None), vb.VEGAS_ERR_NULL),
    (dict(fmt=2), vb.VEGAS_ERR_UNSUPPORTED), (dict(fmt=-1), vb.VEGAS_ERR_UNSUPPORTED), (dict(reserved=1), vb.VEGAS_ERR_SHAPE),
    (dict(k=A + 8), vb.VEGAS_ERR_ALIGN), (dict(v=A + 4), vb.VEGAS_ERR_ALIGN), (dict(scales=A + 4), vb.VEGAS_ERR_ALIGN),
]
BAD_DESCS = [
    (dict(batch=0), vb.VEGAS_ERR_SHAPE), (dict(num_q_heads=30), vb.VEGAS_ERR_SHAPE), (dict(head_dim=96), vb.VEGAS_ERR_UNSUPPORTED),
    (dict(page_size=32), vb.VEGAS_ERR_UNSUPPORTED), (dict(batch=65536), vb.VEGAS_ERR_UNSUPPORTED), (dict(reserved=1), vb.VEGAS_ERR_SHAPE),
    (dict(softmax_scale=0.0), vb.VEGAS_ERR_SHAPE), (dict(max_seq_len=0), vb.VEGAS_ERR_SHAPE), (dict(num_pages=0), vb.VEGAS_ERR_SHAPE),
    (dict(kv_token_stride=1032), vb.VEGAS_ERR_ALIGN), (dict(kv_head_stride=136), vb.VEGAS_ERR_ALIGN), (dict(kv_page_stride=16392), vb.VEGAS_ERR_ALIGN),
    (dict(kv_token_stride=1 << 27), vb.VEGAS_ERR_UNSUPPORTED),
]


def verify(d=None, c=None, q=A, table=A, lens=A, out=A, scores=A, ws=A, wb=1 << 40):
    vb.vegas_verify_attention_quant(d or desc(), c or quant(), q, table, lens, out, scores, ws, workspace_bytes=wb)


def draft(d=None, c=None, q=A, table=A, lens=A, out=A, ws=A, wb=1 << 40):
    vb.vegas_draft_attention_quant(d or desc(), c or quant(), q, table, lens, out, ws, workspace_bytes=wb)


def read(d=None, c=None, table=A, lens=A, first=None, num=16, ko=A, vo=A):
    vb.vegas_read_quant(d or desc(), c or quant(), table, lens, first, num, ko, vo)


def append(d=None, c=None, r=None, n=None, table=A, lens=A, after=A, sel=None, sel_lens=None, page=16):
    vb.vegas_append_quant(d or desc(), c or quant(), r, n or tokens(), table, lens, after, sel, sel_lens, page)


@pytest.mark.parametrize("call", [verify, draft, read, append])
def test_bad_caches_and_descriptors_are_refused(call):
    for over, status in BAD_CACHES:
        refused(lambda: call(c=quant(**over)), status)
    for over, status in BAD_DESCS:
        refused(lambda: call(d=desc(**over)), status)


def test_verification_refusals():
    for name in ("q", "table", "lens", "out", "scores"):
        refused(lambda: verify(**{name: None}), vb.VEGAS_ERR_NULL)
    for name in ("q", "table", "out", "scores"):
        refused(lambda: verify(**{name: A + 8}), vb.VEGAS_ERR_ALIGN)
    refused(lambda: verify(d=desc(page_size=8)), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: verify(d=desc(max_seq_len=32769)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: verify(d=desc(num_queries=0)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: verify(d=desc(num_queries=33)), vb.VEGAS_ERR_UNSUPPORTED)                   # 132 rows per KV head
    refused(lambda: verify(d=desc(num_queries=1 << 30)), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: verify(d=desc(collect_rows=3)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: verify(d=desc(window=-1)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: verify(d=desc(score_metric=2)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: verify(d=desc(collect_rows=0, window=128)), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: verify(d=desc(score_metric=vb.METRIC_TOKEN_LOGITS)), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: verify(d=desc(kv_chunk_tokens=100)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: verify(wb=1024), vb.VEGAS_ERR_WORKSPACE)
    refused(lambda: verify(ws=None), vb.VEGAS_ERR_WORKSPACE)
    refused(lambda: verify(ws=A + 16), vb.VEGAS_ERR_ALIGN)
    refused(lambda: verify(d=desc(max_seq_len=1 << 22, max_blocks=1 << 18, kv_chunk_tokens=32)), vb.VEGAS_ERR_UNSUPPORTED)   # chunks of a grid
    refused(lambda: verify(d=desc(num_q_heads=1024, num_kv_heads=256, num_queries=12)), vb.VEGAS_ERR_UNSUPPORTED)            # rows of a score workgroup


def test_draft_refusals():
    for name in ("q", "table", "lens", "out"):
        refused(lambda: draft(**{name: None}), vb.VEGAS_ERR_NULL)
    for name in ("q", "table", "out"):
        refused(lambda: draft(**{name: A + 8}), vb.VEGAS_ERR_ALIGN)
    refused(lambda: draft(d=desc(max_sel_blocks=0)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: draft(d=desc(max_sel_blocks=100)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: draft(d=desc(page_size=1)), vb.VEGAS_ERR_SHAPE)                             # 2048 pages of one token
    refused(lambda: draft(d=desc(num_q_heads=129, num_kv_heads=1)), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: draft(wb=1024), vb.VEGAS_ERR_WORKSPACE)
    refused(lambda: draft(ws=A + 16), vb.VEGAS_ERR_ALIGN)


def test_read_refusals():
    for name in ("table", "lens", "ko", "vo"):
        refused(lambda: read(**{name: None}), vb.VEGAS_ERR_NULL)
    refused(lambda: read(num=0), vb.VEGAS_ERR_SHAPE)
    refused(lambda: read(num=(1 << 30) + 1), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: read(d=desc(max_sel_blocks=100)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: read(ko=A + 8), vb.VEGAS_ERR_ALIGN)


def test_append_refusals():
    for name in ("table", "lens", "after"):
        refused(lambda: append(**{name: None}), vb.VEGAS_ERR_NULL)
    refused(lambda: append(n=tokens(k=None)), vb.VEGAS_ERR_NULL)
    refused(lambda: append(n=tokens(v=None)), vb.VEGAS_ERR_NULL)
    refused(lambda: append(r=rope(), n=tokens(q=A)), vb.VEGAS_ERR_NULL)
    refused(lambda: append(r=rope(), n=tokens(q_out=A)), vb.VEGAS_ERR_NULL)
    refused(lambda: append(n=tokens(q=A, q_out=A)), vb.VEGAS_ERR_NULL)                          # queries to rotate, and no rotation
    refused(lambda: append(n=tokens(num_new=0)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: append(n=tokens(num_new=(1 << 24) + 1)), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: append(n=tokens(reserved=1)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: append(n=tokens(kv_token_stride=1016)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: append(n=tokens(kv_token_stride=1028)), vb.VEGAS_ERR_ALIGN)
    refused(lambda: append(r=rope(), n=tokens(q=A, q_out=A, q_token_stride=8192)), vb.VEGAS_ERR_SHAPE)   # in place with two strides
    refused(lambda: append(n=tokens(k=A + 8)), vb.VEGAS_ERR_ALIGN)
    refused(lambda: append(d=desc(page_size=8)), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: append(lens=A, after=A + 4), vb.VEGAS_ERR_SHAPE)                            # neither in place nor apart
    refused(lambda: append(sel=A), vb.VEGAS_ERR_NULL)
    refused(lambda: append(sel_lens=A), vb.VEGAS_ERR_NULL)
    refused(lambda: append(sel=A, sel_lens=A, page=4), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: append(d=desc(max_sel_blocks=0), sel=A, sel_lens=A), vb.VEGAS_ERR_SHAPE)
    for over, status in ROPES:
        refused(lambda: append(r=rope(**over)), status)


ROPES = [(dict(freq=None), vb.VEGAS_ERR_NULL), (dict(rot=0), vb.VEGAS_ERR_SHAPE), (dict(rot=144), vb.VEGAS_ERR_SHAPE),
         (dict(rot=40), vb.VEGAS_ERR_UNSUPPORTED), (dict(layout=2), vb.VEGAS_ERR_UNSUPPORTED), (dict(reserved=1), vb.VEGAS_ERR_SHAPE),
         (dict(magnitude=math.inf), vb.VEGAS_ERR_SHAPE), (dict(freq=A + 4), vb.VEGAS_ERR_ALIGN)]


def rotate(r=None, dim=128, num=4, heads=8, pos=A, x=A, out=1 << 20, xs=(1024, 128), os_=(1024, 128)):
    vb.vegas_rotate(r or rope(), dim, num, heads, pos, x, out, x_strides=xs, out_strides=os_)


def test_rotate_refusals():
    for over, status in ROPES:
        refused(lambda: rotate(r=rope(**over)), status)
    refused(lambda: vb.vegas_rotate(None, 128, 4, 8, A, A, A), vb.VEGAS_ERR_NULL)
    for name in ("pos", "x", "out"):
        refused(lambda: rotate(**{name: None}), vb.VEGAS_ERR_NULL)
    refused(lambda: rotate(dim=96), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: rotate(num=-1), vb.VEGAS_ERR_SHAPE)
    refused(lambda: rotate(num=1 << 31), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: rotate(heads=0), vb.VEGAS_ERR_SHAPE)
    refused(lambda: rotate(heads=65536), vb.VEGAS_ERR_UNSUPPORTED)
    refused(lambda: rotate(x=A + 8), vb.VEGAS_ERR_ALIGN)
    refused(lambda: rotate(xs=(1028, 128)), vb.VEGAS_ERR_ALIGN)
    refused(lambda: rotate(os_=(1024, 64)), vb.VEGAS_ERR_SHAPE)
    refused(lambda: rotate(out=A, os_=(2048, 128)), vb.VEGAS_ERR_SHAPE)                         # in place with two strides
    rotate(num=0)                                                                               # nothing to do, nothing launched


def test_tensors_that_are_too_small_are_refused_before_the_library_is_reached():
    d = desc(max_blocks=4, max_sel_blocks=4, max_seq_len=64, num_pages=8)
    k = torch.zeros((8, 16, 8, 128), dtype=torch.uint8)
    sc = torch.zeros((8, 8, 2, 16))
    table, lens = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    out = torch.zeros((2, 5, 32, 128), dtype=torch.bfloat16)
    for cache in (vb.make_quant(k[:7].clone(), k, sc, 0), vb.make_quant(k, k[:7].clone(), sc, 0), vb.make_quant(k, k, sc[:7].clone(), 0)):
        with pytest.raises(ValueError):
            vb.vegas_draft_attention_quant(d, cache, out, table, lens, out, out)
        with pytest.raises(ValueError):
            vb.vegas_read_quant(d, cache, table, lens, None, 4, out, out)
    good = vb.make_quant(k, k, sc, 0)
    with pytest.raises(ValueError):
        vb.vegas_verify_attention_quant(d, good, out[:1].clone(), table, lens, out, sc, out)
    with pytest.raises(ValueError):
        vb.vegas_verify_attention_quant(d, good, out, table, lens, out, torch.zeros(7), out)
    new = vb.make_new_tokens(out[0, 0, :8].clone(), out, 1)
    with pytest.raises(ValueError):
        vb.vegas_append_quant(d, good, None, new, table, lens, lens)
    with pytest.raises(ValueError):
        vb.make_rope(torch.zeros(8), 16)                                                        # not float64
    with pytest.raises(ValueError):
        vb.vegas_rotate(vb.make_rope(torch.zeros(8, dtype=torch.float64), 16), 128, 11, 32, torch.zeros(11, dtype=torch.int32), out, out)


def test_workspace_covers_the_calls_over_an_8_bit_cache():
    """vegas_quant_workspace_bytes(desc) bytes are enough for either call, whatever they are planned as (with a bad pointer behind the check)."""
    for kw in (dict(), dict(batch=16, num_q_heads=64), dict(batch=1, head_dim=64), dict(batch=70, max_seq_len=5000), dict(num_queries=12, num_q_heads=64),
               dict(collect_rows=0), dict(max_seq_len=100), dict(kv_chunk_tokens=256)):
        d = desc(**kw)
        wb = vb.vegas_quant_workspace_bytes(d)
        refused(lambda: verify(d=d, ws=A + 16, wb=wb), vb.VEGAS_ERR_ALIGN)
        refused(lambda: draft(d=d, ws=A + 16, wb=wb), vb.VEGAS_ERR_ALIGN)


def test_structs_are_the_header_s(tmp_path):
    import shutil
    import subprocess
    cc = shutil.which("cc") or shutil.which("gcc")
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "vegas.h"\nint main(void) {\n' + "".join(
        f'printf("%zu ", sizeof({t}));\n' + "".join(f'printf("%zu ", offsetof({t}, {f}));\n' for f, _ in s._fields_)
        for t, s in (("vegas_quant", vb.VegasQuant), ("vegas_rope", vb.VegasRope), ("vegas_new_tokens", vb.VegasNewTokens))) + "return 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.run([cc, "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for s in (vb.VegasQuant, vb.VegasRope, vb.VegasNewTokens):
        want += [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    assert got == want


# ------------------------------------------------------------------------------------------------------- frequencies

def test_frequencies_without_scaling_and_interpolated():
    for rot in (2, 16, 64, 128):
        f, m = vb.vegas_rope_frequencies(rot, 10000.0)
        want = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
        assert m == 1.0 and np.allclose(f, want, rtol=1e-14, atol=0)
        lin, m = vb.vegas_rope_frequencies(rot, 10000.0, vb.ROPE_SCALE_LINEAR, 8.0)
        assert m == 1.0 and np.allclose(lin, np.array(want) / 8.0, rtol=1e-14, atol=0)


def test_ntk_keeps_the_fastest_pair_and_interpolates_the_slowest():
    for rot, factor in ((64, 2.0), (128, 4.0)):
        plain, _ = vb.vegas_rope_frequencies(rot, 1e6)
        f, m = vb.vegas_rope_frequencies(rot, 1e6, vb.ROPE_SCALE_NTK, factor)
        assert m == 1.0 and f[0] == 1.0
        assert math.isclose(f[-1], plain[-1] / factor, rel_tol=1e-12)
        assert all(a > b for a, b in zip(f, f[1:]))
    assert vb.vegas_rope_frequencies(2, 1e6, vb.ROPE_SCALE_NTK, 4.0)[0] == [1.0]


def test_yarn_by_parts():
    """Pairs of more than 32 turns over the original length keep their frequency, of fewer than one are divided, between a blend of both
    whose weight grows with the pair; the magnitude is 0.1 ln(factor) + 1."""
    rot, base, factor, original = 128, 1e6, 4.0, 32768
    plain, _ = vb.vegas_rope_frequencies(rot, base)
    f, m = vb.vegas_rope_frequencies(rot, base, vb.ROPE_SCALE_YARN, factor, original)
    assert math.isclose(m, 0.1 * math.log(factor) + 1.0, rel_tol=1e-7)
    weight = []
    for i, (p, y) in enumerate(zip(plain, f)):
        turns = original * p / (2 * math.pi)
        blend = (p - y) / (p - p / factor)                   # 0: kept, 1: interpolated
        weight.append(blend)
        if turns > 32.0 * base ** (2.0 / rot):               # (the ramp starts at a whole pair)
            assert abs(blend) < 1e-12, i
        if turns < base ** (-2.0 / rot):
            assert abs(blend - 1) < 1e-9, i
        assert -1e-12 <= blend <= 1 + 1e-9
    assert all(b >= a - 1e-9 for a, b in zip(weight, weight[1:])) and 0.2 < weight[int(np.argmin(np.abs(np.array(weight) - 0.5)))] < 0.8
    same, m1 = vb.vegas_rope_frequencies(rot, base, vb.ROPE_SCALE_YARN, 1.0, original)
    assert np.allclose(same, plain, rtol=1e-14, atol=0) and m1 == 1.0


@pytest.mark.parametrize("args,status", [
    ((0, 1e4), vb.VEGAS_ERR_SHAPE), ((-2, 1e4), vb.VEGAS_ERR_SHAPE), ((7, 1e4), vb.VEGAS_ERR_SHAPE), ((64, 1.0), vb.VEGAS_ERR_SHAPE),
    ((64, math.nan), vb.VEGAS_ERR_SHAPE), ((64, math.inf), vb.VEGAS_ERR_SHAPE), ((64, 1e4, 4), vb.VEGAS_ERR_UNSUPPORTED),
    ((64, 1e4, -1), vb.VEGAS_ERR_UNSUPPORTED), ((64, 1e4, vb.ROPE_SCALE_LINEAR, 0.5), vb.VEGAS_ERR_SHAPE),
    ((64, 1e4, vb.ROPE_SCALE_NTK, math.inf), vb.VEGAS_ERR_SHAPE), ((64, 1e4, vb.ROPE_SCALE_YARN, 4.0, 0), vb.VEGAS_ERR_SHAPE),
    ((64, 1e4, vb.ROPE_SCALE_YARN, 4.0, 4096, 1.0, 1.0), vb.VEGAS_ERR_SHAPE), ((64, 1e4, vb.ROPE_SCALE_YARN, 4.0, 4096, 32.0, 0.0), vb.VEGAS_ERR_SHAPE),
])
def test_frequency_refusals(args, status):
    refused(lambda: vb.vegas_rope_frequencies(*args), status)


@pytest.mark.parametrize("num_queries", [1, 5])
def test_any_chunk_length_up_to_the_type_s_end(num_queries):
    """A chunk longer than the bound on the lengths is one chunk."""
    over = dict(num_queries=num_queries, max_blocks=64, max_sel_blocks=64, max_seq_len=1000)
    assert vb.vegas_quant_workspace_bytes(desc(kv_chunk_tokens=2 ** 31 - 32, **over)) == vb.vegas_quant_workspace_bytes(desc(kv_chunk_tokens=1024, **over)) > 0
