"""Whole runs over an 8-bit cache on the GPU: verify -> select -> G x (append and grow -> draft) through the harness, and a prompt that
comes in with rotary positions, is verified, selected from, drafted from and read back.  Every stage against the definition in 64 bits
over the codes that the cache holds; then as a captured graph, replayed between eager work, and on a stream of its own."""
import numpy as np
import pytest
import torch

from paper_2602_07223_amd import binding as vb
from paper_2602_07223_amd import harness, synth
from tests import quant_ref as Q

pytestmark = pytest.mark.gpu
PAGE = 16
DEV = "cuda:0"
CASES = [("b1", 1, 32, 8, 128, 5, [4103], 512), ("b3", 3, 10, 5, 128, 3, [1000, 16, 333], 160), ("b9", 9, 16, 2, 64, 5, [700, 5, 2049, 64, 31, 1500, 100, 16, 900], 256)]


def f64(t):
    return t.detach().cpu().float().numpy().astype(np.float64)


def values(dl):
    """Rows [page, slot, head, dim] that the cache's codes stand for."""
    scales = dl.quant.tensors[2].cpu().numpy().astype(np.float64)
    return [Q.code_values(c) * scales[:, :, w].transpose(0, 2, 1)[..., None] for w, c in enumerate((dl.k_cache, dl.v_cache))]


def check_rows(got, q, rows, n, G, scale):
    ref, spread, l1, _ = Q.attention(q, rows[0], rows[1], n, G, scale)
    assert (np.abs(got - ref) <= Q.out_tolerance(ref, spread, l1, q.shape[-1])).all()


def make(fmt, batch, hq, hkv, dim, G, lens, budget):
    L = synth.with_growth(synth.make_random_case(seed=900 + batch, batch=batch, num_q_heads=hq, num_kv_heads=hkv, num_queries=G, seq_lens=lens,
                                                 head_dim=dim), G)
    dl = harness.DeviceLayer.upload(L).quantised(fmt)
    path = harness.VegasPath.for_layer(L, budget_tokens=budget, growth=G, cache_format=fmt)
    return L, dl, path


def outputs(path, dl):
    return [t.clone() for t in (path.out_verify, path.block_scores, path.sel_table, path.sel_seq_lens, path.out_draft, dl.seq_lens_live, dl.k_cache.view(torch.uint8),
                                dl.v_cache.view(torch.uint8), dl.quant.tensors[2].nan_to_num(nan=-1.0))]


def same(a, b, valid_sel):
    for i, (x, y) in enumerate(zip(a, b)):
        if i == 2:                               # entries past a selection's end are whatever they were
            for row, n in enumerate(valid_sel):
                assert torch.equal(x[row, :n], y[row, :n])
        else:
            assert torch.equal(x, y), i


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("name,batch,hq,hkv,dim,G,lens,budget", CASES)
def test_live_iteration(fmt, name, batch, hq, hkv, dim, G, lens, budget):
    L, dl, path = make(fmt, batch, hq, hkv, dim, G, lens, budget)
    before = values(dl)
    path.live_iteration(dl)
    torch.cuda.synchronize()
    qv, qd, table = f64(dl.q_verify), f64(dl.q_draft), L.block_table
    scores = path.block_scores.cpu().numpy()
    sel, ssl = path.sel_table.cpu().numpy(), path.sel_seq_lens.cpu().numpy()
    after = values(dl)
    assert dl.seq_lens_live.cpu().tolist() == [n + G for n in lens]
    path.verify(dl)                              # the selection before it grew
    path.select(dl)
    torch.cuda.synchronize()
    first, first_len = path.sel_table.cpu().numpy(), path.sel_seq_lens.cpu().numpy()
    for b, n in enumerate(lens):
        pos = np.arange(n)
        slot = table[b, pos // PAGE] * PAGE + pos % PAGE
        check_rows(f64(path.out_verify[b]), qv[b], [x.reshape(-1, hkv, dim)[slot] for x in before], n, G, path.desc_verify.softmax_scale)
        # the selection holds the pages of the best scores (ties aside, there are none among random scores) and grows by the drafted tokens
        kept = -(-int(first_len[b]) // PAGE)
        assert set(first[b, :kept]) <= set(table[b, :-(-n // PAGE)])
        assert ssl[b] == first_len[b] + G
        assert np.array_equal(sel[b, :kept], first[b, :kept])
        for s in range(G):
            m = int(first_len[b]) + s + 1
            at = np.arange(m)
            slot = sel[b, at // PAGE] * PAGE + at % PAGE
            check_rows(f64(path.out_draft[s, b])[None], qd[s, b][None], [x.reshape(-1, hkv, dim)[slot] for x in after], m, 1, path.desc_draft.softmax_scale)
    assert (scores >= 0).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_selection_is_the_bf16_path_s_for_the_same_scores(fmt):
    name, batch, hq, hkv, dim, G, lens, budget = CASES[2]
    L, dl, path = make(fmt, batch, hq, hkv, dim, G, lens, budget)
    plain = harness.VegasPath.for_layer(L, budget_tokens=budget, growth=G)
    path.verify(dl)
    path.select(dl)
    plain.block_scores.copy_(path.block_scores)
    plain.select(harness.DeviceLayer.upload(L))
    torch.cuda.synchronize()
    n = path.sel_seq_lens.cpu().tolist()
    assert torch.equal(path.sel_seq_lens, plain.sel_seq_lens)
    for b in range(batch):
        assert torch.equal(path.sel_table[b, :-(-n[b] // PAGE)], plain.sel_table[b, :-(-n[b] // PAGE)])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("name,batch,hq,hkv,dim,G,lens,budget", CASES)
def test_live_iteration_captured_and_replayed(fmt, name, batch, hq, hkv, dim, G, lens, budget):
    L, dl, path = make(fmt, batch, hq, hkv, dim, G, lens, budget)
    path.live_iteration(dl)
    torch.cuda.synchronize()
    want = outputs(path, dl)
    valid = [-(-int(n) // PAGE) for n in path.sel_seq_lens.cpu()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        path.live_iteration(dl)                  # on a stream of its own
        s.synchronize()
        same(outputs(path, dl), want, valid)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            path.live_iteration(dl)
    other = make(fmt, batch, hq, hkv, dim, G, [max(n // 2, 1) for n in lens], budget)
    for _ in range(4):
        for t in (path.out_verify, path.block_scores, path.out_draft):
            t.fill_(7)
        path.workspace.fill_(0xff)
        other[2].live_iteration(other[1])        # eager work of another layer between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same(outputs(path, dl), want, valid)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hkv,dim,layout", [(16, 4, 128, vb.ROPE_HALF), (6, 3, 64, vb.ROPE_INTERLEAVED)])
def test_prompts_with_positions_verified_drafted_and_read_back(fmt, hq, hkv, dim, layout):
    """Padded prompts of three sequences (one empty) enter with rotated keys, their last G tokens are verified with rotated queries, pages are
    selected, G tokens are drafted whose keys and queries the append rotates, and what was kept is read back."""
    B, T, G, counts, g = 3, 333, 4, [333, 0, 150], torch.Generator().manual_seed(5)
    room = 30
    rnd = lambda *shape: torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)
    k, v, q = rnd(B, T, hkv, dim), rnd(B, T, hkv, dim), rnd(B, G, hq, dim)
    kn, vn, qn = rnd(G, B, 1, hkv, dim), rnd(G, B, 1, hkv, dim), rnd(G, B, 1, hq, dim)
    code, dtype = harness.CACHE_FORMATS[fmt]
    pages = B * room
    kc, vc = (torch.zeros((pages, PAGE, hkv, dim), dtype=dtype, device=DEV) for _ in range(2))
    scales = torch.zeros((pages, hkv, 2, PAGE), device=DEV)
    cache = vb.make_quant(kc, vc, scales, code)
    freq, magnitude = vb.vegas_rope_frequencies(dim)
    rope = vb.make_rope(torch.tensor(freq, dtype=torch.float64, device=DEV), dim, layout, magnitude)
    table = torch.randperm(pages, generator=g).to(torch.int32).view(B, room).to(DEV)
    width = 12
    desc = vb.make_desc(batch=B, num_q_heads=hq, num_kv_heads=hkv, num_queries=G, max_blocks=room, max_sel_blocks=width, max_seq_len=room * PAGE,
                        num_pages=pages, softmax_scale=dim ** -0.5, head_dim=dim, collect_rows=vb.COLLECT_ALL_ROWS)
    drafts = vb.make_desc(batch=B, num_q_heads=hq, num_kv_heads=hkv, num_queries=G, max_blocks=room, max_sel_blocks=width, max_seq_len=width * PAGE,
                          num_pages=pages, softmax_scale=dim ** -0.5, head_dim=dim)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    start, lens = i32([0] * B), i32([-9] * B)
    q_rot, qn_rot = torch.empty_like(q), torch.empty_like(qn)
    positions = i32([[max(n - G, 0) + t for t in range(G)] for n in counts])
    out, scores = torch.empty_like(q), torch.empty((B, room), device=DEV)
    out_draft = torch.empty((G, B, hq, dim), dtype=torch.bfloat16, device=DEV)
    sel, sel_lens = torch.zeros((B, width), dtype=torch.int32, device=DEV), i32([0] * B)
    k_back, v_back = (torch.full((B, width * PAGE, hkv, dim), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = torch.empty(max(vb.vegas_quant_workspace_bytes(desc), vb.vegas_quant_workspace_bytes(drafts)), dtype=torch.uint8, device=DEV)
    prompt = vb.make_new_tokens(k, v, T, new_lens=i32(counts))
    steps = [vb.make_new_tokens(kn[s], vn[s], 1, q=qn[s], q_out=qn_rot[s]) for s in range(G)]

    def run(stream):
        vb.vegas_append_quant(desc, cache, rope, prompt, table, start, lens, stream=stream)
        vb.vegas_rotate(rope, dim, B * G, hq, positions, q, q_rot, stream=stream)
        vb.vegas_verify_attention_quant(desc, cache, q_rot, table, lens, out, scores, ws, stream=stream)
        vb.vegas_select_blocks(desc, scores, table, lens, 100, sel, sel_lens, stream=stream)
        for s in range(G):
            vb.vegas_append_quant(desc, cache, rope, steps[s], table, lens, lens, sel, sel_lens, PAGE, stream=stream)
            vb.vegas_draft_attention_quant(drafts, cache, qn_rot[s], sel, sel_lens, out_draft[s], ws, stream=stream)
        vb.vegas_read_quant(drafts, cache, sel, sel_lens, None, width * PAGE, k_back, v_back, stream=stream)

    run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert lens.cpu().tolist() == [n + G for n in counts]
    held = [Q.code_values(c) * scales.cpu().numpy().astype(np.float64)[:, :, w].transpose(0, 2, 1)[..., None] for w, c in enumerate((kc, vc))]
    held = [x.reshape(-1, hkv, dim) for x in held]
    name = "half" if layout == vb.ROPE_HALF else "interleaved"
    # half a step of a code is 2^-4 of the value and at least 2^-10 scales (e4m3), half a scale (int8); the scale is at most max|x| / top
    half = lambda x: np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * np.abs(x).max(-1, keepdims=True) / 448) if fmt == "e4m3" else 0.5 * np.abs(x).max(-1, keepdims=True) / 127
    for b, n in enumerate(counts):
        at = np.arange(n + G)
        slot = table[b].cpu().numpy()[at // PAGE] * PAGE + at % PAGE
        keys = np.concatenate([f64(k[b, :n]), f64(kn[:, b, 0])])
        keys = Q.rotated(keys, at, freq, magnitude, name)
        vals = np.concatenate([f64(v[b, :n]), f64(vn[:, b, 0])])
        for w, x in enumerate((keys, vals)):
            assert (np.abs(held[w][slot] - x) <= half(x) * (1 + 1e-5) + 4e-6 * np.abs(x).max()).all()      # (fp32 rotation, reciprocal, products)
        turned = Q.rotated(f64(q[b]), positions[b].cpu().numpy(), freq, magnitude, name)
        assert (np.abs(f64(q_rot[b]) - turned) <= 2.0 ** -8 * np.abs(turned) + 4e-6 * np.abs(turned).max()).all()
        if n:
            check_rows(f64(out[b]), f64(q_rot[b]), [x[slot[:n]] for x in held], n, G, dim ** -0.5)
        else:
            assert (out[b] == 0).all()
        m = int(sel_lens[b])
        if n == 0:                               # (an empty selection does not grow: vegas_extend_selection)
            assert m == 0 and (out_draft[:, b] == 0).all() and (k_back[b] == 5.0).all()
            continue
        assert m >= G
        at = np.arange(m)
        chosen = sel[b].cpu().numpy()[at // PAGE] * PAGE + at % PAGE
        for s in range(G):
            now = m - G + s + 1
            turned = Q.rotated(f64(qn[s, b]), [n + s], freq, magnitude, name)
            assert (np.abs(f64(qn_rot[s, b]) - turned) <= 2.0 ** -8 * np.abs(turned) + 4e-6 * np.abs(turned).max()).all()
            check_rows(f64(out_draft[s, b])[None], f64(qn_rot[s, b]), [x[chosen[:now]] for x in held], now, 1, dim ** -0.5)
        for back, x in ((k_back, held[0]), (v_back, held[1])):
            assert (np.abs(f64(back[b, :m]) - x[chosen]) <= 2.0 ** -8 * np.abs(x[chosen]) * (1 + 1e-6)).all()
            assert (back[b, m:] == 5.0).all()
    # captured, replayed between eager work: the same bits
    results = (out, scores, out_draft, k_back, v_back, lens, sel_lens, qn_rot)
    want = [t.clone() for t in results]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(s.cuda_stream)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run(s.cuda_stream)
    for _ in range(4):
        for t in (out, scores, out_draft, qn_rot):
            t.fill_(3)
        ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(results, want):
            assert torch.equal(x, y)


def test_refusals_of_the_harness():
    L = synth.make_random_case(seed=3, batch=1, num_q_heads=4, num_kv_heads=2, num_queries=2, seq_lens=[40])
    dl = harness.DeviceLayer.upload(L)
    path = harness.VegasPath.for_layer(L, budget_tokens=32, cache_format="int8")
    with pytest.raises(ValueError):
        path.verify(dl)                          # a bf16 layer
    with pytest.raises(ValueError):
        harness.VegasPath.for_layer(L, budget_tokens=32).verify(dl.quantised("int8"))
    with pytest.raises(ValueError):
        harness.VegasPath.for_layer(L, budget_tokens=32, cache_format="int8", token_granular=True)
    with pytest.raises(ValueError):
        harness.VegasPath.for_layer(L, budget_tokens=32, cache_format="fp4")
    with pytest.raises(ValueError):
        path.verify(dl.quantised("int8"), stages=1)
