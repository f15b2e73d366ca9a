"""The 8-bit cache's kernels in every form their launch rules choose, each asserted to be the one meant, and calls as a program makes
them: some of a batch's runs, prefixes that sequences share, two streams at once, the way back in a graph.  Bounds are those of
test_gpu_kv8.py."""
import numpy as np
import pytest
import torch

import paper_2402_18789_amd.binding as B
from paper_2402_18789_amd import host as HH
from paper_2402_18789_amd import kv8
from gpu_common import to_np
from kv8_plan import kv8_plan, pieces
from oracle import kv8 as O8
from test_gpu_kv8 import D, F, P, attention_case, check_attention, device, fill_prefixes, from_device, make_batch, shape, to_device
from workload import gen
from workload.configs import Request

pytestmark = pytest.mark.gpu


def plan_of(cfg, reqs_in, split=0):
    reqs, pages, num_pages = make_batch(cfg, reqs_in)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages, split, device=None)
    return kv8_plan(db.host_maps, cfg.n_kv_heads), db.host_maps


# ---- forms of the attention ---------------------------------------------------------------------------------

@pytest.mark.parametrize("cfg,reqs", [(shape(40, 8), [(P, 0, 189)]), (shape(40, 8), [(P, 0, 256)]), (shape(8, 2), [(F, 150, 100)]),
                                      (shape(40, 8), [(P, 100, 30), (D, 20, 1), (D, 200, 1), (P, 0, 2)]), (shape(16, 1), [(P, 0, 250), (D, 255, 1)])])
def test_chunks_in_one_piece(cfg, reqs):
    plan, m = plan_of(cfg, reqs)
    assert plan.whole and m.n_parts > m.n_tiles
    check_attention(cfg, reqs)


@pytest.mark.parametrize("n", [135, 300])
def test_single_tokens_on_two_wavefronts(n):
    cfg = shape(8, 8)
    reqs = [(D, int(v), 1) for v in gen.rng(n, "kv8", "short").integers(0, 90, n)]
    plan, m = plan_of(cfg, reqs)
    assert plan.wavefronts == 2 and m.n_single == m.n_items
    check_attention(cfg, reqs)


@pytest.mark.parametrize("cfg,reqs,least,most", [(shape(8, 2), [(D, 1999, 1)], 2, 8), (shape(8, 2), [(D, 3500, 1)], 9, 16), (shape(8, 8), [(D, 20000, 1)], 17, 1000),
                                                 (shape(32, 8), [(D, 20000, 1), (D, 0, 1), (D, 64, 1), (D, 9000, 1)], 17, 1000),
                                                 (shape(16, 1), [(D, 12345, 1)] * 3, 17, 1000)])
def test_single_tokens_in_pieces(cfg, reqs, least, most):
    plan, m = plan_of(cfg, reqs)
    assert plan.wavefronts == 4 and least <= pieces(m, plan) <= most
    check_attention(cfg, reqs)


@pytest.mark.parametrize("cfg", [shape(8, 2), shape(40, 8)], ids=lambda c: c.name)
def test_pieces_beside_chunks(cfg):
    reqs = [(D, 3000, 1), (P, 900, 70), (D, 1, 1), (D, 1500, 1), (F, 300, 41)]
    plan, m = plan_of(cfg, reqs)
    assert plan.fold > 1 and not plan.whole and 0 < m.n_single < m.n_items
    check_attention(cfg, reqs, rows_of=(0, 1, 31))


@pytest.mark.parametrize("cfg", [shape(4, 2, 64, "f32"), shape(6, 3, 48), shape(16, 2, 256), shape(2, 1, 16, "f32"), shape(34, 2), shape(4, 2, 128, "bf16", 5)],
                         ids=lambda c: c.name)
def test_many_pieces_of_other_shapes(cfg):
    reqs = [(D, 5000, 1), (D, 3, 1), (P, 2100, 20)]
    _, m = plan_of(cfg, reqs)
    assert -(-m.max_pages // m.kv_split_pages) > 16
    check_attention(cfg, reqs, rows_of=(0, 7))
    check_attention(cfg, reqs, rows_of=(0, 7), split=16, use_lse=False)


# Scores that grow from page to page (every step moves the reference of the exponentials), shrink, or jump both ways.
@pytest.mark.parametrize("law", [lambda j: j, lambda j: -j, lambda j: (j * 7) % 11, lambda j: 8 * (j % 5 == 4)])
@pytest.mark.parametrize("cfg", [shape(8, 2), shape(4, 2, 64, "f32")], ids=lambda c: c.name)
def test_scores_that_move(cfg, law):
    def edit(cache, reqs, pages):
        for i in range(len(reqs)):
            for j, page in enumerate(pages[i]):
                cache.scale["k"][page] *= 2.0 ** (0.5 * law(j) // 1)
    check_attention(cfg, [(D, 300, 1), (P, 200, 90), (D, 20, 1), (F, 0, 150)], edit=edit)


def test_one_piece_or_many_the_same_rows():
    """cut by hand into pieces of every size: the same rows but for the order of the sums"""
    cfg = shape(32, 8)
    reqs = [(D, 4000, 1), (D, 77, 1), (P, 500, 60)]
    runs = [attention_case(cfg, reqs, split=s) for s in (2, 8, 64, 256)]
    for r in runs[1:]:
        assert np.max(np.abs(r[5] - runs[0][5])) <= 2 * 2.0 ** -8 * np.max(np.abs(runs[0][5]))
        assert np.max(np.abs(r[6] - runs[0][6])) <= 1e-4


# ---- calls --------------------------------------------------------------------------------------------------

def test_some_of_a_batchs_runs():
    """a call over some of the runs writes their pages, scales and queries and no other"""
    cfg = shape(8, 2)
    reqs, pages, num_pages = make_batch(cfg, [(D, 33, 1), (P, 5, 50), (D, 16, 1), (F, 20, 30)])
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    c, T = HH.c_cfg(cfg), db.host_maps.T
    x = device(gen.rng(0, "kv8", "x").standard_normal((T, cfg.qkv_dim)), cfg)

    def run(groups):
        pool, out = kv8.DevicePool8(cfg, num_pages), torch.full((T, cfg.q_dim), 7.0, dtype=x.dtype, device="cuda")
        for g in groups:
            r = torch.from_numpy(db.host_runs[g]).cuda()
            kv8.flexco_kv8_append(c, db.maps, r, len(r), x, pool.c, out, cfg.q_dim)
        torch.cuda.synchronize()
        return pool, out

    n = db.n_runs
    assert n > 6
    full, q = run([list(range(n))])
    parts, q2 = run([[1, 4], [n - 1], [0, 2, 3] + list(range(5, n - 1))])
    for a, b in ((full.k, parts.k), (full.v, parts.v), (full.k_scale, parts.k_scale), (full.v_scale, parts.v_scale), (q, q2)):
        assert torch.equal(a, b)
    some, q3 = run([[0, 2, 5]])
    rows = np.concatenate([np.arange(t, t + k) for t, k in db.host_runs[[0, 2, 5]]])
    rest = np.setdiff1d(np.arange(T), rows)
    assert torch.equal(q3[rows], q[rows]) and (q3[rest] == 7.0).all()
    slot = db.numpy()["slot"]
    hit = np.unique(slot[rows] // cfg.page_size)
    others = np.setdiff1d(np.arange(num_pages), hit)
    assert torch.equal(some.k[hit], full.k[hit]) and torch.equal(some.v_scale[hit], full.v_scale[hit])
    assert not some.k[others].any() and not some.v[others].any() and not some.k_scale[others].any()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cfg", [shape(40, 8), shape(4, 4, 64, "f32")], ids=lambda c: c.name)
def test_single_tokens_in_any_order_of_runs(cfg, in_place):
    """as many runs as tokens, in the batch's order and in others: the same pages, scales and queries"""
    n = 37
    reqs, pages, num_pages = make_batch(cfg, [(D, int(v), 1) for v in gen.rng(4, "kv8", "pos").integers(0, 90, n)])
    cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, reqs, pages, 0)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    assert db.n_runs == db.host_maps.T == n
    c, got = HH.c_cfg(cfg), []
    x = device(gen.rng(0, "kv8", "x").standard_normal((n, cfg.qkv_dim)), cfg)
    for order in (np.arange(n), np.arange(n)[::-1], gen.rng(5, "kv8", "order").permutation(n)):
        pool, rows = to_device(cfg, cache, num_pages), x.clone()
        q, ld = (rows, cfg.qkv_dim) if in_place else (torch.zeros((n, cfg.q_dim), dtype=x.dtype, device="cuda"), cfg.q_dim)
        runs = torch.from_numpy(np.ascontiguousarray(db.host_runs[order])).cuda()
        kv8.flexco_kv8_append(c, db.maps, runs, n, rows, pool.c, q, ld)
        torch.cuda.synchronize()
        got.append((q, pool.k, pool.v, pool.k_scale, pool.v_scale))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("cfg", [shape(8, 2), shape(4, 2, 64, "f32")], ids=lambda c: c.name)
def test_sequences_that_share_their_prefix(cfg):
    """three sequences whose first pages are the same ones, each with a page of its own behind: the rows of copies in pages of their own"""
    shared, own = [5, 1, 7], [0, 3, 2]
    reqs = [Request(kind=D, seq_id=i, start_pos=48 + i, n_new=1, adapter=-1) for i in range(3)]
    pages = {i: np.array(shared + [own[i]], dtype=np.int32) for i in range(3)}
    apart = {i: np.array([8 + 4 * i + j for j in range(4)], dtype=np.int32) for i in range(3)}
    cache = O8.Cache8(20, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    g = gen.rng(2, "kv8", "shared")
    cache.append(pages[0], 0, *g.standard_normal((2, 48, cfg.kv_dim)))
    for i in range(3):
        cache.append(pages[i], 48, *g.standard_normal((2, 1 + i, cfg.kv_dim)))
        for n in "kv":
            cache.codes[n][apart[i]] = cache.codes[n][pages[i]]
            cache.scale[n][apart[i]] = cache.scale[n][pages[i]]
    pool = to_device(cfg, cache, 20)
    c, outs = HH.c_cfg(cfg), []
    x = device(g.standard_normal((3, cfg.qkv_dim)), cfg)
    for p in (pages, apart):
        db = kv8.DeviceBatch8(cfg, reqs, p, 20)
        q, out = (torch.empty((3, cfg.q_dim), dtype=x.dtype, device="cuda") for _ in range(2))
        ws = HH.Workspace(c, 3, db.host_maps.n_parts)
        kv8.flexco_kv8_append(c, db.maps, db.runs, db.n_runs, x, pool.c, q, cfg.q_dim)
        kv8.flexco_kv8_attention(c, db.maps, q, pool.c, out, None, ws.ptr, ws.bytes)
        outs.append(to_np(out))
    assert np.array_equal(outs[0], outs[1]) and np.isfinite(outs[0]).all()
    with pytest.raises(B.FlexcoError) as e:                         # two tokens into the one shared page: its scale would be chosen twice
        kv8.DeviceBatch8(cfg, [Request(kind=D, seq_id=0, start_pos=40, n_new=1, adapter=-1),
                               Request(kind=D, seq_id=1, start_pos=41, n_new=1, adapter=-1)], pages, 20)
    assert e.value.code == B.FLEXCO_EPAGE


def test_two_streams_at_once():
    """two caches, workspaces and streams, many calls on each without waiting for the other"""
    cfg = shape(40, 8)
    c, jobs = HH.c_cfg(cfg), []
    for i, reqs_in in enumerate(([(D, 1500, 1), (D, 40, 1), (P, 300, 90)], [(D, 5000, 1), (F, 41, 70), (D, 3, 1)])):
        reqs, pages, num_pages = make_batch(cfg, reqs_in, seed=i)
        cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
        fill_prefixes(cfg, cache, reqs, pages, i)
        db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
        T = db.host_maps.T
        x = device(gen.rng(i, "kv8", "x").standard_normal((T, cfg.qkv_dim)), cfg)
        jobs.append(dict(db=db, pool=to_device(cfg, cache, num_pages), x=x, ws=HH.Workspace(c, T, db.host_maps.n_parts), stream=torch.cuda.Stream(),
                         q=torch.empty((T, cfg.q_dim), dtype=x.dtype, device="cuda"), wide=HH.DevicePool(cfg, num_pages),
                         seq=torch.from_numpy(pages[0]).cuda(), n=reqs[0].start_pos + 1,
                         out=[torch.zeros((T, cfg.q_dim), dtype=x.dtype, device="cuda") for _ in range(8)]))

    def step(j, out, stream):
        kv8.flexco_kv8_append(c, j["db"].maps, j["db"].runs, j["db"].n_runs, j["x"], j["pool"].c, j["q"], cfg.q_dim, stream)
        kv8.flexco_kv8_attention(c, j["db"].maps, j["q"], j["pool"].c, out, None, j["ws"].ptr, j["ws"].bytes, stream)
        j["pool"].expand(j["seq"], j["n"], j["wide"], j["seq"], stream)

    want = []
    for j in jobs:
        step(j, j["out"][0], None)                                  # (the first append may raise a scale; from then on all are alike)
        step(j, j["out"][0], None)
        torch.cuda.synchronize()
        want.append((j["out"][0].clone(), j["pool"].v.clone(), j["wide"].k.clone()))
    for i in range(8):
        for j in jobs:
            step(j, j["out"][i], j["stream"].cuda_stream)
    torch.cuda.synchronize()
    for j, (out, v, k) in zip(jobs, want):
        assert all(torch.equal(o, out) for o in j["out"]) and torch.equal(j["pool"].v, v) and torch.equal(j["wide"].k, k)


def test_a_windows_way_back_in_a_graph():
    """append, attention, the pages written out and attention's gradients captured as one graph, replayed with eager calls between"""
    cfg, start, n = shape(8, 2), 37, 50
    reqs, pages, num_pages = make_batch(cfg, [(F, start, n)])
    cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, reqs, pages, 0, 0.3)
    pool, db, c = to_device(cfg, cache, num_pages), kv8.DeviceBatch8(cfg, reqs, pages, num_pages), HH.c_cfg(cfg)
    x = device(gen.rng(1, "kv8", "qkv").standard_normal((n, cfg.qkv_dim)), cfg)
    dout = device(gen.rng(2, "kv8", "dout").standard_normal((n, cfg.q_dim)), cfg)
    ws = HH.Workspace(c, n, db.host_maps.n_parts, n, start + n)
    q, out, dq = (torch.empty((n, cfg.q_dim), dtype=x.dtype, device="cuda") for _ in range(3))
    lse = torch.empty((n, cfg.n_q_heads), device="cuda")
    dk, dv = (torch.zeros((start + n, cfg.kv_dim), device="cuda") for _ in range(2))
    wide, src = HH.DevicePool(cfg, len(pages[0])), torch.from_numpy(pages[0]).cuda()
    dst = torch.arange(len(pages[0]), dtype=torch.int32, device="cuda")

    def step():
        dk.zero_()
        dv.zero_()
        kv8.flexco_kv8_append(c, db.maps, db.runs, db.n_runs, x, pool.c, q, cfg.q_dim)
        kv8.flexco_kv8_attention(c, db.maps, q, pool.c, out, lse, ws.ptr, ws.bytes)
        pool.expand(src, start + n, wide, dst)
        B.flexco_attention_window_bwd(c, wide.c, dst, len(dst), start, n, q, out, lse, dout, dq, dk, dv, ws.ptr, ws.bytes)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (out, lse, dq, dk, dv)]

    def close(a, b):
        return all(torch.allclose(u.float(), v.float(), rtol=1e-5, atol=1e-5 * float(v.float().abs().max())) for u, v in zip(a, b))

    step()
    step()
    eager = results()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t in (out, lse, dq, dk, dv):
            t.fill_(5.0)
        graph.replay()
        assert close(results(), eager), i
        if i == 1:
            step()
            assert close(results(), eager)


def test_a_page_is_read_for_two():
    """the same page of the cache at two places of a sequence that is written out"""
    cfg = shape(4, 2)
    pool = kv8.DevicePool8(cfg, 3)
    pool.k.copy_(torch.arange(pool.k.numel(), device="cuda").view_as(pool.k) % 120)
    pool.v.copy_(torch.arange(pool.v.numel(), device="cuda").view_as(pool.v) % 113)
    pool.k_scale.fill_(0.5)
    pool.v_scale.fill_(2.0)
    wide = HH.DevicePool(cfg, 4)
    pool.expand(torch.tensor([2, 2, 1], dtype=torch.int32, device="cuda"), 48, wide, torch.tensor([0, 3, 1], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(wide.k[0], wide.k[3]) and torch.equal(wide.v[0], wide.v[3]) and not wide.k[2].any()
    codes, scale = from_device(pool)
    assert np.array_equal(to_np(wide.v[1]), (O8.decode(codes["v"][1]) * 2.0).transpose(1, 2, 0))


def test_append_and_pages_written_out_past_4_gib():
    """pages whose codes, and whose elements in the wide pool, lie beyond 2^32 bytes: what pages at the front get"""
    cfg = shape(32, 16)
    first, wide_first = (1 << 32) // (16 * 16 * 128), (1 << 32) // (16 * 16 * 128 * 2)
    reqs, pages, n = make_batch(cfg, [(D, 33, 1), (P, 5, 50), (D, 16, 1)])
    x = device(gen.rng(0, "kv8", "x").standard_normal((52, cfg.qkv_dim)), cfg)
    c, got = HH.c_cfg(cfg), []
    for at, wide_at in ((0, 0), (first, wide_first)):
        pool, wide = kv8.DevicePool8(cfg, at + n), HH.DevicePool(cfg, wide_at + 4)
        db = kv8.DeviceBatch8(cfg, reqs, {i: p + np.int32(at) for i, p in pages.items()}, at + n)
        q = torch.empty((52, cfg.q_dim), dtype=x.dtype, device="cuda")
        kv8.flexco_kv8_append(c, db.maps, db.runs, db.n_runs, x, pool.c, q, cfg.q_dim)
        src = torch.from_numpy(pages[1] + np.int32(at)).cuda()
        pool.expand(src, 55, wide, torch.arange(wide_at, wide_at + 4, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        got.append([t.clone() for t in (q, pool.k[at:], pool.v[at:], pool.k_scale[at:], pool.v_scale[at:], wide.k[wide_at:], wide.v[wide_at:])])
        assert not pool.k[:at].any() and not wide.v[:wide_at].any()
        del pool, wide
    assert all(torch.equal(a, b) for a, b in zip(*got))
