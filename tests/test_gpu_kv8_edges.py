"""The 8-bit cache where its rules meet each other.  Bounds are those of test_gpu_kv8.py unless a test says otherwise."""
import numpy as np
import pytest
import torch

from gpu_common import to_np
from kv8_plan import kv8_plan, pieces
from oracle import kv8 as O8
from oracle import layer as OL
from oracle.maps import build_maps
from paper_2402_18789_amd import host as HH
from paper_2402_18789_amd import kv8
from test_gpu_kv8 import C1, C2, D, F, P, check_append, check_attention, device, fill_prefixes, from_device, half_step, make_batch, say, shape, to_device
from workload import gen
from workload.configs import KIND_FINETUNE

pytestmark = pytest.mark.gpu


# ---- NaN keys in a piece of their own -----------------------------------------------------------------------

# Bf16 of head_dim 128: a request of one token of 1025 or 4097 keys is cut into pieces of 16 pages (asserted below), the last of them one
# key.  Other shapes and chunks: pieces of `split` pages.  In each case the requests' keys in `odd` are NaN, in one channel of the last kv head.
BF16, F32, F32W = shape(8, 2), shape(4, 2, 64, "f32"), shape(4, 2, 128, "f32")
CUT = [
    # the last key of a single token, the first of a chunk's last piece, a chunk's piece in the middle: merged a group of lanes per row
    (BF16, 2, [(D, 1024, 1), (P, 96, 20), (F, 64, 70), (D, 40, 1)], {0: [(1024, 1025)], 1: [(96, 97)], 2: [(32, 64)]}, 5),
    (BF16, 0, [(D, 1024, 1)], {0: [(1024, 1025)]}, 5),
    (BF16, 0, [(D, 1024, 1), (D, 900, 1)], {0: [(256, 512)], 1: [(0, 256)]}, 5),
    (BF16, 8, [(P, 512, 40), (P, 0, 300)], {0: [(512, 513)], 1: [(128, 256)]}, None),
    # by a block per row
    (BF16, 2, [(D, 4096, 1)], {0: [(4096, 4097)]}, 17),
    (BF16, 2, [(D, 4096, 1), (P, 96, 20)], {0: [(1024, 1280)], 1: [(64, 96)]}, 17),
    # other shapes: a wavefront per row, a group of lanes, a block
    (F32, 2, [(D, 64, 1), (P, 96, 20), (F, 64, 70)], {0: [(64, 65)], 1: [(96, 97)], 2: [(32, 64)]}, None),
    (F32, 8, [(D, 384, 1), (P, 0, 200)], {0: [(128, 256)], 1: [(128, 129)]}, None),
    (F32W, 2, [(D, 64, 1), (P, 96, 20)], {0: [(64, 65)], 1: [(32, 64)]}, None),
    (F32, 2, [(D, 1024, 1), (P, 96, 20)], {0: [(1024, 1025)], 1: [(96, 97)]}, None),
    (shape(34, 2), 2, [(D, 1024, 1), (P, 96, 20)], {0: [(512, 544)], 1: [(96, 97)]}, None),
]


@pytest.mark.parametrize("cfg,split,reqs,odd,n_pieces", CUT, ids=lambda v: getattr(v, "name", None))
def test_nan_keys_alone_in_a_piece_show(cfg, split, reqs, odd, n_pieces):
    """a row that sees a NaN key is NaN and so is its log-sum-exp, however its context is cut; other heads and rows are what they are"""
    batch, pages, num_pages = make_batch(cfg, reqs)
    m = kv8.DeviceBatch8(cfg, batch, pages, num_pages, split, device=None).host_maps
    if n_pieces:
        assert pieces(m, kv8_plan(m, cfg.n_kv_heads)) == n_pieces
    else:
        assert m.n_parts > m.n_tiles

    def edit(cache, requests, pages_of):
        for i, ranges in odd.items():
            for lo, hi in ranges:
                for at in range(lo, hi):
                    cache.codes["k"][pages_of[i][at // 16], at % 16, cfg.n_kv_heads - 1, 5] = 0x7F

    check_attention(cfg, reqs, split=split, edit=edit, rows_of=(0, 1, 30, 69, 127, 128, 255, 256))


# ---- runs ---------------------------------------------------------------------------------------------------

def appended(cfg, db, num_pages, cache, x, runs):
    pool, q = to_device(cfg, cache, num_pages), torch.full((db.host_maps.T, cfg.q_dim), 7.0, dtype=x.dtype, device="cuda")
    runs = torch.from_numpy(np.ascontiguousarray(runs, dtype=np.int32)).cuda()
    kv8.flexco_kv8_append(HH.c_cfg(cfg), db.maps, runs, len(runs), x, pool.c, q, cfg.q_dim)
    torch.cuda.synchronize()
    return q, pool.k, pool.v, pool.k_scale, pool.v_scale


@pytest.mark.parametrize("cfg", [shape(), shape(40, 8), shape(4, 4, 64, "f32"), shape(6, 3, 48), shape(4, 2, 128, "bf16", 5)], ids=lambda c: c.name)
@pytest.mark.parametrize("reqs_in", [[(D, 33, 1), (P, 5, 50)], [(F, 9, 70)], [(D, 33, 1), (P, 0, 2)], [(D, 7, 1), (D, 16, 1), (D, 0, 1)]], ids=str)
def test_runs_with_places_left_free(cfg, reqs_in):
    """a list as long as the batch, its places behind the runs (or between them) filled with runs outside the batch: what the runs alone give"""
    reqs, pages, num_pages = make_batch(cfg, reqs_in)
    cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, reqs, pages, 0)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    T = db.host_maps.T
    x = device(gen.rng(0, "kv8", "x").standard_normal((T, cfg.qkv_dim)), cfg)
    some = db.host_runs if db.n_runs < T else db.host_runs[:-1]
    want = appended(cfg, db, num_pages, cache, x, some)
    free = np.tile(np.array([[-1, 0]], dtype=np.int32), (T - len(some), 1))
    behind = np.concatenate((some, free))
    say("append", cfg.name, reqs_in, "%d runs in %d places" % (len(some), T))
    for runs in (behind, behind[gen.rng(1, "kv8", "places").permutation(T)]):
        assert all(torch.equal(a, b) for a, b in zip(appended(cfg, db, num_pages, cache, x, runs), want))


# ---- many kv heads -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("cfg", [shape(64, 64, 256), shape(64, 64, 256, "f32")], ids=lambda c: c.name)
def test_append_of_many_kv_heads(cfg):
    check_append(cfg, [(D, 33, 1), (P, 5, 20)])


# ---- the top of the number range ----------------------------------------------------------------------------

TOP = [1.0, 1.74, 1.75, 1.76, 1.87, 1.875, 1.9, 1.9374, 1.9376, 1.97, 1.9921875]     # times 2^127


@pytest.mark.parametrize("cfg", [shape(), shape(4, 2, 64, "f32"), shape(16, 16, 256), shape(3, 3, 48, "f32"), shape(4, 2, 128, "f32", 5)], ids=lambda c: c.name)
@pytest.mark.parametrize("reqs_in", [[(D, 0, 1), (D, 33, 1)], [(P, 0, 33), (D, 0, 1), (D, 5, 1)]], ids=str)
def test_the_largest_numbers_stay_finite(cfg, reqs_in):
    """Finite rows of up to 1.99 x 2^127 read back as finite numbers off by at most 2^-4 of themselves (half a step of the code, and 1.875 x 2^127,
    that nothing is stored beyond, is 0.0588 below 1.9922 x 2^127), or, of elements below 2^-6 of the scale, half the smallest code: 2^-10 of it."""
    reqs, pages, num_pages = make_batch(cfg, reqs_in)
    cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, reqs, pages, 0)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    T, qd, kd, half = db.host_maps.T, cfg.q_dim, cfg.kv_dim, cfg.head_dim // 2
    g = gen.rng(0, "kv8", "top")
    x = np.zeros((T, cfg.qkv_dim))
    big = lambda n: g.choice(TOP, (T, n)) * 2.0 ** 127 * g.choice([-1, 1], (T, n))  # noqa: E731
    # (of a pair of a key's channels one is zero: what the rotation makes of the other is no larger than it)
    x[:, qd:qd + kd].reshape(T, cfg.n_kv_heads, 2, half)[:, :, 0] = big(kd // 2).reshape(T, cfg.n_kv_heads, half)
    x[:, qd + kd:] = big(kd)
    x = gen.storage_round(cfg, x.astype(np.float32)).astype(np.float64)
    assert np.isfinite(x).all()
    xd = device(x, cfg)
    pool, c = to_device(cfg, cache, num_pages), HH.c_cfg(cfg)
    q = torch.zeros((T, qd), dtype=xd.dtype, device="cuda")
    say("append", cfg.name, reqs_in, "at the top of the range")
    kv8.flexco_kv8_append(c, db.maps, db.runs, db.n_runs, xd, pool.c, q, qd)
    codes, scale = from_device(pool)
    pos = np.concatenate([np.arange(r.start_pos, r.start_pos + r.n_new) for r in reqs])
    from oracle import ops
    rows = {"k": ops.rope(x[:, qd:qd + kd], pos, cfg.n_kv_heads, cfg.head_dim, cfg.rope_theta), "v": x[:, qd + kd:]}
    t0 = 0
    for r in reqs:
        end = r.start_pos + r.n_new
        wide = HH.DevicePool(cfg, len(pages[r.seq_id]))
        seq = torch.arange(len(pages[r.seq_id]), dtype=torch.int32, device="cuda")
        pool.expand(torch.from_numpy(pages[r.seq_id]).cuda(), end, wide, seq)
        got = {"k": to_np(wide.k).transpose(0, 2, 1, 3).reshape(-1, kd)[r.start_pos:end],
               "v": to_np(wide.v).transpose(0, 3, 1, 2).reshape(-1, kd)[r.start_pos:end]}
        for name in "kv":
            want = rows[name][t0:t0 + r.n_new]
            s = np.repeat(scale[name][pages[r.seq_id][np.arange(r.start_pos, end) // cfg.page_size]], cfg.head_dim, 1)
            assert s.max() <= 2.0 ** 120 and np.isfinite(got[name]).all(), name
            # (1e-6: the angles' part, as in check_append)
            assert np.all(np.abs(got[name] - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s) + 1e-6 * 2.0 ** 128), name
        t0 += r.n_new
    # a token alone, with equal scores for all of its one key: its value as it is cached
    alone = [t for t, r in zip(np.cumsum([0] + [r.n_new for r in reqs]), reqs) if r.start_pos == 0 and r.n_new == 1]
    ws = HH.Workspace(c, T, db.host_maps.n_parts)
    out = torch.empty_like(q)
    kv8.flexco_kv8_attention(c, db.maps, q, pool.c, out, None, ws.ptr, ws.bytes)
    i = [r for r in reqs if r.start_pos == 0 and r.n_new == 1][0].seq_id
    cached = O8.decode(codes["v"][pages[i][0], 0]) * scale["v"][pages[i][0]][:, None]
    want = np.repeat(cached, cfg.n_q_heads // cfg.n_kv_heads, 0).reshape(-1)
    assert np.all(np.abs(to_np(out)[alone[0]] - want) <= 2.0 ** -22 * np.abs(want))


# ---- the layer ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("single", [False, True], ids=["mixed", "decode"])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_rows_that_the_layer_caches(name, single):
    """every key and value element that flexco_kv8_layer_forward caches, against the definition in 64 bits: within half a code's step, the
    rotation's error and that of the storage type and the sums, element by element (a quiet head has a bound of its own size).

    With A = sum of |h| |W| (and of the adapter's |h| |A| |B|) of an element: the norm's rows, the adapter's inner rows and the element itself are stored once
    each, 2^-8 A at most in bf16 (fp32: 2^-24 A); sums of hidden + 64 terms in fp32, those of the norm among them."""
    cfg = (C2.with_(name="kv8_layer", hidden=512, n_q_heads=8, n_kv_heads=2, ffn=1408) if name == "bf16" else C1)
    seed = 4
    batch = gen.batch_scaled(seed, 6, 3, 200, [] if single else [(0, 70, 70), (64, 40, 150)], [] if single else [(96, 50, 146)])
    W, lora = gen.layer_weights(cfg, seed, 0), gen.lora_weights(cfg, seed, 0)
    for w in ("wk", "wv"):                                             # the first head a thousandth as loud as the last
        W[w][:cfg.head_dim] = gen.storage_round(cfg, W[w][:cfg.head_dim] * np.float32(1e-3))
    dev = HH.DeviceLayer(cfg, W, lora)
    ft_req = [r for r in batch.requests if r.kind == KIND_FINETUNE]
    L = batch.seq_capacity[ft_req[0].seq_id] if ft_req else 0
    cache = O8.Cache8(batch.num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    pool = to_device(cfg, cache, batch.num_pages)
    db = kv8.DeviceBatch8(cfg, batch.requests, batch.seq_pages, batch.num_pages)
    hm = db.host_maps
    ws = HH.Workspace(dev.c, hm.T, hm.n_parts, ft_req[0].n_new if ft_req else 0, L)
    x = device(gen.layer_input(cfg, seed, hm.T), cfg)
    y, ft = torch.empty_like(x), HH.DeviceFtState(cfg, L) if ft_req else None
    say("layer", cfg.name, hm.T, "tokens")
    kv8.flexco_kv8_layer_forward(dev.c, dev.w, dev.lora, db.maps, db.runs, db.n_runs, x, y, pool.c, ft.c if ft else None, ws.ptr, ws.bytes)
    codes, scale = from_device(pool)
    om = build_maps(batch.requests, batch.seq_pages, batch.page_size, batch.num_pages)
    states = {ft_req[0].seq_id: OL.FtState(cfg, L)} if ft_req else None
    want = OL.layer_forward_mixed(cfg, W, lora, om, to_np(x), OL.KVPool(batch.num_pages, cfg.page_size, cfg.kv_dim), states, return_all=True)
    slot = om["slot"].astype(np.int64)
    page, at = slot // cfg.page_size, slot % cfg.page_size
    h = np.abs(want["h1"])
    step, fp32 = (2.0 ** -8 if name == "bf16" else 2.0 ** -24), 2.0 ** -24 * (cfg.hidden + 64)
    quiet = 1.0
    for n in "kv":
        A = h @ np.abs(W["w" + n]).astype(np.float64).T + (np.abs(W["b" + n]) if "b" + n in W else 0)
        if n in lora:
            A += cfg.lora_scale * (h @ np.abs(lora[n][0])) @ np.abs(lora[n][1])
        err = (3 * step + fp32) * A
        if n == "k":                                                  # a rotated element has the errors of both of its pair
            pair = err.reshape(hm.T, cfg.n_kv_heads, 2, -1)
            err = np.repeat(pair.sum(2, keepdims=True), 2, 2).reshape(hm.T, -1)
            B = np.abs(want["k"]).reshape(hm.T, cfg.n_kv_heads, 2, -1)
            err = err + 2e-6 * np.repeat(B.sum(2, keepdims=True), 2, 2).reshape(hm.T, -1)
        rows = want[n]
        s = np.repeat(scale[n][page], cfg.head_dim, 1)
        got = (O8.decode(codes[n][page, at]) * scale[n][page][:, :, None]).reshape(hm.T, -1)
        assert np.all(np.abs(got - rows) <= half_step(np.abs(rows) + err, s) + err), n
        # the scale is that of the page's own elements, and not of something larger
        most = np.zeros((batch.num_pages, cfg.n_kv_heads))
        np.maximum.at(most, page, (np.abs(rows) + err).reshape(hm.T, cfg.n_kv_heads, -1).max(2))
        for p in np.unique(page):
            for j in range(cfg.n_kv_heads):
                assert 0 < scale[n][p, j] <= O8.scale_for(most[p, j]), (n, p, j)
        by_head = np.abs(rows).reshape(hm.T, cfg.n_kv_heads, -1).mean((0, 2))
        quiet = min(quiet, by_head[0] / by_head[-1])
    assert quiet < 0.5
