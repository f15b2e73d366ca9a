"""The 8-bit cache on the GPU against the fp64 oracle (oracle/kv8.py): append, attention, pages written out, the layer over such a
cache and its window's backward pass.

Tolerances, derived element by element from the roundings a result passes:
* a cached element: half a step of e4m3 (2^-4 relative, 2^-10 of the scale for the smallest), and for keys and queries
  the rotation's error, |cos|, |sin| to 1e-6;
* attention, with w = sum_j p_j |v_j| of the row: bf16 out 2^-8 |out| (its storage) + 2^-8 w (the probabilities of the second
  product) + the fp32 part; fp32 out the fp32 part alone: each score is off by ds <= 2^-24 ((d + 4)
  sum|q k| / sqrt d + 4 max|s - m|), a probability by 2 ds relative, the sums by 2^-24 (keys + 8);
* log-sum-exp m + log z: ds + 2^-24 (keys + 8) + 2^-23 (|m| + |log z|).
"""
import numpy as np
import pytest
import torch

import paper_2402_18789_amd.binding as B
from paper_2402_18789_amd import host as HH
from paper_2402_18789_amd import kv8
from gpu_common import to_np
from oracle import kv8 as O8
from oracle import ops
from workload import gen
from workload.configs import CONFIGS, KIND_DECODE, KIND_FINETUNE, KIND_PREFILL, Request

pytestmark = pytest.mark.gpu

C2, C1 = CONFIGS["c2_llama8b_layer"], CONFIGS["c1_tiny_f32"]


def shape(nq=8, nkv=2, d=128, dtype="bf16", ps=16, theta=1e4):
    return C2.with_(name="kv8_%d_%d_%d_%s_%d" % (nq, nkv, d, dtype, ps), hidden=256, ffn=256, n_q_heads=nq, n_kv_heads=nkv, head_dim=d,
                    dtype=dtype, page_size=ps, rope_theta=theta, lora_targets=())


def say(*a):
    print(*a, flush=True)


def make_batch(cfg, reqs, seed=0, extra_pages=3, first_page=0):
    """reqs: (kind, start, new tokens).  -> (requests, pages of each sequence, pages in the pool)"""
    n = [-(-(s + k) // cfg.page_size) for _, s, k in reqs]
    ids = gen.rng(seed, "kv8", "pages").permutation(sum(n) + extra_pages) + first_page
    at = np.cumsum([0] + n)
    pages = {i: ids[at[i]:at[i + 1]].astype(np.int32) for i in range(len(n))}
    return [Request(kind=k, seq_id=i, start_pos=s, n_new=m, adapter=-1) for i, (k, s, m) in enumerate(reqs)], pages, first_page + sum(n) + extra_pages


def to_device(cfg, cache, num_pages):
    """the oracle's cache as a device pool"""
    pool = kv8.DevicePool8(cfg, num_pages)
    n, ps, nkv, d = cache.codes["k"].shape
    pool.k[:n] = torch.from_numpy(np.ascontiguousarray(cache.codes["k"].reshape(n, ps, nkv, d // 16, 16).transpose(0, 2, 3, 1, 4)))
    pool.v[:n] = torch.from_numpy(np.ascontiguousarray(cache.codes["v"].transpose(0, 2, 3, 1)))
    pool.k_scale[:n] = torch.from_numpy(cache.scale["k"]).float()
    pool.v_scale[:n] = torch.from_numpy(cache.scale["v"]).float()
    return pool


def from_device(pool):
    """codes [pages, positions, nkv, d] and scales of a device pool"""
    k, v = pool.k.cpu().numpy(), pool.v.cpu().numpy()
    n, nkv, _, ps, _ = k.shape
    return {"k": k.transpose(0, 3, 1, 2, 4).reshape(n, ps, nkv, -1), "v": v.transpose(0, 3, 1, 2)}, \
           {"k": to_np(pool.k_scale), "v": to_np(pool.v_scale)}


def fill_prefixes(cfg, cache, reqs, pages, seed, spread=1.0):
    """cached rows of every sequence up to its first new token, and stale ones in every other slot of the pool"""
    g = gen.rng(seed, "kv8", "prefix")
    for n in "kv":
        cache.codes[n][...] = g.integers(0, 256, cache.codes[n].shape, dtype=np.uint8)       # stale: any code, NaN among them
        cache.scale[n][...] = 2.0 ** g.integers(-10, 3, cache.scale[n].shape)
    for r in reqs:
        if r.start_pos:
            gain = np.exp(spread * g.standard_normal((2, 1, cfg.kv_dim)))
            rows = g.standard_normal((2, r.start_pos, cfg.kv_dim)) * gain
            cache.append(pages[r.seq_id], 0, rows[0], rows[1])


def device(x, cfg):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to("cuda", HH.TORCH_DTYPE[cfg.dtype])


# ---- append -------------------------------------------------------------------------------------------------

def half_step(x, s):
    """half the distance between neighbouring cached numbers at x (scale s)"""
    a = np.abs(x) / s
    return s * np.maximum(2.0 ** -10, 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -9))) - 4))


def check_append(cfg, reqs_in, seed=0, in_place=False, ld_extra=0, loud=1.0, edit=None):
    reqs, pages, num_pages = make_batch(cfg, reqs_in, seed)
    cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, reqs, pages, seed)
    pool = to_device(cfg, cache, num_pages)
    before = from_device(pool)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    T, qd, kd = db.host_maps.T, cfg.q_dim, cfg.kv_dim
    x = gen.storage_round(cfg, gen.rng(seed, "kv8", "qkv").standard_normal((T, cfg.qkv_dim), dtype=np.float32) * loud)
    if edit is not None:
        edit(x)
    xd = device(x, cfg)
    keep = xd.clone()
    if in_place:
        out, ld = xd, cfg.qkv_dim
    else:
        out, ld = torch.full((T, qd + ld_extra), 7.0, dtype=xd.dtype, device="cuda"), qd + ld_extra
    say("append", cfg.name, reqs_in, "in place" if in_place else "")
    kv8.flexco_kv8_append(HH.c_cfg(cfg), db.maps, db.runs, db.n_runs, xd, pool.c, out, ld)
    torch.cuda.synchronize()
    # nothing but the queries' columns is written
    if in_place:
        assert torch.equal(torch.nan_to_num(xd[:, qd:]), torch.nan_to_num(keep[:, qd:]))
    else:
        assert torch.equal(torch.nan_to_num(xd), torch.nan_to_num(keep)) and (out[:, qd:] == 7.0).all()
    pos = np.concatenate([np.arange(r.start_pos, r.start_pos + r.n_new) for r in reqs])
    x64 = x.astype(np.float64)
    with np.errstate(invalid="ignore"):
        q = ops.rope(x64[:, :qd], pos, cfg.n_q_heads, cfg.head_dim, cfg.rope_theta)
        k = ops.rope(x64[:, qd:qd + kd], pos, cfg.n_kv_heads, cfg.head_dim, cfg.rope_theta)
    v = x64[:, qd + kd:]

    def turned(cols, heads):          # |x| + |partner|: what an angle's error is multiplied by
        t = np.abs(cols).reshape(T, heads, 2, -1)
        return np.repeat(t.sum(2, keepdims=True), 2, 2).reshape(T, -1)

    # (a relative step ends at the type's smallest normal number, 2^-126: below it fp32 numbers lie 2^-149 apart and bf16 ones
    # 2^-133; two products and a sum in fp32, half a step each, and half a step of the result's storage)
    least = 1.5 * 2.0 ** -149 + (2.0 ** -134 if cfg.dtype == "bf16" else 0.0)
    e = 1e-6 * turned(x64[:, :qd], cfg.n_q_heads) + (2.0 ** -8 if cfg.dtype == "bf16" else 2.0 ** -23) * np.abs(q) + least
    ok = np.isfinite(q)
    assert np.all(np.abs(to_np(out[:, :qd]) - q)[ok] <= e[ok]) and not np.isfinite(to_np(out[:, :qd])[~ok]).any()
    # the cache: against the rows themselves, element by element, and every slot that was not written
    t0 = 0
    for r in reqs:
        cache.append(pages[r.seq_id], r.start_pos, k[t0:t0 + r.n_new], v[t0:t0 + r.n_new])
        t0 += r.n_new
    codes, scale = from_device(pool)
    for name in "kv":
        assert np.array_equal(scale[name], cache.scale[name]), name
    assert np.array_equal(O8.decode(codes["v"]), O8.decode(cache.codes["v"]), equal_nan=True)
    t0 = 0
    slack = 1e-6 * turned(x64[:, qd:qd + kd], cfg.n_kv_heads)
    for r in reqs:
        p = np.arange(r.start_pos, r.start_pos + r.n_new)
        pg = pages[r.seq_id][p // cfg.page_size]
        s = np.repeat(cache.scale["k"][pg], cfg.head_dim, 1)
        got = (O8.decode(codes["k"][pg, p % cfg.page_size]) * cache.scale["k"][pg][:, :, None]).reshape(r.n_new, -1)
        kr = k[t0:t0 + r.n_new]
        ok = np.isfinite(kr)
        err = np.abs(got - kr)
        assert np.all(err[ok] <= (half_step(kr, s) + 2 * slack[t0:t0 + r.n_new])[ok]) and np.isnan(got[~ok]).all()
        # the oracle's rounding of the same keys is the device's own but where an angle's error crosses a tie
        codes["k"][pg, p % cfg.page_size] = cache.codes["k"][pg, p % cfg.page_size]
        t0 += r.n_new
    assert np.array_equal(O8.decode(codes["k"]), O8.decode(cache.codes["k"]), equal_nan=True)      # slots not written to
    touched = {int(pages[r.seq_id][p // cfg.page_size]) for r in reqs for p in range(r.start_pos, r.start_pos + r.n_new)}
    others = [i for i in range(num_pages) if i not in touched]
    for name in "kv":
        assert np.array_equal(from_device(pool)[0][name][others], before[0][name][others])
    return pool


D, P, F = KIND_DECODE, KIND_PREFILL, KIND_FINETUNE


@pytest.mark.parametrize("cfg", [shape(), shape(4, 4, 64, "f32"), shape(5, 1, 128), shape(16, 2, 256), shape(3, 3, 48), shape(2, 1, 16, "f32"),
                                 shape(40, 2, 80), shape(4, 2, 64, "f32", 32), shape(4, 2, 128, "bf16", 5), shape(8, 8, 112, "bf16", 64)],
                         ids=lambda c: c.name)
def test_append(cfg):
    check_append(cfg, [(D, 0, 1), (D, 15, 1), (D, 16, 1), (D, 700, 1), (P, 0, 1), (P, 0, 16), (P, 3, 40), (P, 32, 17), (F, 9, 100)])


def test_append_one_token():
    for start in (0, 1, 15, 16, 4095):
        check_append(shape(32, 8), [(D, start, 1)], seed=start)


@pytest.mark.parametrize("in_place,ld_extra", [(True, 0), (False, 8), (False, 1000)])
def test_append_strides(in_place, ld_extra):
    for cfg in (shape(), shape(4, 2, 64, "f32")):
        check_append(cfg, [(D, 33, 1), (P, 5, 50)], in_place=in_place, ld_extra=ld_extra)


@pytest.mark.parametrize("loud", [1e4, 1e-4, 1e30, 1e-30, 1e-38, 0.0])
def test_append_scales(loud):
    """pages whose scale grows a thousandfold, stays, or stands at its least"""
    check_append(shape(4, 2, 64, "f32"), [(D, 33, 1), (D, 16, 1), (P, 5, 50)], loud=loud)
    check_append(shape(), [(D, 33, 1), (D, 16, 1), (P, 5, 50)], loud=loud)


def test_append_values_that_are_no_number():
    def edit(x):
        x[0, :] = np.inf
        x[1, ::3] = np.nan
        x[5, 5::7] = -np.inf
    check_append(shape(), [(D, 33, 1), (D, 16, 1), (P, 5, 50)], edit=edit)
    check_append(shape(4, 2, 64, "f32", 5), [(D, 33, 1), (D, 16, 1), (P, 5, 50)], edit=edit)


def test_append_far_positions():
    """angles of positions up to 2^20 (the cached rows before them are not looked at: few pages, given again and again)"""
    cfg = shape(4, 2, 64, "f32", 16, 1e6)
    start = (1 << 20) - 7
    pages = np.zeros(-(-(start + 20) // 16), dtype=np.int32)
    pages[start // 16:] = [1, 2]
    reqs = [Request(kind=P, seq_id=0, start_pos=start, n_new=20, adapter=-1)]
    db = kv8.DeviceBatch8(cfg, reqs, {0: pages}, 3)
    pool = kv8.DevicePool8(cfg, 3)
    x = gen.rng(0, "kv8", "far").standard_normal((20, cfg.qkv_dim), dtype=np.float32)
    out = torch.empty((20, cfg.q_dim), device="cuda")
    kv8.flexco_kv8_append(HH.c_cfg(cfg), db.maps, db.runs, db.n_runs, device(x, cfg), pool.c, out, cfg.q_dim)
    q = ops.rope(x[:, :cfg.q_dim].astype(np.float64), np.arange(start, start + 20), 4, 64, cfg.rope_theta)
    assert np.max(np.abs(to_np(out) - q)) <= 2e-6 * np.max(np.abs(x)) * 2


def test_every_code_is_rounded_and_read_as_the_format_says():
    """all 256 codes through the pool in 16 and 32 bits, and all midpoints and their neighbours through append"""
    for dtype in ("f32", "bf16"):
        cfg = shape(1, 1, 16, dtype)
        pool = kv8.DevicePool8(cfg, 2)
        pool.k[1] = torch.arange(256, dtype=torch.uint8).view(1, 1, 16, 16)
        pool.v[1] = torch.arange(256, dtype=torch.uint8).view(1, 16, 16)
        pool.k_scale[1], pool.v_scale[1] = 2.0 ** -117, 2.0 ** 100
        wide = HH.DevicePool(cfg, 1)
        pool.expand(torch.tensor([1], dtype=torch.int32, device="cuda"), 16, wide, torch.tensor([0], dtype=torch.int32, device="cuda"))
        assert np.array_equal(to_np(wide.k).reshape(-1), O8.decode(np.arange(256)) * 2.0 ** -117, equal_nan=True)
        assert np.array_equal(to_np(wide.v).reshape(-1), O8.decode(np.arange(256)) * 2.0 ** 100, equal_nan=True)
    cfg = shape(1, 1, 16, "f32")
    m = O8.MAGNITUDES
    mid = ((m[1:] + m[:-1]) / 2).astype(np.float32)
    x = np.concatenate([m.astype(np.float32), mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(500))])
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-len(x) % 15, dtype=np.float32)]).reshape(-1, 15)
    n = len(x)
    v = np.concatenate([np.full((n, 1), 448.0, dtype=np.float32), x], 1)       # every row's scale is one
    reqs, pages, num_pages = make_batch(cfg, [(P, 0, n)])
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    pool = kv8.DevicePool8(cfg, num_pages)
    qkv = np.concatenate([np.zeros((n, 32), dtype=np.float32), v], 1)
    kv8.flexco_kv8_append(HH.c_cfg(cfg), db.maps, db.runs, db.n_runs, device(qkv, cfg), pool.c, torch.empty((n, 16), device="cuda"), 16)
    codes = from_device(pool)[0]["v"][pages[0]].reshape(-1, 16)[:n]
    assert np.array_equal(O8.decode(codes), O8.decode(O8.encode(v)))


def test_runs_outside_the_batch_or_the_page_are_left_out():
    cfg = shape(4, 2, 64, "f32")
    reqs, pages, num_pages = make_batch(cfg, [(D, 33, 1), (P, 5, 50)])
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    pool = kv8.DevicePool8(cfg, num_pages)
    x = device(gen.rng(0, "kv8", "x").standard_normal((51, cfg.qkv_dim)), cfg)
    out = torch.full((51, cfg.q_dim), 7.0, device="cuda")
    bad = torch.tensor([[-1, 2], [50, 2], [51, 1], [3, 0], [3, 17], [1, 12], [1 << 30, 1]], dtype=torch.int32, device="cuda")
    kv8.flexco_kv8_append(HH.c_cfg(cfg), db.maps, bad, len(bad), x, pool.c, out, cfg.q_dim)
    torch.cuda.synchronize()
    assert (out == 7.0).all() and not pool.k.any() and not pool.v.any() and not pool.k_scale.any()


# ---- attention ----------------------------------------------------------------------------------------------

def attention_case(cfg, reqs_in, seed=0, split=0, loud=1.0, spread=0.5, edit=None, first_page=0, use_lse=True):
    """device and oracle on one batch whose new tokens are in the cache already -> errors checked row by row"""
    reqs, pages, num_pages = make_batch(cfg, reqs_in, seed, first_page=first_page)
    local = {i: p - first_page for i, p in pages.items()}
    cache = O8.Cache8(num_pages - first_page, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    whole = [Request(kind=r.kind, seq_id=r.seq_id, start_pos=r.start_pos + r.n_new, n_new=1, adapter=-1) for r in reqs]
    fill_prefixes(cfg, cache, whole, local, seed, spread)
    if edit is not None:
        edit(cache, reqs, local)
    if first_page:
        pool = kv8.DevicePool8(cfg, num_pages)
        part = to_device(cfg, cache, num_pages - first_page)
        for a, b in ((pool.k, part.k), (pool.v, part.v), (pool.k_scale, part.k_scale), (pool.v_scale, part.v_scale)):
            a[first_page:] = b
    else:
        pool = to_device(cfg, cache, num_pages)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages, split)
    T = db.host_maps.T
    q = gen.storage_round(cfg, gen.rng(seed, "kv8", "q").standard_normal((T, cfg.q_dim), dtype=np.float32) * loud)
    ws = HH.Workspace(HH.c_cfg(cfg), T, db.host_maps.n_parts)
    ws.buf.fill_(0xFF)                                           # (partial rows that are not written are NaN)
    out = torch.full((T, cfg.q_dim), float("nan"), dtype=HH.TORCH_DTYPE[cfg.dtype], device="cuda")
    lse = torch.full((T, cfg.n_q_heads), float("nan"), device="cuda") if use_lse else None
    say("attention", cfg.name, reqs_in if len(reqs_in) < 12 else len(reqs_in), "split", split)
    kv8.flexco_kv8_attention(HH.c_cfg(cfg), db.maps, device(q, cfg), pool.c, out, lse, ws.ptr, ws.bytes)
    torch.cuda.synchronize()
    return cfg, cache, reqs, local, q, to_np(out), None if lse is None else to_np(lse)


def check_attention(cfg, reqs_in, rows_of=None, **kw):
    cfg, cache, reqs, pages, q, out, lse = attention_case(cfg, reqs_in, **kw)
    nq, nkv, d, g = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.n_q_heads // cfg.n_kv_heads
    bf16, t0 = cfg.dtype == "bf16", 0
    worst = 0.0
    for r in reqs:
        end = r.start_pos + r.n_new
        K, V = cache.rows("k", pages[r.seq_id], end), cache.rows("v", pages[r.seq_id], end)
        for i in range(r.n_new):
            if rows_of is not None and i not in rows_of and i != r.n_new - 1:
                continue
            n = r.start_pos + i + 1
            qi = q[t0 + i].astype(np.float64).reshape(nkv, g, d)
            k, v = K[:n].reshape(n, nkv, d), V[:n].reshape(n, nkv, d)
            with np.errstate(invalid="ignore"):
                s = np.einsum("hgd,nhd->hgn", qi, k) / np.sqrt(d)
                size = np.einsum("hgd,nhd->hgn", np.abs(qi), np.abs(k)).max(2) / np.sqrt(d)
                m = s.max(2, keepdims=True)
                p = np.exp(s - m)
                z = p.sum(2)
                o = np.einsum("hgn,nhd->hgd", p, v) / z[..., None]
                w = np.einsum("hgn,nhd->hgd", p, np.abs(v)) / z[..., None]
                far = (m[..., 0] - s.min(2))
                want = m[..., 0] + np.log(z)
                ds = 2.0 ** -24 * ((d + 4) * size + 4 * np.minimum(far, 100.0))
                fp32 = (2 * ds + 2.0 ** -24 * (n + 8))[..., None] * w + 2.0 ** -23 * np.abs(o)
                # (a probability below fp32's smallest normal number, relative to the row's largest, may be zero: with scores 300 apart the
                # exact e^-300 of a key is all that a channel in which the nearest keys' codes are zero has)
                fp32 = fp32 + n * 2.0 ** -126 * np.abs(v).max(0)[:, None]
                tol = fp32 + (2.0 ** -8 * np.abs(o) + 2.0 ** -8 * w if bf16 else 0)
                got = out[t0 + i].reshape(nkv, g, d)
                assert np.array_equal(np.isnan(o), np.isnan(got)), (r, i)
                ok = ~np.isnan(o)
                ratio = np.max((np.abs(got - o) / np.maximum(tol, 1e-300))[ok], initial=0.0)
            worst = max(worst, ratio)
            assert ratio <= 1.0, (r, i, ratio)
            if lse is not None:
                gl = lse[t0 + i].reshape(nkv, g)
                okl = ~np.isnan(want)
                assert np.array_equal(okl, ~np.isnan(gl))
                # (m and log z are rounded each at their own size, and may cancel: hence not 2^-23 |lse|)
                tol = ds + 2.0 ** -24 * (n + 8) + 2.0 ** -23 * (np.abs(m[..., 0]) + np.abs(np.log(z)))
                assert np.all((np.abs(gl - want) <= tol)[okl]), (r, i, np.abs(gl - want) / tol, want, m[..., 0])
        t0 += r.n_new
    say("  worst error / bound %.2f" % worst)


MIXED = [(D, 0, 1), (D, 15, 1), (D, 16, 1), (D, 63, 1), (D, 64, 1), (D, 333, 1), (P, 0, 1), (P, 0, 33), (P, 70, 18), (F, 41, 70)]


@pytest.mark.parametrize("cfg", [shape(), shape(4, 4, 64, "f32"), shape(32, 8), shape(40, 8), shape(16, 1), shape(8, 8), shape(3, 1), shape(14, 2),
                                 shape(32, 1), shape(4, 2, 64), shape(16, 2, 256), shape(6, 3, 48, "f32"), shape(4, 2, 128, "f32"),
                                 shape(2, 2, 80), shape(4, 2, 64, "f32", 32), shape(4, 2, 128, "bf16", 5), shape(4, 4, 112, "bf16", 64)],
                         ids=lambda c: c.name)
@pytest.mark.parametrize("split", [0, 2])
def test_attention(cfg, split):
    check_attention(cfg, MIXED, split=split)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 1000])
def test_attention_lengths(n):
    """one token, every kind of end of a page, of a group of pages and of a step"""
    check_attention(shape(8, 2), [(D, n - 1, 1)], seed=n)
    check_attention(shape(8, 2), [(P, 0, n)], seed=n, rows_of=(0, 1, n // 2, n - 2))


@pytest.mark.parametrize("split", [0, 2, 4, 8, 16, 32, 64, 256])
def test_attention_splits(split):
    check_attention(shape(8, 2), [(D, 3000, 1), (D, 700, 1), (D, 2, 1), (P, 900, 70), (F, 1300, 33)], split=split, rows_of=(0, 31))


def test_attention_long_and_many():
    check_attention(shape(10, 2), [(D, 20000, 1)])
    check_attention(shape(8, 1), [(D, 20000, 1), (D, 5, 1)])
    check_attention(shape(8, 2), [(D, int(v), 1) for v in gen.rng(3, "kv8", "many").integers(0, 400, 300)])
    check_attention(shape(8, 2), [(P, 1100, 300)], rows_of=(0, 100, 255))


@pytest.mark.parametrize("loud,spread", [(30.0, 0.5), (1e-3, 0.5), (1.0, 3.0), (1e-20, 0.5), (0.0, 0.5)])
def test_attention_ranges(loud, spread):
    """sharp and flat softmaxes, pages of very different scales, queries next to nothing"""
    for cfg in (shape(8, 2), shape(4, 2, 64, "f32")):
        check_attention(cfg, [(D, 333, 1), (D, 40, 1), (P, 70, 40)], loud=loud, spread=spread)


def test_attention_scales_far_apart():
    """a page of values a million times another's, in either order, and one of zeros"""
    def edit(cache, reqs, pages):
        for i, r in enumerate(reqs):
            for j, page in enumerate(pages[i][:-1]):
                cache.scale["v"][page] *= 2.0 ** [0, 20, -20, 0, 9, -40][(i + j) % 6]
                if (i + j) % 7 == 6:
                    cache.codes["v"][page] = 0
                    cache.scale["v"][page] = 2.0 ** -117
    for split in (0, 2):
        check_attention(shape(8, 2), [(D, 333, 1), (D, 40, 1), (D, 250, 1), (P, 70, 40), (P, 0, 100)], edit=edit, split=split)


def test_attention_what_is_masked_never_shows():
    """stale slots are NaN codes already (fill_prefixes); here every position behind a token's own is NaN too, for the
    earlier tokens of the same chunk, and NaN at a visible position shows in every row that sees it"""
    def edit(cache, reqs, pages):
        for name in "kv":
            for i, at in ((1, 60), (2, 5), (3, 100)):
                cache.codes[name][pages[i][at // 16], at % 16, 0, 7] = 0x7F
        cache.codes["v"][pages[0][2], 3, 1, 100] = 0xFF
    check_attention(shape(8, 2), [(D, 333, 1), (P, 30, 64), (P, 0, 40), (F, 41, 70), (D, 50, 1)], edit=edit)
    check_attention(shape(4, 2, 64, "f32"), [(D, 333, 1), (P, 30, 64), (P, 0, 40), (F, 41, 70), (D, 50, 1)], edit=lambda *a: None)


def test_attention_without_lse():
    check_attention(shape(8, 2), [(D, 333, 1), (P, 70, 40)], use_lse=False)
    check_attention(shape(8, 2), [(D, 333, 1), (P, 70, 40)], use_lse=False, split=2)


def test_attention_pool_past_4_gib():
    """pages whose codes lie beyond 2^32 bytes"""
    cfg = shape(32, 16)
    first = (1 << 32) // (16 * 16 * 128)
    check_attention(cfg, [(D, 333, 1), (P, 70, 40)], first_page=first)


def test_same_inputs_same_bits():
    cfg = shape(40, 8)
    reqs = [(D, 2000, 1), (D, 900, 1), (P, 300, 90), (F, 41, 70)]
    a, b = attention_case(cfg, reqs, split=8), attention_case(cfg, reqs, split=8)
    assert np.array_equal(a[5], b[5]) and np.array_equal(a[6], b[6])


# ---- pages written out, gradients, the layer ----------------------------------------------------------------

@pytest.mark.parametrize("cfg", [shape(), shape(4, 4, 64, "f32"), shape(3, 3, 48, "bf16", 5), shape(2, 1, 16, "f32", 32), shape(8, 8, 112, "bf16", 64)],
                         ids=lambda c: c.name)
@pytest.mark.parametrize("short", [0, 1, -1])
def test_expand(cfg, short):
    n = 7
    left = {0: 0, 1: 1, -1: cfg.page_size - 1}[short]          # slots behind the sequence's last token
    g = gen.rng(0, "kv8", "expand")
    cache = O8.Cache8(n, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    for name in "kv":
        cache.codes[name][...] = g.integers(0, 256, cache.codes[name].shape, dtype=np.uint8)
        cache.scale[name][...] = 2.0 ** g.integers(-10, 3, cache.scale[name].shape)
    pool = to_device(cfg, cache, n)
    wide = HH.DevicePool(cfg, 9)
    src = torch.tensor([5, 0, -1, 6, 7, 2, 1], dtype=torch.int32, device="cuda")
    dst = torch.tensor([8, 1, 2, 9, 3, 4, -5], dtype=torch.int32, device="cuda")     # pairs outside a pool are left out
    wide.k.fill_(3.0)
    wide.v.fill_(3.0)
    src[-1], dst[-2], dst[-1] = 2, -5, 4                                           # (the pages' last is the sequence's last)
    pool.expand(src, n * cfg.page_size - left, wide, dst)
    k, v = to_np(wide.k), to_np(wide.v)
    for page in range(9):
        at = {8: 5, 1: 0, 4: 2}.get(page)
        if at is None:
            assert (k[page] == 3.0).all() and (v[page] == 3.0).all()
        else:
            x = {m: O8.decode(cache.codes[m][at]) * cache.scale[m][at][None, :, None] for m in "kv"}
            if page == 4 and left:
                x["k"][-left:] = x["v"][-left:] = 0.0
            assert np.array_equal(k[page], x["k"].transpose(1, 0, 2), equal_nan=True)
            assert np.array_equal(v[page], x["v"].transpose(1, 2, 0), equal_nan=True)


@pytest.mark.parametrize("cfg", [shape(8, 2), shape(4, 2, 64, "f32")], ids=lambda c: c.name)
def test_window_backward_on_the_expanded_pages(cfg):
    """append a window, attend, write the pages out, attention's backward: against the formulas, and the formulas against
    differences of the attention over the cache"""
    start, n = 37, 50
    reqs, pages, num_pages = make_batch(cfg, [(F, start, n)])
    cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, reqs, pages, 0, 0.3)
    pool = to_device(cfg, cache, num_pages)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages)
    c, x = HH.c_cfg(cfg), device(gen.rng(1, "kv8", "qkv").standard_normal((n, cfg.qkv_dim)), cfg)
    ws = HH.Workspace(c, n, db.host_maps.n_parts, n, start + n)
    q, out = (torch.empty((n, cfg.q_dim), dtype=x.dtype, device="cuda") for _ in range(2))
    lse = torch.empty((n, cfg.n_q_heads), device="cuda")
    kv8.flexco_kv8_append(c, db.maps, db.runs, db.n_runs, x, pool.c, q, cfg.q_dim)
    kv8.flexco_kv8_attention(c, db.maps, q, pool.c, out, lse, ws.ptr, ws.bytes)
    wide = HH.DevicePool(cfg, len(pages[0]))
    seq = torch.arange(len(pages[0]), dtype=torch.int32, device="cuda")
    pool.expand(torch.from_numpy(pages[0]).cuda(), start + n, wide, seq)
    dout = device(gen.rng(2, "kv8", "dout").standard_normal((n, cfg.q_dim)), cfg)
    dq = torch.empty_like(q)
    dk = torch.zeros((start + n, cfg.kv_dim), device="cuda")
    dv = torch.zeros_like(dk)
    B.flexco_attention_window_bwd(c, wide.c, seq, len(seq), start, n, q, out, lse, dout, dq, dk, dv, ws.ptr, ws.bytes)
    codes, scale = from_device(pool)
    cache.codes, cache.scale = codes, scale
    K, V = cache.rows("k", pages[0], start + n), cache.rows("v", pages[0], start + n)
    Q, pos = to_np(q), np.arange(start, start + n)
    want = ops.attention_bwd(Q, pos, K, V, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, to_np(dout))
    for got, ref in zip((dq, dk, dv), want):
        assert np.max(np.abs(to_np(got) - ref)) <= (1e-4 if cfg.dtype == "f32" else 2e-2) * np.max(np.abs(ref))
    f = lambda a, b, v: np.sum(ops.attention(a, pos, b, v, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim)[0] * to_np(dout))  # noqa: E731
    g = gen.rng(3, "kv8", "dir")
    for i, base in enumerate((Q, K, V)):
        step = 1e-5 * g.standard_normal(base.shape)
        plus, minus = [Q, K, V], [Q, K, V]
        plus[i], minus[i] = base + step, base - step
        assert abs((f(*plus) - f(*minus)) / 2 - np.sum(want[i] * step)) <= 1e-6 * np.sum(np.abs(want[i] * step))


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_layer_over_the_8_bit_cache_and_its_windows_way_back(name):
    """flexco_kv8_layer_forward leaves the state that flexco_layer_forward leaves on a 16-bit pool holding the same cached
    numbers: the second runs on pages written out of the first's cache, so only the new rows' rounding lies between the two, and that is
    taken out by giving the 16-bit layer's later tokens nothing but expanded pages: one decode-sized window."""
    cfg = (C2.with_(name="kv8_layer", hidden=512, n_q_heads=8, n_kv_heads=2, ffn=1408) if name == "bf16" else C1)
    seed = 4
    batch = gen.batch_scaled(seed, 6, 3, 200, [(0, 70, 70), (64, 40, 150)], [(96, 50, 146)])
    W, lora = gen.layer_weights(cfg, seed, 0), gen.lora_weights(cfg, seed, 0)
    dev = HH.DeviceLayer(cfg, W, lora)
    ft_req = [r for r in batch.requests if r.kind == KIND_FINETUNE][0]
    L = batch.seq_capacity[ft_req.seq_id]
    cache = O8.Cache8(batch.num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, batch.requests, batch.seq_pages, seed, 0.2)
    pool = to_device(cfg, cache, batch.num_pages)
    db = kv8.DeviceBatch8(cfg, batch.requests, batch.seq_pages, batch.num_pages)
    hm = db.host_maps
    ws = HH.Workspace(dev.c, hm.T, hm.n_parts, ft_req.n_new, L)
    x = device(gen.layer_input(cfg, seed, hm.T), cfg)
    y, ft = torch.empty_like(x), HH.DeviceFtState(cfg, L)
    kv8.flexco_kv8_layer_forward(dev.c, dev.w, dev.lora, db.maps, db.runs, db.n_runs, x, y, pool.c, ft.c, ws.ptr, ws.bytes)
    # the oracle's layer with the device's own cached numbers in the place of its pool
    from oracle import layer as OL
    from oracle.maps import build_maps
    codes, scale = from_device(pool)
    cache.codes, cache.scale = codes, scale

    class Cached(OL.KVPool):
        """takes the batch's rows and keeps what the 8-bit cache made of them"""
        def __init__(self):
            super().__init__(batch.num_pages, cfg.page_size, cfg.kv_dim)
            every = np.repeat(np.arange(batch.num_pages), cfg.page_size), np.tile(np.arange(cfg.page_size), batch.num_pages)
            for n in "kv":
                rows = O8.decode(codes[n][every]) * scale[n][every[0]][:, :, None]
                arr = np.nan_to_num(rows.reshape(len(rows), -1))
                frozen = arr.view(Frozen)
                setattr(self, n, frozen)

    class Frozen(np.ndarray):
        def __setitem__(self, at, rows):
            near = np.asarray(self[at])
            # what was written must be the rows' rounding, up to the storage type's error of the rows themselves
            assert np.max(np.abs(near - rows)) <= (2.0 ** -4 + 0.03) * np.max(np.abs(rows))

    st = OL.FtState(cfg, L)
    om = build_maps(batch.requests, batch.seq_pages, batch.page_size, batch.num_pages)
    want = OL.layer_forward_mixed(cfg, W, lora, om, to_np(x), Cached(), {ft_req.seq_id: st})
    tol = 1e-4 if name == "f32" else 2e-2
    assert np.max(np.abs(to_np(y) - want)) <= tol * np.max(np.abs(want))
    win = slice(ft_req.start_pos, ft_req.start_pos + ft_req.n_new)
    for a in ("q_cache", "attn", "x2", "gate", "up", "lse"):
        got, ref = to_np(getattr(ft, a))[win], np.asarray(getattr(st, a))[win]
        assert np.max(np.abs(got - ref)) <= tol * np.max(np.abs(ref)), a
    # back through the layer on the expanded pages
    pages = batch.seq_pages[ft_req.seq_id]
    end = ft_req.start_pos + ft_req.n_new
    wide = HH.DevicePool(cfg, len(pages))
    seq = torch.arange(len(pages), dtype=torch.int32, device="cuda")
    pool.expand(torch.from_numpy(np.asarray(pages, dtype=np.int32)).cuda(), end, wide, seq)
    dY = device(gen.storage_round(cfg, gen.layer_input(cfg, seed, ft_req.n_new, tag="dy")), cfg)
    dX = torch.empty_like(dY)
    B.flexco_lora_bwd(dev.c, dev.w, dev.lora, wide.c, seq, len(seq), ft.c, ft_req.start_pos, ft_req.n_new, dY, dX, ws.ptr, ws.bytes)
    grads = {}
    K, V = cache.rows("k", pages, end), cache.rows("v", pages, end)
    want_dx = OL.layer_backward_window(cfg, W, lora, st, K, V, ft_req.start_pos, ft_req.n_new, to_np(dY), grads)
    tol = 1e-4 if name == "f32" else 4e-2        # (bf16: the storage type alone is 2.5e-2 on windows of under 100 keys)
    assert np.max(np.abs(to_np(dX) - want_dx)) <= tol * np.max(np.abs(want_dx))
    for t, (dA, dB) in dev.grads_numpy().items():
        for got, ref in zip((dA, dB), grads[t]):
            assert np.max(np.abs(got - ref)) <= tol * np.max(np.abs(ref)), t


def test_generation_step_by_step_equals_whole_chunks():
    """a prompt appended whole or token by token, attended to from the last token: the same where no page's scale grew, and in any
    case within what the cache's rounding allows"""
    cfg = shape(8, 2)
    n = 45
    x = gen.storage_round(cfg, gen.rng(5, "kv8", "steps").standard_normal((n, cfg.qkv_dim), dtype=np.float32))
    x[::16] = np.sign(x[::16]) * 3.9                        # each page's first row is its loudest
    x = np.clip(x, -3.9, 3.9)
    x[:, cfg.q_dim:cfg.q_dim + cfg.kv_dim] *= 0.5
    pages, outs = {0: np.array([2, 0, 1], dtype=np.int32)}, []
    for steps in ([n], [1] * n, [7, 20, 18]):
        pool, at = kv8.DevicePool8(cfg, 3), 0
        for m in steps:
            reqs = [Request(kind=P if m > 1 else D, seq_id=0, start_pos=at, n_new=m, adapter=-1)]
            db = kv8.DeviceBatch8(cfg, reqs, pages, 3)
            q, out = torch.empty((m, cfg.q_dim), dtype=torch.bfloat16, device="cuda"), torch.empty((m, cfg.q_dim), dtype=torch.bfloat16, device="cuda")
            ws = HH.Workspace(HH.c_cfg(cfg), m, db.host_maps.n_parts)
            kv8.flexco_kv8_append(HH.c_cfg(cfg), db.maps, db.runs, db.n_runs, device(x[at:at + m], cfg), pool.c, q, cfg.q_dim)
            kv8.flexco_kv8_attention(HH.c_cfg(cfg), db.maps, q, pool.c, out, None, ws.ptr, ws.bytes)
            at += m
        outs.append((to_np(out[-1]), to_np(pool.v_scale), pool.v.clone()))
    for o, s, v in outs[1:]:
        assert np.array_equal(s, outs[0][1]) and torch.equal(v, outs[0][2])
        assert np.max(np.abs(o - outs[0][0])) <= 2e-2 * np.max(np.abs(o))


def test_calls_replay_from_a_graph_and_follow_their_stream():
    """append, attention and expand captured once, replayed on new inputs with eager work between, on a stream of their own; two
    graphs over the one workspace run one after the other"""
    cfg = shape(8, 2)
    reqs, pages, num_pages = make_batch(cfg, [(D, 333, 1), (D, 40, 1), (P, 70, 40), (F, 41, 70)])
    cache = O8.Cache8(num_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
    fill_prefixes(cfg, cache, reqs, pages, 0)
    db = kv8.DeviceBatch8(cfg, reqs, pages, num_pages, 4)
    c, T = HH.c_cfg(cfg), db.host_maps.T
    ws = HH.Workspace(c, T, db.host_maps.n_parts)
    x = device(gen.rng(7, "kv8", "x").standard_normal((T, cfg.qkv_dim)), cfg)
    fresh = to_device(cfg, cache, num_pages)
    pool = to_device(cfg, cache, num_pages)
    q, out = (torch.zeros((T, cfg.q_dim), dtype=x.dtype, device="cuda") for _ in range(2))
    lse = torch.zeros((T, cfg.n_q_heads), device="cuda")
    seq = torch.from_numpy(pages[3]).cuda()
    wide = HH.DevicePool(cfg, num_pages)

    def reset():
        for a, b in ((pool.k, fresh.k), (pool.v, fresh.v), (pool.k_scale, fresh.k_scale), (pool.v_scale, fresh.v_scale)):
            a.copy_(b)
        out.zero_()

    def step():
        kv8.flexco_kv8_append(c, db.maps, db.runs, db.n_runs, x, pool.c, q, cfg.q_dim)
        kv8.flexco_kv8_attention(c, db.maps, q, pool.c, out, lse, ws.ptr, ws.bytes)
        pool.expand(seq, 111, wide, seq)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (q, out, lse, pool.k, pool.v, pool.k_scale, wide.k, wide.v)]

    def same(a, b):
        return all(torch.equal(torch.nan_to_num(u.float()), torch.nan_to_num(v.float())) for u, v in zip(a, b))

    reset()
    step()
    eager = results()
    side = torch.cuda.Stream()
    reset()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert same(results(), eager)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for i in range(4):
        reset()
        x.add_(0.0)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        assert same(results(), eager), i
    x.copy_(device(gen.rng(8, "kv8", "x").standard_normal((T, cfg.qkv_dim)), cfg))
    reset()
    step()
    eager2 = results()
    reset()
    graphs[1].replay()
    assert same(results(), eager2) and not same(eager2, eager)
