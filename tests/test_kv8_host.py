"""The 8-bit cache without a GPU: the oracle's number format and append against hand values and torch's type, the runs of a
batch, what the entry points refuse before anything is launched, and the header against the binding."""
import ctypes as C
import os
import re
from types import SimpleNamespace as NS

import numpy as np
import pytest
import torch

import paper_2402_18789_amd.binding as B
from paper_2402_18789_amd import kv8
from oracle import kv8 as O8
from workload import CONFIGS, gen

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
full_library = pytest.mark.skipif(B.HOST_ONLY, reason="needs the whole library, this is a host-only build")


@full_library
def test_header_and_binding_name_the_same_entry_points():
    header = open(os.path.join(ROOT, "include", "flexco_kv8.h")).read()
    code = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    assert set(re.findall(r"\b(flexco_kv8_[a-z_0-9]+)\s*\(", code)) == set(kv8.EXPORTS)
    lib = C.CDLL(B.LIB_PATH)
    assert all(hasattr(lib, n) for n in kv8.EXPORTS)
    assert kv8.flexco_kv8_abi_version() == kv8.KV8_ABI_VERSION


# ---- the oracle ---------------------------------------------------------------------------------------------

def test_e4m3_hand_values():
    for code, value in ((0x00, 0.0), (0x01, 2.0 ** -9), (0x07, 7 * 2.0 ** -9), (0x08, 2.0 ** -6), (0x38, 1.0), (0x39, 1.125), (0x7E, 448.0), (0xB8, -1.0), (0xFE, -448.0)):
        assert O8.decode(code) == value and O8.encode(value) == code
    assert np.isnan(O8.decode([0x7F, 0xFF])).all()
    # ties go to the even code, values beyond the last step's half stay at it
    assert O8.encode(1.0625) == 0x38 and O8.encode(1.1875) == 0x3A and O8.encode(2.0 ** -10) == 0 and O8.encode(1.5 * 2.0 ** -9) == 2


def test_e4m3_against_torchs_type():
    codes = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(O8.decode(codes), t, equal_nan=True)
    x = np.concatenate([gen.rng(0, "e4m3", i).standard_normal(4000) * s for i, s in enumerate((100.0, 1.0, 2.0 ** -6, 2.0 ** -9))]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    assert np.array_equal(O8.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_scale_is_the_least_power_of_two():
    assert [O8.scale_for(v) for v in (448.0, 448.001, 1.75, 1.7500001, 1.0, 0.0, 1e-40)] == [1.0, 2.0, 2.0 ** -8, 2.0 ** -7, 2.0 ** -8, 2.0 ** -117, 2.0 ** -117]


def test_append_raises_a_pages_scale_and_rounds_what_was_there():
    c = O8.Cache8(2, 4, 1, 16)
    one = np.ones((1, 16))
    c.append([1], 0, one, one)
    assert c.scale["k"][1, 0] == 2.0 ** -8 and O8.decode(c.codes["k"][1, 0, 0, 0]) == 256.0
    c.append([1], 1, 2000 * one, 0.25 * one)
    assert c.scale["k"][1, 0] == 8.0 and c.scale["v"][1, 0] == 2.0 ** -8          # 2000 / 8 = 250 -> 256; the values keep theirs
    assert np.array_equal(c.rows("k", [1], 2)[:, 0], [1.0, 2048.0])                # (1 = 2^-3 * 8, still exact)
    assert np.array_equal(c.rows("v", [1], 2)[:, 0], [1.0, 0.25])
    c.append([1], 2, 1e-3 * one, one)                                            # 1e-3 / 8 is below half the smallest code
    assert c.rows("k", [1], 3)[2, 0] == 0.0
    c.append([1], 0, one, one)                                                   # a run that begins the page begins its scale
    assert c.scale["k"][1, 0] == 2.0 ** -8


def test_append_does_not_depend_on_the_chunks_where_the_scale_does_not():
    rows = gen.rng(1, "kv8", "rows").standard_normal((2, 23, 32))
    rows[:, 0, :] = 4.0                                                          # every page's largest comes first ...
    rows[:, 8, :] = rows[:, 16, :] = 4.0
    rows = np.clip(rows, -4, 4)
    a, b = O8.Cache8(3, 8, 2, 16), O8.Cache8(3, 8, 2, 16)
    a.append([2, 0, 1], 0, *rows)
    for i in range(23):
        b.append([2, 0, 1], i, rows[0, i:i + 1], rows[1, i:i + 1])
    for n in "kv":
        assert np.array_equal(a.rows(n, [2, 0, 1], 23), b.rows(n, [2, 0, 1], 23))
        assert np.max(np.abs(a.rows(n, [2, 0, 1], 23) - rows["kv".index(n)]) / np.abs(rows["kv".index(n)])) <= 2.0 ** -4


# ---- runs ---------------------------------------------------------------------------------------------------

def host_maps(reqs, pages, ps=4, num_pages=16, nq=4, nkv=2):
    desc, keep = B.make_batch_desc([r.kind for r in reqs], [r.start_pos for r in reqs], [r.n_new for r in reqs], [r.adapter for r in reqs],
                                   [pages[r.seq_id] for r in reqs])
    m, blob = B.flexco_build_maps(desc, ps, num_pages, nq, nkv)
    return m, (blob, keep)


def R(kind, seq, start, n):
    return NS(kind=kind, seq_id=seq, start_pos=start, n_new=n, adapter=-1)


def test_runs_are_the_tokens_of_a_page():
    m, keep = host_maps([R(0, 0, 5, 1), R(1, 1, 0, 9), R(1, 2, 3, 2), R(0, 3, 0, 1), R(0, 4, 1, 1)],
                        {0: [3, 1], 1: [2, 0, 5], 2: [4, 6], 3: [7], 4: [8]})
    assert kv8.flexco_kv8_runs(m).tolist() == [[0, 1], [1, 4], [5, 4], [9, 1], [10, 1], [11, 1], [12, 1], [13, 1]]


@pytest.mark.parametrize("seed", range(4))
def test_runs_tile_the_batch(seed):
    b = gen.batch_scaled(seed, 9, 1, 90, [(0, 37, 37), (64, 50, 130)], [(96, 33, 129)])
    m, keep = host_maps(b.requests, b.seq_pages, b.page_size, b.num_pages)
    runs = kv8.flexco_kv8_runs(m)
    slots = B.maps_to_numpy(m, keep[0])["slot"]
    assert runs[0, 0] == 0 and np.array_equal(runs[1:, 0], runs[:-1].sum(1)) and runs[-1].sum() == b.n_tokens
    seen = set()
    for t, n in runs:
        assert np.array_equal(slots[t:t + n], np.arange(slots[t], slots[t] + n)) and slots[t] // b.page_size == slots[t + n - 1] // b.page_size
        assert slots[t] // b.page_size not in seen
        seen.add(slots[t] // b.page_size)


def test_two_runs_in_one_page_are_refused():
    # two sequences that share a page, each writing a slot of its own; a sequence that holds a page twice
    for reqs, pages in (([R(0, 0, 1, 1), R(0, 1, 2, 1)], {0: [3], 1: [3]}), ([R(1, 0, 2, 4)], {0: [3, 3]}),
                        ([R(0, 0, 1, 1), R(0, 1, 0, 1), R(0, 2, 3, 1)], {0: [3], 1: [4], 2: [3]})):
        m, keep = host_maps(reqs, pages)
        with pytest.raises(B.FlexcoError) as e:
            kv8.flexco_kv8_runs(m)
        assert e.value.code == B.FLEXCO_EPAGE and "page 3" in str(e.value)
    # ... reading a shared page is no matter
    m, keep = host_maps([R(0, 0, 4, 1), R(0, 1, 4, 1)], {0: [3, 4], 1: [3, 5]})
    assert len(kv8.flexco_kv8_runs(m)) == 2


def test_runs_refuse_bad_arguments():
    m, keep = host_maps([R(1, 0, 0, 9)], {0: [1, 2, 3]})
    with pytest.raises(B.FlexcoError) as e:
        kv8.flexco_kv8_runs(m, capacity=2)
    assert e.value.code == B.FLEXCO_EWORKSPACE
    assert len(kv8.flexco_kv8_runs(m, capacity=3)) == 3
    with pytest.raises(B.FlexcoError) as e:
        kv8.flexco_kv8_runs(B.Maps())
    assert e.value.code == B.FLEXCO_EINVAL
    with pytest.raises(B.FlexcoError):
        kv8.flexco_kv8_runs(m, capacity=-1)


# ---- refusals -----------------------------------------------------------------------------------------------

def refused(code, fn, *args):
    with pytest.raises(B.FlexcoError) as e:
        fn(*args)
    assert e.value.code == code, str(e.value)
    return str(e.value)


@full_library
def test_calls_are_refused_before_anything_is_launched():
    """(every address below is a number: nothing is read or written, no device is there)"""
    from paper_2402_18789_amd.host import c_cfg
    cfg = CONFIGS["c1_tiny_f32"]
    c = c_cfg(cfg)
    m, keep = host_maps([R(0, 0, 5, 1), R(1, 1, 0, 30)], {0: [3], 1: [2, 0]}, 16, 8, cfg.n_q_heads, cfg.n_kv_heads)
    qd, qkvd = cfg.q_dim, cfg.qkv_dim
    good = dict(k_codes=4096, v_codes=8192, k_scale=64, v_scale=128, num_pages=8, page_size=16)
    P = lambda **kw: kv8.Pool(**dict(good, **kw))  # noqa: E731
    A = kv8.flexco_kv8_append
    big = 1 << 30
    for pool, code in ((P(k_codes=None), B.FLEXCO_EINVAL), (P(v_scale=None), B.FLEXCO_EINVAL), (P(k_codes=4104), B.FLEXCO_EINVAL),
                       (P(k_scale=66), B.FLEXCO_EINVAL), (P(num_pages=0), B.FLEXCO_EINVAL), (P(page_size=32), B.FLEXCO_ESHAPE),
                       (P(num_pages=7), B.FLEXCO_EPAGE)):
        refused(code, A, c, m, 256, 3, big, pool, 2 * big, qd, 0)
        refused(code, kv8.flexco_kv8_attention, c, m, big, pool, 2 * big, None, 4 * big, big, 0)
        if code != B.FLEXCO_EPAGE:
            refused(code, kv8.flexco_kv8_expand, c, pool, 256, 1, B.KVPool(16, 32, 4, 16), 512, 0)
    for runs, n in ((None, 3), (258, 3), (256, 0), (256, 32), (256, -1)):
        refused(B.FLEXCO_EINVAL, A, c, m, runs, n, big, P(), 2 * big, qd, 0)
    for qkv, q, ld, code in ((None, big, qd, B.FLEXCO_EINVAL), (big, None, qd, B.FLEXCO_EINVAL), (big + 4, 2 * big, qd, B.FLEXCO_EINVAL),
                             (big, 2 * big + 8, qd, B.FLEXCO_EINVAL), (big, 2 * big, qd - 4, B.FLEXCO_ESHAPE), (big, 2 * big, qd + 1, B.FLEXCO_ESHAPE),
                             (big, big, qd, B.FLEXCO_EINVAL), (big, big + 16, qkvd, B.FLEXCO_EINVAL), (big, big - 4 * qd, qd, B.FLEXCO_EINVAL)):
        refused(code, A, c, m, 256, 3, qkv, P(), q, ld, 0)
    for q, out, lse, ws, size, code in ((None, big, None, big, big, B.FLEXCO_EINVAL), (big, None, None, big, big, B.FLEXCO_EINVAL),
                                        (big, big, None, None, big, B.FLEXCO_EINVAL), (big, big, 8, big, big, B.FLEXCO_EINVAL),
                                        (big, big, None, big, 64, B.FLEXCO_EWORKSPACE)):
        refused(code, kv8.flexco_kv8_attention, c, m, q, P(), out, lse, ws, size, 0)
    wide = B.KVPool(16, 32, 4, 16)
    refused(B.FLEXCO_EINVAL, kv8.flexco_kv8_expand, c, P(), None, 9, wide, 512, 0)
    refused(B.FLEXCO_EINVAL, kv8.flexco_kv8_expand, c, P(), 256, 9, wide, 514, 0)
    refused(B.FLEXCO_EINVAL, kv8.flexco_kv8_expand, c, P(), 256, -1, wide, 512, 0)
    refused(B.FLEXCO_EINVAL, kv8.flexco_kv8_expand, c, P(), 256, 1, B.KVPool(16, None, 4, 16), 512, 0)
    refused(B.FLEXCO_ESHAPE, kv8.flexco_kv8_expand, c, P(), 256, 1, B.KVPool(16, 32, 4, 8), 512, 0)
    kv8.flexco_kv8_expand(c, P(), None, 0, wide, None, 0)                        # no tokens: nothing to do
    # head sizes that are no multiple of 16, maps of other heads
    odd = c_cfg(cfg.with_(head_dim=72))
    assert "16" in refused(B.FLEXCO_ESHAPE, A, odd, m, 256, 3, big, P(), 2 * big, 4 * 72, 0)
    refused(B.FLEXCO_ESHAPE, kv8.flexco_kv8_attention, odd, m, big, P(), 2 * big, None, 4 * big, big, 0)
    refused(B.FLEXCO_ESHAPE, kv8.flexco_kv8_attention, c_cfg(cfg.with_(n_kv_heads=1)), m, big, P(), 2 * big, None, 4 * big, big, 0)
    w = B.BaseWeights(*[16 * i for i in range(1, 8)])
    refused(B.FLEXCO_EINVAL, kv8.flexco_kv8_layer_forward, c, w, None, m, None, 3, big, 2 * big, P(), None, 64, big, 0)
    refused(B.FLEXCO_EPAGE, kv8.flexco_kv8_layer_forward, c, w, None, m, 256, 3, big, 2 * big, P(num_pages=7), None, 64, big, 0)
