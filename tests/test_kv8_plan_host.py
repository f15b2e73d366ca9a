"""How the 8-bit attention cuts a work list (no GPU): the choices at the sizes they were measured at, and what holds for any list."""
import math

import numpy as np
import pytest

import paper_2402_18789_amd.binding as B
from kv8_plan import MAX_PAGES, kv8_plan, pieces
from workload.configs import KIND_DECODE as D, KIND_PREFILL as P


def build(nq, nkv, requests, split=0):
    pages = [-(-(start + n) // 16) for _, start, n in requests]
    first = np.concatenate(([0], np.cumsum(pages)))
    desc, keep = B.make_batch_desc([k for k, _, _ in requests], [s for _, s, _ in requests], [n for _, _, n in requests], [-1] * len(requests),
                                   [np.arange(a, b, dtype=np.int32) for a, b in zip(first, first[1:])])
    return B.flexco_build_maps(desc, 16, int(first[-1]), nq, nkv, split), keep


def plan_of(nq, nkv, requests, split=0):
    (maps, _), _keep = build(nq, nkv, requests, split)
    return kv8_plan(maps, nkv), maps


def decode(n, lo, hi):
    return [(D, int(lo + (i + 0.5) / n * (hi + 1 - lo)) - 1, 1) for i in range(n)]


# (contexts, kv heads) -> pages of a piece (None: whole), wavefronts
@pytest.mark.parametrize("nq,nkv,requests,pages,wavefronts", [
    (32, 8, decode(1, 700, 700), None, 4), (32, 8, decode(4, 1000, 1000), None, 4), (32, 8, decode(32, 100, 1000), None, 4),
    (32, 8, decode(1, 2000, 2000), 16, 4), (8, 1, decode(64, 500, 4096), 32, None), (40, 8, decode(1, 32000, 32000), 64, 4),
    (40, 8, decode(3, 9000, 32765), 64, 4), (40, 8, decode(8, 8000, 8000), 64, 4), (32, 8, decode(96, 4000, 4000), None, 4),
    (32, 8, decode(128, 100, 4096), None, 4), (32, 8, decode(256, 512, 4096), None, 4), (32, 8, decode(256, 10, 600), None, 2),
    (32, 8, decode(512, 16, 400), None, 2)])
def test_single_tokens_at_the_measured_sizes(nq, nkv, requests, pages, wavefronts):
    plan, maps = plan_of(nq, nkv, requests)
    if pages is None:
        assert pieces(maps, plan) == 1
    else:
        assert plan.fold * maps.kv_split_pages == pages and pieces(maps, plan) > 1
    assert wavefronts is None or plan.wavefronts == wavefronts


@pytest.mark.parametrize("requests,whole", [([(P, 0, 189)], True), ([(P, 0, 256)], True), ([(P, 0, 257)], False), ([(P, 372, 13)], False),
                                            ([(P, 400, 100)] + decode(8, 300, 500), False), ([(P, 100, 30)] + decode(3, 20, 250), True)])
def test_short_lists_with_chunks_are_not_cut(requests, whole):
    plan, maps = plan_of(40, 8, requests)
    assert plan.whole == whole and plan.wavefronts == 2
    if whole:
        assert maps.n_parts > maps.n_tiles and plan.fold * maps.kv_split_pages >= maps.max_pages


@pytest.mark.parametrize("seed", range(40))
def test_what_holds_for_any_list(seed):
    g = np.random.default_rng(seed)
    nq, nkv = [(32, 8), (40, 8), (16, 1), (8, 8)][seed % 4]
    reqs = [(D, int(math.exp(g.uniform(0, 9.5))), 1) for _ in range(int(g.choice([0, 1, 3, 40, 300])))]
    reqs += [(P, int(g.integers(0, 2000)), int(g.integers(1, 400))) for _ in range(int(g.integers(0 if reqs else 1, 3)))]
    split = int(g.choice([0, 0, 2, 6, 16, 256, 512]))
    plan, maps = plan_of(nq, nkv, reqs, split)
    sp = maps.kv_split_pages
    assert plan.fold >= 1 and plan.fold & (plan.fold - 1) == 0 and plan.wavefronts in (2, 4)
    assert plan.fold == 1 or plan.fold * sp <= MAX_PAGES
    if maps.n_single != maps.n_items:
        assert plan.wavefronts == 2                              # a list with chunks: two wavefronts' blocks
    if maps.n_single == 0:
        assert plan.fold == 1 or plan.whole
    if plan.whole:
        assert maps.max_pages <= 16 and plan.fold * sp >= maps.max_pages
    if maps.n_parts == maps.n_tiles:
        assert plan.fold == 1 and not plan.whole                 # nothing is cut: nothing to take together
