"""The operators of the 8-bit paged key / value cache: what they compute, in plain torch, and calls of them to be timed.

The cache holds e4m3 numbers (OCP: largest 448, no infinities) in pages of 16 positions, with one scale for each page and
kv head of K and of V, a power of two.  K codes lie [page, kv head, head_dim / 16, position, 16], V codes
[page, kv head, head_dim, position].

* append: the new tokens' keys are turned to their positions, keys and values are rounded into the cache, queries are turned
  and returned.  The tokens a batch writes into one page (a run) share the page's scale: the least power of two that keeps
  them within 448, and no less than the page's own where the run does not begin the page; codes that were there are rounded
  anew to a scale that has grown.
* attention: every token of a mixed batch (decode tokens, prefill chunks, a finetune window) over its sequence's cached positions.
* expand: a sequence's pages written out in the type of the activations, as the window's backward pass and 16-bit pools have
  them; slots behind its last token are zeros there.

`own` false: `run` is that, in elementary operations; true: the package's calls.  Heads are those of the 8B, 14B / 32B and
small fp32 configurations.  Lengths are a function of the case; values and physical pages come from the seed.
"""
import math
from types import SimpleNamespace

import torch

own = False

PAGE = 16
LARGEST = 448.0
LEAST_EXP = -117          # of a scale: every code times it is then a normal number in bfloat16 too
E4M3 = torch.float8_e4m3fn

_HEADS = {  # query heads, kv heads, head_dim, rope base
    "8b": (32, 8, 128, 5e5),
    "14b": (40, 8, 128, 1e6),
    "tiny": (4, 4, 64, 1e4),
    "mqa": (16, 1, 128, 1e4),      # one kv head for all
    "mha": (8, 8, 128, 1e4),       # as many kv heads as query heads
}
_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases ------------------------------------------------------------------------------------------------------

def _batch(decode=0, lo=0, hi=0, median=0, sigma=0.0, prefill="", window=0, seq=0):
    """decode requests with contexts uniform in lo..hi (median 0) or log-normal, clipped to lo..hi; prefill chunks
    "tokens@start" separated by blanks; the last `window` tokens of a finetune sequence of `seq` tokens"""
    return {"decode": decode, "lo": lo, "hi": hi, "median": median, "sigma": sigma, "prefill": prefill, "window": window, "seq": seq}


def listed():
    return [
        # one user's token in a conversation of some hundred tokens: latency is all there is
        dict(name="attend_one_700", op="attention", heads="8b", dtype="bf16", **_batch(decode=1, lo=700, hi=700)),
        # the decode tokens of the benchmark's batch: the cache is the bytes
        dict(name="attend_decode_8b_256", op="attention", heads="8b", dtype="bf16", **_batch(decode=256, lo=512, hi=4096)),
        # few users with long documents: a long axis and few rows
        dict(name="attend_long_14b_3", op="attention", heads="14b", dtype="bf16", **_batch(decode=3, lo=9001, hi=32765)),
        # no request is decoding: whole prompts, a later chunk and a finetune window, the matrix cores' work
        dict(name="attend_chunks_14b_4096", op="attention", heads="14b", dtype="bf16", **_batch(prefill="2048@0 1024@1999", window=1024, seq=4096)),
        # a co-served iteration of all three kinds, ragged
        dict(name="attend_mixed_14b", op="attention", heads="14b", dtype="bf16", **_batch(decode=301, lo=16, hi=8192, median=700, sigma=0.8, prefill="211@0 77@800", window=205, seq=2000)),
        # the fp32 configuration
        dict(name="attend_f32", op="attention", heads="tiny", dtype="f32", **_batch(decode=4, lo=16, hi=64, prefill="32@0", window=32, seq=64)),
        # one decode token is written
        dict(name="append_one", op="append", heads="8b", dtype="bf16", **_batch(decode=1, lo=700, hi=700)),
        # a decode step's tokens, one in a page each
        dict(name="append_decode_14b_512", op="append", heads="14b", dtype="bf16", **_batch(decode=512, lo=17, hi=400)),
        # a budget of prompts and a window, whole pages and their ragged ends
        dict(name="append_chunks_8b_4000", op="append", heads="8b", dtype="bf16", **_batch(decode=77, lo=16, hi=300, prefill="2011@0 700@333", window=1212, seq=2000)),
        # the fp32 configuration
        dict(name="append_f32", op="append", heads="tiny", dtype="f32", **_batch(decode=4, lo=16, hi=64, prefill="32@0", window=32, seq=64)),
        # a finetune sequence's pages for its backward pass
        dict(name="expand_8b_2048", op="expand", heads="8b", dtype="bf16", tokens=2048, spare=100),
        # a long sequence that moves to a pool in 16 bits
        dict(name="expand_14b_32749", op="expand", heads="14b", dtype="bf16", tokens=32749, spare=100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("decode", "decode", "long", "chunks", "mixed", "small", "append", "append", "expand"))
    heads = rng.choice(("8b", "14b", "8b", "14b", "mqa", "mha"))
    chunk = lambda most: "%d@%d" % (_log(rng, 2, most), rng.choice((0, rng.randint(1, 2000))))  # noqa: E731
    if op == "decode":
        lo = rng.randint(1, 500)
        return dict(op="attention", heads=heads, dtype="bf16", **_batch(decode=_log(rng, 1, 256), lo=lo, hi=rng.randint(lo, 4096)))
    if op == "long":
        return dict(op="attention", heads=heads, dtype="bf16", **_batch(decode=rng.randint(1, 6), lo=_log(rng, 3000, 12000), hi=rng.randint(12000, 32000)))
    if op == "chunks":
        window = rng.choice((0, _log(rng, 16, 700)))
        return dict(op="attention", heads=heads, dtype="bf16", **_batch(prefill=" ".join(chunk(800) for _ in range(rng.randint(1, 3))), window=window, seq=window + rng.randint(0, 3000)))
    if op == "mixed":
        return dict(op="attention", heads=heads, dtype="bf16", **_batch(decode=_log(rng, 8, 250), lo=16, hi=4096, median=rng.randint(200, 1000), sigma=0.8, prefill=chunk(500), window=_log(rng, 16, 400), seq=rng.randint(500, 3000)))
    if op == "small":
        window = _log(rng, 1, 100)
        return dict(op=rng.choice(("attention", "append")), heads="tiny", dtype="f32", **_batch(decode=_log(rng, 1, 20), lo=1, hi=rng.randint(20, 300), prefill=chunk(130).split("@")[0] + "@0", window=window, seq=window + rng.randint(0, 200)))
    if op == "append":
        return dict(op="append", heads=heads, dtype="bf16", **_batch(decode=_log(rng, 1, 500), lo=1, hi=rng.randint(30, 400), prefill=" ".join(chunk(1000) for _ in range(rng.randint(0, 2))), window=_log(rng, 1, 900), seq=rng.randint(901, 2000)))
    return dict(op="expand", heads=heads, dtype=rng.choice(("bf16", "bf16", "f32")), tokens=_log(rng, 1, 16384), spare=rng.randint(0, 50))


def _lengths(case):
    """context length of each decode request, the new token included"""
    n, out = case["decode"], []
    for i in range(n):
        u = (i + 0.5) / n
        if case["median"]:
            z = math.sqrt(2.0) * float(torch.erfinv(torch.tensor(2 * u - 1, dtype=torch.float64)))
            c = case["median"] * math.exp(case["sigma"] * z)
        else:
            c = case["lo"] + u * (case["hi"] + 1 - case["lo"])
        out.append(max(1, min(case["hi"], max(case["lo"], int(c)))))
    return out


def _requests(case):
    """[(kind, first position, new tokens, tokens the sequence's pages hold)]; kinds: 0 decode, 1 prefill, 2 finetune"""
    reqs = [(0, n - 1, 1, n) for n in _lengths(case)]
    for p in case["prefill"].split():
        n, start = (int(v) for v in p.split("@"))
        reqs.append((1, start, n, start + n))
    if case["window"]:
        reqs.append((2, case["seq"] - case["window"], case["window"], case["seq"]))
    return reqs


def work(case):
    nq, nkv, d, _ = _HEADS[case["heads"]]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "expand":
        pages = -(-case["tokens"] // PAGE)
        return {"bytes": pages * nkv * (2 * d * PAGE * (1 + e) + 8), "flops": 2 * pages * nkv * d * PAGE}
    reqs = _requests(case)
    T = sum(r[2] for r in reqs)
    if case["op"] == "append":
        runs = sum((r[1] + r[2] - 1) // PAGE - r[1] // PAGE + 1 for r in reqs)
        return {"bytes": T * (nq + 2 * nkv) * d * e + T * nq * d * e + 2 * T * nkv * d + 16 * runs * nkv, "flops": 3 * T * (nq + nkv) * d + 2 * T * nkv * d}
    seen = sum(r[1] + r[2] for r in reqs)
    pages = sum(-(-(r[1] + r[2]) // PAGE) for r in reqs)
    pairs = sum(r[1] * r[2] + r[2] * (r[2] + 1) // 2 for r in reqs)
    return {"bytes": 2 * seen * nkv * d + 8 * pages * nkv + 2 * T * nq * d * e + 4 * T * nq, "flops": 4 * pairs * nq * d}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _inputs(case, seed):
    """what the call reads, as torch tensors on the GPU"""
    nq, nkv, d, theta = _HEADS[case["heads"]]
    g = torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1))
    order = torch.Generator().manual_seed(seed + 77)
    st = SimpleNamespace(op=case["op"], nq=nq, nkv=nkv, d=d, theta=theta, dtype=_DTYPE[case["dtype"]], f32=case["dtype"] == "f32")
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    if case["op"] == "expand":
        counts = [-(-case["tokens"] // PAGE)]
        extra = case["spare"]
    else:
        st.reqs = _requests(case)
        counts = [-(-r[3] // PAGE) for r in st.reqs]
        extra = 3
    st.num_pages = sum(counts) + extra
    # the pages of all sequences, scattered over the pool
    ids = torch.randperm(st.num_pages, generator=order)
    st.pages, at = [], 0
    for n in counts:
        st.pages.append(ids[at:at + n])
        at += n
    # cached rows: keys have a few loud channels, as rotated keys do; every slot holds something, also those behind a
    # sequence's end (a page's last owner left it there)
    st.k_codes = torch.empty((st.num_pages, nkv, d // 16, PAGE, 16), dtype=torch.uint8, device="cuda")
    st.v_codes = torch.empty((st.num_pages, nkv, d, PAGE), dtype=torch.uint8, device="cuda")
    st.k_scale = torch.empty((st.num_pages, nkv), device="cuda")
    st.v_scale = torch.empty_like(st.k_scale)
    k_gain, v_gain = (0.5 * normal(nkv, d, 1)).exp_(), (0.3 * normal(nkv, d, 1)).exp_()
    step = max(1, (1 << 27) // (nkv * d * PAGE))
    for o in range(0, st.num_pages, step):
        n = min(step, st.num_pages - o)
        for gain, codes, scale, keys in ((k_gain, st.k_codes, st.k_scale, True), (v_gain, st.v_codes, st.v_scale, False)):
            x = normal(n, nkv, d, PAGE).mul_(gain)
            s = _scale_of(x.abs().amax((2, 3)))
            c = (x / s[:, :, None, None]).to(E4M3).view(torch.uint8)
            codes[o:o + n] = c.view(n, nkv, d // 16, 16, PAGE).transpose(3, 4) if keys else c
            scale[o:o + n] = s
    if case["op"] == "expand":
        st.tokens = case["tokens"]
        st.src = st.pages[0].to(torch.int32).cuda()
        st.dst = torch.randperm(counts[0], generator=order).to(torch.int32).cuda()
        st.out_k = torch.zeros((counts[0], nkv, PAGE, d), dtype=st.dtype, device="cuda")
        st.out_v = torch.zeros((counts[0], nkv, d, PAGE), dtype=st.dtype, device="cuda")
        return st
    st.T = sum(r[2] for r in st.reqs)
    st.pos = torch.cat([torch.arange(r[1], r[1] + r[2]) for r in st.reqs]).cuda()
    if case["op"] == "attention":
        st.q = (1.5 * normal(st.T, nq * d)).to(st.dtype)
    else:
        x = normal(st.T, (nq + 2 * nkv) * d)
        x[:, nq * d:(nq + nkv) * d].view(st.T, nkv, d).mul_(1.3 * k_gain[:, :, 0])
        x[:, (nq + nkv) * d:].view(st.T, nkv, d).mul_(1.3 * v_gain[:, :, 0])
        st.qkv = x.to(st.dtype)
    return st


def _scale_of(amax):
    """least power of two s with amax / s <= 448"""
    m, x = torch.frexp(amax)                                  # amax = m 2^x, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, x - 9, x - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, LEAST_EXP)).clamp(min=LEAST_EXP)
    return ((e.int() + 127) << 23).view(torch.float32)        # 2^e


def _pad(rows, fill):
    w = max(len(r) for r in rows)
    out = torch.full((len(rows), w), fill, dtype=torch.int64)
    for i, r in enumerate(rows):
        out[i, :len(r)] = r
    return out.cuda()


def _runs(st):
    """the batch's tokens by the page they are written to: [(first token, tokens, page, first position in the page)]"""
    out, at = [], 0
    for r, pages in zip(st.reqs, st.pages):
        p = r[1]
        while p < r[1] + r[2]:
            n = min(PAGE - p % PAGE, r[1] + r[2] - p)
            out.append((at, n, int(pages[p // PAGE]), p % PAGE))
            at += n
            p += n
    return out


def prepare(case, seed):
    st = _inputs(case, seed)
    if st.op == "attention":
        # the requests' tokens and pages as padded tables: one table for single tokens, one for chunks
        first, at = [], 0
        for r in st.reqs:
            first.append(at)
            at += r[2]
        st.groups = []
        for single in (True, False):
            of = [i for i, r in enumerate(st.reqs) if (r[2] == 1) == single]
            if of:
                need = [-(-(st.reqs[i][1] + st.reqs[i][2]) // PAGE) for i in of]
                st.groups.append((_pad([st.pages[i][:n] for i, n in zip(of, need)], 0),
                                  _pad([torch.arange(first[i], first[i] + st.reqs[i][2]) for i in of], -1),
                                  torch.tensor([st.reqs[i][1] for i in of]).cuda()))
        st.out = torch.empty((st.T, st.nq * st.d), dtype=st.dtype, device="cuda")
        st.lse = torch.empty((st.T, st.nq), device="cuda")
    elif st.op == "append":
        runs = _runs(st)
        st.run_tok = _pad([torch.arange(t, t + n) for t, n, _, _ in runs], -1)
        st.run_tok = torch.nn.functional.pad(st.run_tok, (0, PAGE - st.run_tok.shape[1]), value=-1)
        st.run_page = torch.tensor([r[2] for r in runs]).cuda()
        st.run_at = torch.tensor([r[3] for r in runs]).cuda()
        st.q_out = torch.empty((st.T, st.nq * st.d), dtype=st.dtype, device="cuda")
    if own:
        _own_plan(st)          # a server's index maps of the batch, workspace and handles: the same for every layer of a model
    return st


# ---- the plain form -------------------------------------------------------------------------------------------------

def _rows(codes, scale, pages, keys):
    """fp32 cached rows of the padded page table: keys [R, kv heads, head_dim, positions], values [.., positions, head_dim]"""
    R, P = pages.shape
    x = codes[pages.view(-1)].view(E4M3).float() * scale[pages.view(-1)].view(R * P, -1, *(1,) * (codes.dim() - 2))
    if keys:           # [R P, h, d/16, PAGE, 16]
        return x.view(R, P, x.shape[1], -1, PAGE, 16).permute(0, 2, 3, 5, 1, 4).reshape(R, x.shape[1], -1, P * PAGE)
    return x.view(R, P, x.shape[1], -1, PAGE).permute(0, 2, 1, 4, 3).reshape(R, x.shape[1], P * PAGE, -1)


def _attend(st, pages, toks, start):
    """one padded table of requests: softmax over every row's own and earlier positions"""
    R, W = toks.shape
    g, there = st.nq // st.nkv, toks >= 0
    q = st.q[toks.clamp(min=0)].float().view(R, W, st.nkv, g, st.d).permute(0, 2, 3, 1, 4).reshape(R, st.nkv, g * W, st.d)
    s = torch.matmul(q, _rows(st.k_codes, st.k_scale, pages, True)).mul_(1.0 / math.sqrt(st.d)).view(R, st.nkv, g, W, -1)
    own_pos = start[:, None] + torch.arange(W, device="cuda")
    later = torch.arange(s.shape[-1], device="cuda") > own_pos[:, :, None]
    s.masked_fill_(later[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(R, st.nkv, g * W, -1), _rows(st.v_codes, st.v_scale, pages, False)).view(R, st.nkv, g, W, st.d) / l
    st.out[toks[there]] = o.permute(0, 3, 1, 2, 4).reshape(R, W, -1)[there].to(st.dtype)
    st.lse[toks[there]] = (m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(R, W, -1)[there]


def _turn(x, pos, theta):
    """rotation of the pairs (i, i + d/2) by pos * theta^(-2 i / d); angles in 64 bits"""
    half = x.shape[-1] // 2
    f = theta ** (-torch.arange(half, dtype=torch.float64, device=x.device) * 2 / x.shape[-1])
    a = pos.double()[:, None] * f
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    p, q = x[..., :half], x[..., half:]
    return torch.cat((p * cos - q * sin, q * cos + p * sin), -1)


def _store(st, x, codes, scale, keys):
    """rows x [T, kv heads, head_dim] into the cache"""
    there = st.run_tok >= 0
    rows = x[st.run_tok.clamp(min=0)] * there[:, :, None, None]                       # [runs, PAGE, h, d]
    old = scale[st.run_page]
    new = _scale_of(rows.abs().amax((1, 3)))
    new = torch.where(st.run_at[:, None] == 0, new, torch.maximum(new, old))
    # slot by slot of the page: a new row, or what was there at the new scale
    slot = torch.arange(PAGE, device="cuda")[None] - st.run_at[:, None]
    from_new = (slot >= 0) & (slot < there.sum(1, keepdim=True))
    rows = torch.gather(rows, 1, slot.clamp(0, PAGE - 1)[:, :, None, None].expand_as(rows)).permute(0, 2, 3, 1) / new[:, :, None, None]
    now = codes[st.run_page]
    if keys:
        now = now.transpose(3, 4).reshape(rows.shape)
    kept = torch.where((st.run_at == 0)[:, None], torch.ones_like(old), old / new)[:, :, None, None]
    c = torch.where(from_new[:, None, None], rows, now.view(E4M3).float() * kept).to(E4M3).view(torch.uint8)
    codes[st.run_page] = c.view(*c.shape[:2], -1, 16, PAGE).transpose(3, 4) if keys else c
    scale[st.run_page] = new


def run(st):
    if own:
        return _own_run(st)
    if st.op == "attention":
        for table in st.groups:
            _attend(st, *table)
        return {"out": st.out, "lse": st.lse}
    if st.op == "append":
        nq, nkv, d = st.nq, st.nkv, st.d
        x = st.qkv.float().view(st.T, nq + 2 * nkv, d)
        turned = _turn(x[:, :nq + nkv], st.pos, st.theta)
        st.q_out.copy_(turned[:, :nq].reshape(st.T, -1))
        _store(st, turned[:, nq:], st.k_codes, st.k_scale, True)
        _store(st, x[:, nq + nkv:], st.v_codes, st.v_scale, False)
        return {"q": st.q_out, "k": st.k_codes.view(E4M3), "v": st.v_codes.view(E4M3), "k_scale": st.k_scale, "v_scale": st.v_scale}
    src, dst = st.src.long(), st.dst.long()
    there = (torch.arange(len(src) * PAGE, device="cuda") < st.tokens).view(-1, 1, PAGE)
    x = st.k_codes[src].view(E4M3).float() * st.k_scale[src][:, :, None, None, None]
    x = x.transpose(2, 3).reshape(len(src), st.nkv, PAGE, st.d)
    st.out_k[dst] = torch.where(there[..., None], x, torch.zeros_like(x)).to(st.dtype)
    x = st.v_codes[src].view(E4M3).float() * st.v_scale[src][:, :, None, None]
    st.out_v[dst] = torch.where(there[:, :, None], x, torch.zeros_like(x)).to(st.dtype)
    return {"k": st.out_k, "v": st.out_v}


# ---- the package's calls --------------------------------------------------------------------------------------------

def _own_plan(st):
    from paper_2402_18789_amd import binding as B
    from paper_2402_18789_amd import host as HH
    from paper_2402_18789_amd import kv8

    st.kv8 = kv8
    st.cfg = B.LayerCfg(st.nq * st.d, st.nq, st.nkv, st.d, 256, B.FLEXCO_F32 if st.f32 else B.FLEXCO_BF16, PAGE, 0, 0, 1e-5, st.theta, 1.0)
    st.pool = kv8.Pool(st.k_codes.data_ptr(), st.v_codes.data_ptr(), st.k_scale.data_ptr(), st.v_scale.data_ptr(), st.num_pages, PAGE)
    if st.op == "expand":
        st.wide = B.KVPool(st.out_k.data_ptr(), st.out_v.data_ptr(), st.out_k.shape[0], PAGE)
        return
    reqs = [SimpleNamespace(kind=r[0], start_pos=r[1], n_new=r[2], adapter=-1, seq_id=i) for i, r in enumerate(st.reqs)]
    shape = SimpleNamespace(page_size=PAGE, n_q_heads=st.nq, n_kv_heads=st.nkv)
    st.batch = kv8.DeviceBatch8(shape, reqs, [p.numpy() for p in st.pages], st.num_pages)
    if st.op == "attention":
        st.ws = HH.Workspace(st.cfg, st.T, st.batch.host_maps.n_parts)


def _own_run(st):
    if st.op == "attention":
        st.kv8.flexco_kv8_attention(st.cfg, st.batch.maps, st.q, st.pool, st.out, st.lse, st.ws.ptr, st.ws.bytes)
        return {"out": st.out, "lse": st.lse}
    if st.op == "append":
        st.kv8.flexco_kv8_append(st.cfg, st.batch.maps, st.batch.runs, st.batch.n_runs, st.qkv, st.pool, st.q_out, st.nq * st.d)
        return {"q": st.q_out, "k": st.k_codes.view(E4M3), "v": st.v_codes.view(E4M3), "k_scale": st.k_scale, "v_scale": st.v_scale}
    st.kv8.flexco_kv8_expand(st.cfg, st.pool, st.src, st.tokens, st.wide, st.dst)
    return {"k": st.out_k, "v": st.out_v}


# ---- the same in 64 bits, request by request ------------------------------------------------------------------------

def _cached64(st, i, n):
    """the first n cached key / value rows of sequence i, [kv heads, n, head_dim]"""
    p = st.pages[i][: -(-n // PAGE)].cuda()
    k = st.k_codes[p].view(E4M3).double() * st.k_scale[p].double()[:, :, None, None, None]
    v = st.v_codes[p].view(E4M3).double() * st.v_scale[p].double()[:, :, None, None]
    k = k.permute(1, 0, 3, 2, 4).reshape(st.nkv, -1, st.d)
    v = v.permute(1, 0, 3, 2).reshape(st.nkv, -1, st.d)
    return k[:, :n].contiguous(), v[:, :n].contiguous()


def _power64(amax):
    """the scale's definition by trial: no smaller power of two keeps amax within 448"""
    s = 2.0 ** torch.ceil(torch.log2(amax.clamp(min=1e-300) / LARGEST))
    s = torch.where(amax / s > LARGEST, 2 * s, s)
    s = torch.where(amax / (s / 2) <= LARGEST, s / 2, s)
    return s.clamp(min=2.0 ** LEAST_EXP)


def exact(case, seed):
    st = _inputs(case, seed)
    if st.op == "expand":
        k, v = _cached64(st, 0, PAGE * len(st.pages[0]))
        k[:, st.tokens:], v[:, st.tokens:] = 0.0, 0.0
        dst = st.dst.long()
        out_k = torch.empty(st.out_k.shape, dtype=torch.float64, device="cuda")
        out_v = torch.empty(st.out_v.shape, dtype=torch.float64, device="cuda")
        out_k[dst] = k.view(st.nkv, -1, PAGE, st.d).transpose(0, 1)
        out_v[dst] = v.view(st.nkv, -1, PAGE, st.d).permute(1, 0, 3, 2)
        return {"k": out_k, "v": out_v}
    if st.op == "attention":
        out = torch.empty((st.T, st.nq * st.d), dtype=torch.float64, device="cuda")
        lse = torch.empty((st.T, st.nq), dtype=torch.float64, device="cuda")
        g, at = st.nq // st.nkv, 0
        for i, (_, start, n, _) in enumerate(st.reqs):
            k, v = _cached64(st, i, start + n)
            q = st.q[at:at + n].double().view(n, st.nkv, g, st.d)
            for h in range(st.nkv):
                s = torch.matmul(q[:, h].reshape(n * g, st.d), k[h].T.contiguous()).view(n, g, -1) / math.sqrt(st.d)
                later = torch.arange(start + n, device="cuda")[None] > (start + torch.arange(n, device="cuda"))[:, None]
                s = s.masked_fill(later[:, None], -math.inf)
                z = torch.logsumexp(s, -1)
                lse[at:at + n, h * g:(h + 1) * g] = z
                o = torch.matmul(torch.exp(s - z[..., None]).view(n * g, -1), v[h])
                out[at:at + n, h * g * st.d:(h + 1) * g * st.d] = o.view(n, g * st.d)
            at += n
        return {"out": out, "lse": lse}
    half = st.d // 2
    x = st.qkv.double().view(st.T, -1, st.d)
    inv = torch.tensor([st.theta ** (-2.0 * i / st.d) for i in range(half)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), st.pos.double()[:, None] * inv)[:, None]
    z = torch.complex(x[:, :st.nq + st.nkv, :half].contiguous(), x[:, :st.nq + st.nkv, half:].contiguous()) * turn
    qk = torch.cat((z.real, z.imag), -1)
    new = {"k": qk[:, st.nq:], "v": x[:, st.nq + st.nkv:]}
    codes = {"k": st.k_codes.view(E4M3).double().transpose(2, 3).reshape(st.num_pages, st.nkv, PAGE, st.d),
             "v": st.v_codes.view(E4M3).double().transpose(2, 3).contiguous()}
    scale = {"k": st.k_scale.double(), "v": st.v_scale.double()}
    for t, n, page, at in _runs(st):
        for name in ("k", "v"):
            rows = new[name][t:t + n].transpose(0, 1)                             # [h, n, d]
            s = _power64(rows.abs().amax((1, 2)))
            if at:
                s = torch.maximum(s, scale[name][page])
                codes[name][page] = (codes[name][page] * (scale[name][page] / s)[:, None, None]).to(E4M3).double()
            codes[name][page, :, at:at + n] = (rows / s[:, None, None]).to(E4M3).double()
            scale[name][page] = s
    return {"q": qk[:, :st.nq].reshape(st.T, -1), "k": codes["k"].view(st.num_pages, st.nkv, PAGE, st.d // 16, 16).transpose(2, 3).contiguous(),
            "v": codes["v"].transpose(2, 3).contiguous(), "k_scale": scale["k"], "v_scale": scale["v"]}
