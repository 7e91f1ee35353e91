"""The operators of serving in 8 and 4 bits, as timed cases: each in its plain form (elementary torch operations in 32 bits) and,
with `own` set, through the library's calls.

Operators and kinds of cases
  cache    a GQA cache in 8 bits: E4M3 codes and, for each block of 16 tokens and KV head, one power-of-two scale for the keys and
           one for the values, the smallest that no entry of the block overflows
             decode   one decode iteration: append of the new token (rotated inside the step) and attention over the cached rows
             chunk    one prefill step over the next pieces of prompts whose earlier part is cached
             rows     a piece of a request's rows into its pages, and all its rows back (as a request migrates)
  norm     RMS norm with the residual's addition; output in bf16, or as MX E4M3: codes and a scale 2^e per 32 entries
  quant    the gate and up weights of a gated FFN as MXFP4 (E2M1 codes, a scale 2^e per 32 entries), and the values they stand for
  ffn      the gated FFN's first step: MX E4M3 rows by MXFP4 weights, silu(gate) * up
"""
import math
import random

import torch

own = False  # True: run() goes through the library

# q heads, KV heads, head dim
LAYERS = {"tiny": (8, 8, 64), "8b": (32, 8, 128), "70b": (64, 8, 128)}
# hidden, inter: a small layer, the 8B layer, a tensor-parallel quarter of the 70B one
FFNS = {"small": (1024, 2816), "8b": (4096, 14336), "70b/4": (8192, 7168)}
PAGE = 16
THETA = 500000.0
EPS = 1e-5
# prefill / decode CUs
SPLITS = ((64, 192), (96, 160), (128, 128), (160, 96), (192, 64), (256, 256))
MOST_FLOPS, MOST_BYTES = 1.95e12, 1.0e9  # a drawn case costs no more than the largest listed one


def listed():
    return [
        # a handful of chat users on the whole chip: launches and host work are most of an iteration
        dict(name="decode_few", kind="decode", layer="8b", n=4, lo=100, hi=1500, dist="uniform", rope=True, prefill_cus=256, decode_cus=256, len_seed=1),
        # the headline decode batch on half the chip
        dict(name="decode_8b", kind="decode", layer="8b", n=64, lo=512, hi=4096, dist="uniform", rope=True, prefill_cus=128, decode_cus=128, len_seed=1001),
        # a full decode batch with the long-tailed contexts of real traffic
        dict(name="decode_70b", kind="decode", layer="70b", n=128, lo=2000, hi=8192, dist="lognormal", rope=True, prefill_cus=128, decode_cus=128, len_seed=1002),
        # chunked prefill: ragged pieces behind cached prefixes
        dict(name="chunk_8b", kind="chunk", layer="8b", n=4, lo=201, hi=1024, dist="uniform", pre_hi=7680, rope=True, prefill_cus=128, decode_cus=128, len_seed=7),
        # a long request's last piece comes in and the request moves on; the piece begins inside a block
        dict(name="rows_8b", kind="rows", layer="8b", n=16001, start=7003, prefill_cus=128, decode_cus=128),
        # behind attention in a decode iteration of a few users
        dict(name="norm_few", kind="norm", n=3, hidden=4096, mx=False, prefill_cus=256, decode_cus=256),
        # ahead of the FFN of a prompt batch
        dict(name="norm_prompt", kind="norm", n=8192, hidden=4096, mx=True, prefill_cus=128, decode_cus=128),
        # a layer's weights at load time: a small layer, and the 8B one
        dict(name="quant_small", kind="quant", ffn="small", prefill_cus=256, decode_cus=256),
        dict(name="quant_8b", kind="quant", ffn="8b", prefill_cus=256, decode_cus=256),
        # gated FFN behind one user's token on the whole chip, a decode batch, and a prompt batch
        dict(name="ffn_token", kind="ffn", ffn="8b", n=1, prefill_cus=256, decode_cus=256, phase="decode"),
        dict(name="ffn_decode", kind="ffn", ffn="8b", n=64, prefill_cus=128, decode_cus=128, phase="decode"),
        dict(name="ffn_prompt", kind="ffn", ffn="8b", n=8192, prefill_cus=128, decode_cus=128, phase="prefill"),
    ]


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and (c["kind"] != "chunk" or _padded(c) <= 1.5e9):
            return c


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw(rng):
    kind = rng.choice(("decode", "decode", "chunk", "rows", "norm", "norm", "quant", "ffn", "ffn"))
    p, d = rng.choice(SPLITS)
    c = dict(kind=kind, prefill_cus=p, decode_cus=d)
    if kind in ("decode", "chunk"):
        c.update(layer=rng.choice(tuple(LAYERS)), rope=rng.random() < 0.7, len_seed=rng.randrange(1 << 30))
        c.update(n=_log(rng, 1, 256 if kind == "decode" else 12), dist="uniform")
        most = 16384 if kind == "decode" else 2048
        a, b = _log(rng, 1, most), _log(rng, 1, most)
        c.update(lo=min(a, b), hi=max(a, b))
        if kind == "decode":
            c["dist"] = rng.choice(("uniform", "lognormal"))
        else:
            c["pre_hi"] = _log(rng, 1, 8192)
    elif kind == "rows":
        c.update(layer=rng.choice(tuple(LAYERS)), n=_log(rng, 1, 65536))
        c["start"] = rng.randrange(c["n"]) if rng.random() < 0.7 else 0
    elif kind == "norm":
        c.update(n=_log(rng, 1, 16384), mx=rng.random() < 0.6)
        c["hidden"] = 128 * _log(rng, 1, 128) if c["mx"] else 8 * _log(rng, 1, 2048)
    elif kind == "quant":
        c.update(hidden=128 * _log(rng, 1, 64), inter=128 * _log(rng, 1, 112))
    else:
        c.update(n=_log(rng, 1, 8192), phase=rng.choice(("prefill", "decode")))
        if rng.random() < 0.5:
            c["ffn"] = rng.choice(tuple(FFNS))
        else:
            c.update(hidden=128 * _log(rng, 1, 64), inter=128 * _log(rng, 1, 112))
    return c


# --------------------------------------------------------------------------- lengths and work
def _lengths(n, lo, hi, dist, seed):
    """n lengths: uniform in lo .. hi, or lognormal (median lo, sigma 0.8) capped at hi."""
    r = random.Random(seed)
    if dist == "uniform":
        return [r.randint(lo, hi) for _ in range(n)]
    return [min(hi, max(1, round(math.exp(r.gauss(math.log(lo), 0.8))))) for _ in range(n)]


def _new_lengths(c):
    return _lengths(c["n"], c["lo"], c["hi"], c["dist"], c["len_seed"])


def _prefixes(c):
    """Cached tokens of each request of a chunk case; the first of several has none, and one at least has some."""
    pre = [0 if i == 0 and c["n"] > 1 else x for i, x in enumerate(_lengths(c["n"], 0, c["pre_hi"], "uniform", c["len_seed"] + 2))]
    pre[-1] = max(1, pre[-1])
    return pre


def _shape(c):
    return FFNS[c["ffn"]] if "ffn" in c else (c["hidden"], c["inter"])


def _padded(c):
    """Scores of a chunk case with all requests as long as the longest."""
    new, pre = _new_lengths(c), _prefixes(c)
    return c["n"] * LAYERS[c["layer"]][0] * max(new) * max(a + b for a, b in zip(new, pre))


def _token_bytes(Hkv, d):
    """A cached token's codes and its share of the scales."""
    return Hkv * (2 * d + 2 / 16)


def work(case):
    c = case
    if c["kind"] == "norm":
        out = 1 + 1 / 32 if c["mx"] else 2
        return {"bytes": c["n"] * c["hidden"] * (6 + out) + 2 * c["hidden"], "flops": 6.0 * c["n"] * c["hidden"]}
    if c["kind"] in ("quant", "ffn"):
        hidden, inter = _shape(c)
        packed = 2 * hidden * inter * 17 / 32
        if c["kind"] == "quant":
            return {"bytes": 8 * hidden * inter + packed, "flops": 8.0 * hidden * inter}
        return {"bytes": packed + c["n"] * (hidden * 33 / 32 + 2 * inter), "flops": 4.0 * c["n"] * hidden * inter}
    H, Hkv, d = LAYERS[c["layer"]]
    row = _token_bytes(Hkv, d)
    if c["kind"] == "rows":
        return {"bytes": (c["n"] - c["start"]) * (4 * Hkv * d + row) + c["n"] * (row + 4 * Hkv * d), "flops": 4.0 * c["n"] * Hkv * d}
    new = _new_lengths(c)
    if c["kind"] == "decode":
        return {"bytes": sum(new) * row + c["n"] * (4 * H * d + 4 * Hkv * d + row), "flops": 4.0 * H * d * sum(new)}
    pre = _prefixes(c)
    pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, pre))
    T = sum(new)
    nbytes = T * (4 * H * d + 4 * Hkv * d + row) + sum(pre) * row + (T * 2 * (H + Hkv) * d if c["rope"] else 0)
    return {"bytes": nbytes, "flops": 4.0 * H * d * pairs}


# --------------------------------------------------------------------------- inputs
def _inputs(c, seed):
    """The tensors that a case begins with, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    def spread(*shape):
        """Magnitudes that differ from row to row, as activations' do."""
        return randn(*shape) * torch.exp2(torch.randn(shape[:-1] + (1,), generator=gen, device="cuda")).to(torch.bfloat16)

    kind = c["kind"]
    if kind == "norm":
        return dict(x=spread(c["n"], c["hidden"]), residual=spread(c["n"], c["hidden"]),
                    weight=(1 + 0.2 * torch.randn(c["hidden"], generator=gen, device="cuda")).to(torch.bfloat16))
    if kind in ("quant", "ffn"):
        hidden, inter = _shape(c)
        t = dict(gate=randn(inter, hidden).mul_(hidden ** -0.5), up=randn(inter, hidden).mul_(hidden ** -0.5))
        if kind == "ffn":
            t["x"] = spread(c["n"], hidden)
        return t
    H, Hkv, d = LAYERS[c["layer"]]
    if kind == "rows":
        return dict(k=spread(c["n"], Hkv, d), v=spread(c["n"], Hkv, d))
    new = _new_lengths(c)
    cached = sum(n - 1 for n in new) if kind == "decode" else sum(_prefixes(c))
    T = len(new) if kind == "decode" else sum(new)
    return dict(k_old=spread(cached, Hkv, d), v_old=spread(cached, Hkv, d), q=randn(T, H, d), k=spread(T, Hkv, d), v=spread(T, Hkv, d))


# --------------------------------------------------------------------------- plain forms: 8-bit blocks, MX blocks, rotation
def _exponent(amax, top, least=-126):
    """The smallest e >= least with amax <= top * 2^e."""
    m, e = torch.frexp(amax.double() / top)
    return torch.where(amax == 0, torch.full_like(e, least), torch.where(m == 0.5, e - 1, e)).clamp(min=least)


def _e4m3(x):
    """x (magnitudes up to 448) as E4M3 codes, nearest even."""
    return x.float().to(torch.float8_e4m3fn)


def _power(e):
    return torch.exp2(e.double())


def _mx8(y):
    """Rows [T, n] as E4M3 codes [T, n] and scales [n / 128, T, 4] (2^e per 32 entries)."""
    T, n = y.shape
    blocks = y.reshape(T, n // 32, 32)
    e = _exponent(blocks.abs().amax(-1), 448.0)
    codes = _e4m3(blocks.double() * _power(-e)[..., None]).reshape(T, n)
    scales = (e + 127).to(torch.uint8).reshape(T, n // 128, 4).permute(1, 0, 2).contiguous()
    return codes, scales.view(torch.float8_e8m0fnu)


def _mx8_values(codes, scales):
    """The values [T, n] that _mx8's answer stands for, in 32 bits."""
    T, n = codes.shape
    return (codes.float().reshape(T, n // 32, 32) * scales.float().permute(1, 0, 2).reshape(T, n // 32, 1)).reshape(T, n)


def _mx4_values(w):
    """Rows [m, n] rounded to MXFP4: E2M1 multiples of 2^e, e per 32 entries."""
    blocks = w.float().reshape(w.shape[0], -1, 32)
    e = _exponent(blocks.abs().amax(-1), 6.0)[..., None]
    a = blocks * _power(-e).float()
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
    return (torch.round(a / step) * step * _power(e).float()).reshape(w.shape).to(torch.bfloat16)


def _rotate(x, pos):
    """Rows x [..., heads, d] at positions pos [...]: pairs (i, i + d / 2) turned by pos * theta^(-2 i / d); bf16."""
    half = x.shape[-1] // 2
    w = THETA ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    angle = (pos.double()[..., None] * w)[..., None, :]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)


def _cache_write(cache, blocks, slots, rows):
    """Rows [R, Hkv, d] into slots 0 .. 15 of the cache's blocks [R].  A block that is written from slot 0 on begins anew; otherwise the rows
    ahead of the first new one stay, under the larger of the two scales.  Rows behind the last new one are no longer there."""
    codes, exps = cache
    touched, at = torch.unique(blocks, return_inverse=True)
    n = touched.numel()
    wide = torch.zeros((n,) + codes.shape[1:], device=rows.device)
    wide[at, slots] = rows.float()
    first = torch.full((n,), 16, device=rows.device).scatter_reduce_(0, at, slots, "amin")
    kept = (torch.arange(16, device=rows.device) < first[:, None])[..., None, None]
    e_old = exps[touched]
    e = _exponent(wide.abs().amax((1, 3)), 448.0)
    e = torch.where(first[:, None] > 0, torch.maximum(e, e_old), e)
    old = codes[touched].float() * _power(e_old).float()[:, None, :, None]
    wide = torch.where(kept, old, wide)
    codes[touched] = _e4m3(wide * _power(-e).float()[:, None, :, None])
    exps[touched] = e


def _cache_rows(cache, table):
    """The rows [..., 16, Hkv, d] of blocks `table`, in 32 bits."""
    codes, exps = cache
    return codes[table].float() * _power(exps[table]).float()[..., None, :, None]


def _softmax_over(scores, seen):
    """Weights of the scores [.., keys] where `seen`; the others weigh nothing."""
    s = torch.where(seen, scores, torch.full_like(scores, -math.inf))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


# --------------------------------------------------------------------------- states
_context = None
_split = None


def _ctx(split):
    """The process's one context, with the partition `split` staged for the next steps if it is not the current one."""
    global _context, _split
    from paper_2504_19867_amd import semipd as S
    if _context is None:
        _context = S.Context(0)
    if _split != split:
        _context.set_partition(*split)
        _split = split
    return _context


class State:
    """What a worker keeps between calls: its pool with the live requests, laid-out weights, the tensors of the next call."""

    def __init__(self, case):
        self.case, self.kind = case, case["kind"]
        self.split = (case["prefill_cus"], case["decode_cus"])
        self.pool = None

    def __del__(self):
        if self.pool is not None and _context is not None:
            _context.phase_sync(0)
            _context.phase_sync(1)
            self.pool.close()


def _own_pool(st, lens, rng):
    """A pool a quarter larger than `lens` need, its free list in random order as after long serving."""
    from paper_2504_19867_amd import semipd as S
    _, Hkv, d = LAYERS[st.case["layer"]]
    ctx = _ctx(st.split)
    pages = sum(-(-n // PAGE) for n in lens) * 5 // 4 + 16
    nbytes = S.pool_bytes(S.SPD_KV_GQA_FP8, PAGE, Hkv, d, d, pages)
    st.pool = S.Pool(ctx, torch.empty(nbytes, dtype=torch.uint8, device="cuda"), nbytes, S.SPD_KV_GQA_FP8, PAGE, Hkv, d, d, pages)
    ids = [(1 << 40) + i for i in range(pages)]
    for i in ids:
        st.pool.kv_reserve(i, 1)
    rng.shuffle(ids)
    for i in ids:
        st.pool.kv_free(i)


def _tables(st, lens, rng):
    """Block tables [n, blocks of the longest] of requests of `lens` tokens, over blocks in random order."""
    need = [-(-n // PAGE) for n in lens]
    order = list(range(sum(need)))
    rng.shuffle(order)
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [0] * (max(need) - n))
        at += n
    st.table = torch.tensor(table, device="cuda")
    _, Hkv, d = LAYERS[st.case["layer"]]
    st.caches = [(torch.zeros(at, PAGE, Hkv, d, device="cuda", dtype=torch.float8_e4m3fn), torch.full((at, Hkv), -126, device="cuda")) for _ in range(2)]


def _places(st, req, pos):
    """Blocks and slots of positions `pos` of the requests `req`."""
    return st.table[req, pos // PAGE], pos % PAGE


def _ragged(starts, lens):
    """Request and position of every row of pieces of `lens` rows from `starts` on."""
    lens_t = torch.tensor(lens, device="cuda")
    req = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens_t)
    ahead = torch.cumsum(lens_t, 0) - lens_t
    row = torch.arange(int(sum(lens)), device="cuda") - ahead[req]
    return req, row, torch.tensor(starts, device="cuda")[req] + row


def prepare(case, seed):
    c = case
    st = State(c)
    t = _inputs(c, seed)
    rng = random.Random(seed)
    st.__dict__.update({k: v for k, v in t.items() if k not in ("k_old", "v_old")})
    st.phase = 0 if c.get("phase", "decode") == "prefill" else 1
    if st.kind == "norm":
        st.out = torch.empty(c["n"], c["hidden"], device="cuda", dtype=torch.float8_e4m3fn if c["mx"] else torch.bfloat16)
        st.scales = torch.empty(c["hidden"] // 128, c["n"], 4, device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu) if c["mx"] else None
        st.ctx = _ctx(st.split) if own else None
    elif st.kind in ("quant", "ffn"):
        hidden, inter = _shape(c)
        st.hidden, st.inter = hidden, inter
        if st.kind == "ffn":
            st.x, st.scales = _mx8(st.x)
            st.out = torch.empty(c["n"], inter, device="cuda", dtype=torch.bfloat16)
        if own:
            from paper_2504_19867_amd import semipd as S
            st.ctx = _ctx(st.split)
            st.w = torch.empty(S.ffn_mx_bytes(hidden, inter), device="cuda", dtype=torch.uint8)
            if st.kind == "ffn":
                torch.cuda.synchronize()
                st.ctx.ffn_pack_gate_up_mx(st.phase, st.gate, st.up, st.w, hidden, inter)
                st.ctx.phase_sync(st.phase)
                st.gate = st.up = None
        elif st.kind == "ffn":
            st.gate, st.up = _mx4_values(st.gate), _mx4_values(st.up)
        if st.kind == "quant":
            st.gate_out, st.up_out = torch.empty_like(st.gate), torch.empty_like(st.up)
    else:
        _prepare_cache(st, t, rng)
    torch.cuda.synchronize()
    return st


def _prepare_cache(st, t, rng):
    c = st.case
    H, Hkv, d = LAYERS[c["layer"]]
    st.scale = d ** -0.5
    if st.kind == "rows":
        st.lens, st.pre = [c["n"]], [c["start"]]
        k_old, v_old = st.k[:c["start"]], st.v[:c["start"]]
        st.k_new, st.v_new = st.k[c["start"]:].clone(), st.v[c["start"]:].clone()
        st.k_out, st.v_out = torch.empty_like(st.k), torch.empty_like(st.v)
    else:
        new = _new_lengths(c)
        st.new = new
        if st.kind == "decode":
            st.lens, st.pre = new, [n - 1 for n in new]
        else:
            st.pre = _prefixes(c)
            st.lens = [n + p for n, p in zip(new, st.pre)]
            st.cu = [0]
            for n in new:
                st.cu.append(st.cu[-1] + n)
        k_old, v_old = t["k_old"], t["v_old"]
        st.out = torch.empty_like(st.q)
    st.ids = [1000 + i for i in range(len(st.lens))]
    if own:
        from paper_2504_19867_amd import semipd as S
        _own_pool(st, st.lens, rng)
        st.ctx = _ctx(st.split)
        st.rope = S.rope_config(theta=THETA, rotary_dim=d) if c.get("rope") else None
        torch.cuda.synchronize()
        at = 0
        for rid, n, p in zip(st.ids, st.lens, st.pre):
            st.pool.kv_reserve(rid, n)
            if p:
                st.pool.kv_write(1, rid, 0, p, k_old[at:at + p], v_old[at:at + p])
            at += p
        st.ctx.phase_sync(1)
        return
    _tables(st, st.lens, rng)
    if sum(st.pre):
        req, _, pos = _ragged([0] * len(st.pre), st.pre)
        for cache, rows in zip(st.caches, (k_old, v_old)):
            _cache_write(cache, *_places(st, req, pos), rows)
    st.n_all = torch.tensor(st.lens, device="cuda")
    if st.kind == "decode":
        st.at = (torch.arange(c["n"], device="cuda"), st.n_all - 1)
    else:
        st.req, st.row, st.pos = _ragged(st.pre, [n - p for n, p in zip(st.lens, st.pre)])
    st.key = torch.arange(st.table.shape[1] * PAGE, device="cuda")


# --------------------------------------------------------------------------- one pass
def run(st):
    return _run_own(st) if own else _RUN[st.kind](st)


def _run_own(st):
    c, ctx = st.case, _ctx(st.split)
    if st.kind == "norm":
        ctx.rmsnorm(st.phase, st.x, st.residual, st.weight, EPS, st.out, c["n"], c["hidden"], out_scales=st.scales)
        return {"out": st.out, "scales": st.scales, "residual": st.residual}
    if st.kind == "quant":
        ctx.ffn_pack_gate_up_mx(st.phase, st.gate, st.up, st.w, st.hidden, st.inter)
        ctx.ffn_unpack_gate_up_mx(st.phase, st.w, st.gate_out, st.up_out, st.hidden, st.inter)
        return {"gate": st.gate_out, "up": st.up_out}
    if st.kind == "ffn":
        ctx.ffn_gate_up_mx(st.phase, st.x, st.scales, st.w, st.out, c["n"], st.hidden, st.inter)
        return st.out
    if st.kind == "rows":
        st.pool.kv_write(1, st.ids[0], c["start"], c["n"] - c["start"], st.k_new, st.v_new)
        st.pool.kv_gather(1, st.ids[0], c["n"], st.k_out, st.v_out)
        return {"k": st.k_out, "v": st.v_out}
    H, Hkv, d = LAYERS[c["layer"]]
    if st.kind == "decode":
        st.pool.decode_step(st.ids, st.lens, st.q, st.out, H, st.scale, k_new=st.k, v_new=st.v, rope=st.rope)
        return st.out
    st.pool.prefill_step(st.ids, st.cu, st.q, st.k, st.v, st.out, H, Hkv, d, d, st.scale, prefix_lens=st.pre, rope=st.rope)
    return {"out": st.out, "q": st.q, "k": st.k}  # q, k rotated in place with RoPE


def _run_norm(st):
    st.residual = (st.x.float() + st.residual.float()).to(torch.bfloat16)
    h = st.residual.double()  # (in 64 bits: a code that lies next to a border goes by the last bits)
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * st.weight.double()
    if not st.case["mx"]:
        return {"out": y.to(torch.bfloat16), "scales": None, "residual": st.residual}
    codes, scales = _mx8(y.float())
    return {"out": codes, "scales": scales, "residual": st.residual}


def _run_quant(st):
    return {"gate": _mx4_values(st.gate), "up": _mx4_values(st.up)}


def _run_ffn(st):
    x = _mx8_values(st.x, st.scales)
    g, u = x @ st.gate.float().T, x @ st.up.float().T
    return (g / (1 + torch.exp(-g)) * u).to(torch.bfloat16)


def _run_rows(st):
    blocks, slots = _places(st, st.req, st.pos)
    got = []
    for cache, rows in zip(st.caches, (st.k_new, st.v_new)):
        _cache_write(cache, blocks, slots, rows)
        got.append(_cache_rows(cache, st.table[0]).flatten(0, 1)[:st.case["n"]].to(torch.bfloat16))
    return {"k": got[0], "v": got[1]}


def _run_decode(st):
    H, Hkv, d = LAYERS[st.case["layer"]]
    req, pos = st.at
    q, k = (_rotate(st.q, pos), _rotate(st.k, pos)) if st.case["rope"] else (st.q, st.k)
    blocks, slots = _places(st, req, pos)
    for cache, rows in zip(st.caches, (k, st.v)):
        _cache_write(cache, blocks, slots, rows)
    qs = q.float().reshape(-1, Hkv, H // Hkv, d)
    keys = _cache_rows(st.caches[0], st.table).flatten(1, 2).permute(0, 2, 3, 1)  # [n, Hkv, d, keys]
    p = _softmax_over(torch.matmul(qs, keys) * st.scale, (st.key < st.n_all[:, None])[:, None, None])
    del keys
    values = _cache_rows(st.caches[1], st.table).flatten(1, 2).transpose(1, 2)
    return torch.matmul(p, values).reshape(-1, H, d).to(torch.bfloat16)


def _run_chunk(st):
    H, Hkv, d = LAYERS[st.case["layer"]]
    if st.case["rope"]:
        st.q, st.k = _rotate(st.q, st.pos), _rotate(st.k, st.pos)
    blocks, slots = _places(st, st.req, st.pos)
    n, most = len(st.lens), max(st.new)
    wide = []
    for cache, rows in zip(st.caches, (st.k, st.v)):
        got = _cache_rows(cache, st.table).flatten(1, 2)  # [n, keys, Hkv, d]: the cached rows ...
        got[st.req, st.pos] = rows.float()  # ... and the pieces' own as they are given
        wide.append(got.transpose(1, 2))
        _cache_write(cache, blocks, slots, rows)
    q = torch.zeros(n, most, H, d, device="cuda")
    q[st.req, st.row] = st.q.float()
    q = q.reshape(n, most, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(n, Hkv, -1, d)
    pre = torch.tensor(st.pre, device="cuda")
    seen = st.key <= (pre[:, None] + torch.arange(most, device="cuda"))[..., None]  # [n, most, keys]
    seen = seen.repeat(1, H // Hkv, 1)[:, None]
    p = _softmax_over(torch.matmul(q, wide[0].transpose(-1, -2)) * st.scale, seen)
    o = torch.matmul(p, torch.where((st.key < st.n_all[:, None])[:, None, :, None], wide[1], torch.zeros((), device="cuda")))
    o = o.reshape(n, Hkv, H // Hkv, most, d).permute(0, 3, 1, 2, 4).reshape(n, most, H, d)
    return {"out": o[st.req, st.row].to(torch.bfloat16), "q": st.q, "k": st.k}


_RUN = {"norm": _run_norm, "quant": _run_quant, "ffn": _run_ffn, "rows": _run_rows, "decode": _run_decode, "chunk": _run_chunk}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _grid(bits_exp, bits_man, bias, top):
    """The values 0 .. top of a small floating-point format, in order."""
    got = []
    for e in range(1 << bits_exp):
        for m in range(1 << bits_man):
            got.append(math.ldexp(m, 1 - bias - bits_man) if e == 0 else math.ldexp((1 << bits_man) + m, e - bias - bits_man))
    return [v for v in got if v <= top]


def _nearest(x, grid):
    """x [..] to the nearest value of the grid, halfway to the one with the even number."""
    g = torch.tensor(grid, device=x.device, dtype=torch.float64)
    a = x.abs().clamp(max=grid[-1])
    hi = torch.searchsorted(g, a).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = g[hi] - a, a - g[lo]
    pick = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), g[lo], g[hi])
    return torch.copysign(pick, x)


def _block_scale(amax, top):
    """2^e [..] with the smallest e >= -126 that amax <= top 2^e allows, by counting."""
    e = torch.floor(torch.log2(amax.clamp(min=2.0 ** -140) / top)) - 1
    for _ in range(3):
        e = torch.where(amax > top * torch.exp2(e), e + 1, e)
    return torch.exp2(e.clamp(min=-126))


def _exact_block(rows, keep, scale_before):
    """One block's values after rows [16, Hkv, d] are in it: those from `keep` on are new."""
    E4M3 = _grid(4, 3, 7, 448.0)
    s = _block_scale(rows[keep:].abs().amax((0, 2)), 448.0)
    if keep:
        s = torch.maximum(s, scale_before)
    return _nearest(rows / s[:, None], E4M3) * s[:, None], s


def _exact_cache(rows, cuts):
    """The values that rows [n, Hkv, d] stand for, written in pieces that end at `cuts`; the dequantised rows."""
    E4M3 = _grid(4, 3, 7, 448.0)
    n, Hkv, d = rows.shape
    nb = -(-n // 16)
    pad = torch.zeros(nb * 16, Hkv, d, device=rows.device, dtype=torch.float64)
    pad[:n] = rows
    whole = pad.reshape(nb, 16, Hkv, d)
    out = torch.empty_like(whole)
    for at in range(0, nb, 4096):
        s = _block_scale(whole[at:at + 4096].abs().amax((1, 3)), 448.0)[:, None, :, None]
        out[at:at + 4096] = _nearest(whole[at:at + 4096] / s, E4M3) * s
    for cut in cuts:  # the block that a piece's end cuts is written twice
        if 0 < cut < n and cut % 16:
            b, t = cut // 16, cut % 16
            first = whole[b].clone()
            first[t:] = 0
            vals, s = _exact_block(first, 0, None)
            both = whole[b].clone()
            both[:t] = vals[:t]
            out[b], _ = _exact_block(both, t, s)
    return out.reshape(nb * 16, Hkv, d)[:n]


def _exact_rotate(x, pos):
    d = x.shape[-1]
    z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double())
    angle = pos.double()[:, None] * torch.exp(-math.log(THETA) * torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([z.real, z.imag], -1).to(torch.bfloat16)


def exact(case, seed):
    c = case
    t = _inputs(c, seed)
    if c["kind"] == "norm":
        h = (t["x"].double() + t["residual"].double()).to(torch.bfloat16)
        x = h.double()
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["hidden"] + EPS) * t["weight"].double()
        if not c["mx"]:
            return {"out": y, "scales": None, "residual": h.double()}
        s = _block_scale(y.reshape(c["n"], -1, 32).abs().amax(-1), 448.0)
        codes = torch.cat([_nearest(a / b[..., None], _grid(4, 3, 7, 448.0)) for a, b in zip(y.reshape(c["n"], -1, 32).split(512), s.split(512))])
        return {"out": codes.reshape(y.shape), "scales": s.reshape(c["n"], -1, 4).transpose(0, 1).contiguous(), "residual": h.double()}
    if c["kind"] in ("quant", "ffn"):
        w = []
        for name in ("gate", "up"):
            blocks = t[name].double().reshape(t[name].shape[0], -1, 32)
            s = _block_scale(blocks.abs().amax(-1), 6.0)[..., None]
            w.append(torch.cat([_nearest(a / b, _grid(2, 1, 1, 6.0)) * b for a, b in zip(blocks.split(1024), s.split(1024))]).reshape(t[name].shape))
        if c["kind"] == "quant":
            return {"gate": w[0], "up": w[1]}
        x = t["x"].double().reshape(c["n"], -1, 32)
        s = _block_scale(x.abs().amax(-1), 448.0)[..., None]
        x = torch.cat([_nearest(a / b, _grid(4, 3, 7, 448.0)) * b for a, b in zip(x.split(512), s.split(512))]).reshape(c["n"], -1)
        g, u = x @ w[0].T, x @ w[1].T
        return g * torch.sigmoid(g) * u
    H, Hkv, d = LAYERS[c["layer"]]
    if c["kind"] == "rows":
        return {"k": _exact_cache(t["k"].double(), [c["start"]]), "v": _exact_cache(t["v"].double(), [c["start"]])}
    new = _new_lengths(c)
    pre = [n - 1 for n in new] if c["kind"] == "decode" else _prefixes(c)
    count = [1] * len(new) if c["kind"] == "decode" else new
    pos = torch.cat([torch.arange(p, p + n, device="cuda") for p, n in zip(pre, count)])
    q, k = (_exact_rotate(t["q"], pos), _exact_rotate(t["k"], pos)) if c["rope"] else (t["q"], t["k"])
    outs, old, at = [], 0, 0
    for p, n in zip(pre, count):
        kk = torch.cat([t["k_old"][old:old + p], k[at:at + n]]).double()
        vv = torch.cat([t["v_old"][old:old + p], t["v"][at:at + n]]).double()
        if c["kind"] == "decode":
            kk, vv = _exact_cache(kk, [p]), _exact_cache(vv, [p])
        elif p:
            kk[:p], vv[:p] = _exact_cache(kk[:p], []), _exact_cache(vv[:p], [])
        qq = q[at:at + n].double().reshape(n, Hkv, H // Hkv, d)
        causal = torch.arange(p + n, device="cuda")[None] > torch.arange(p, p + n, device="cuda")[:, None]
        o = torch.empty(n, Hkv, H // Hkv, d, device="cuda", dtype=torch.float64)
        for h in range(Hkv):
            s = torch.einsum("ngd,kd->gnk", qq[:, h], kk[:, h]) * d ** -0.5
            o[:, h] = torch.matmul(torch.softmax(s.masked_fill(causal, -math.inf), -1), vv[:, h]).transpose(0, 1)
        outs.append(o.reshape(n, H, d))
        old, at = old + p, at + n
    out = torch.cat(outs)
    return out if c["kind"] == "decode" else {"out": out, "q": q.double(), "k": k.double()}
