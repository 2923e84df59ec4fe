"""The operators of a generation that follows several candidates on a small
cache, measured: scoring tokens, forking their cache pages, and a cache in 4
bits with the attention that reads it.

Kinds of case:

* ``score``   log probabilities of given tokens, the entropy of their rows and
              the rows' top alternatives (``spec_token_logprobs``)
* ``pages``   copies of cache pages in every layer of a pool: forks and
              compaction (``spec_op_kv_copy_pages``)
* ``append``  rotary embedding and the append of rows to a 4-bit cache, the
              rows read back (``spec_op_rope_kv4``, ``spec_op_kv4_read``)
* ``read``    cached rows back as values (``spec_op_kv4_read``)
* ``attn``    paged causal attention over a 4-bit cache (``spec_op_attention_kv4``)

Sizes are those of the configured models (``workloads/configs.py``).

The 4-bit cache holds a head's vector in blocks of 32 dims: values of
{0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign, and a power of two for each block,
the smallest that keeps 6 times it at or above the block's largest magnitude.
"""

import math

import numpy as np
import torch

from workloads import configs as C

own = False

MODELS = {"tiny": C.TINY_TARGET, "small": C.SMALL_TARGET, "1b": C.L1B_DRAFT, "8b": C.L8B_TARGET}
DEV = "cuda"


def listed():
    return [
        # the small pair's 8 sequences, one decoded token each, with the usual five alternatives: all latency
        {"name": "score_small", "kind": "score", "rows": 8, "vocab": 32000, "top": 5, "greedy": 0.0, "masked": 0.0, "coarse": False},
        # every verified row of a large batch (256 sequences x 7 rows), twenty alternatives each
        {"name": "score_stress", "kind": "score", "rows": 1792, "vocab": 128256, "top": 20, "greedy": 0.0, "masked": 0.0, "coarse": False},
        # a beam step of the small pair: each of 8 sequences gets its own copy of the partial last page
        {"name": "pages_fork_small", "kind": "pages", "model": "small", "layers": 12, "bits": 16, "pages": 512, "sources": 8, "copies": 1},
        # compaction of the serving batch's pool: a third of its pages moved (8 of the layers)
        {"name": "pages_compact_8b", "kind": "pages", "model": "8b", "layers": 8, "bits": 16, "pages": 6912, "sources": 2304, "copies": 1},
        # the rows of one sequence's verify
        {"name": "append_single", "kind": "append", "model": "8b", "rows": 6, "far": 2048},
        # a long prompt's prefill chunk
        {"name": "append_prefill", "kind": "append", "model": "8b", "rows": 8192, "far": 0},
        # a page of the small pair's cache back as values
        {"name": "read_small", "kind": "read", "model": "small", "rows": 16},
        # a 4096-token prefix of the 8B-shaped target
        {"name": "read_prefix", "kind": "read", "model": "8b", "rows": 4096},
        # the headline verify: one sequence, k = 5, context 2048
        {"name": "attn_single", "kind": "attn", "model": "8b", "batch": 1, "rows": 6, "lo": 2047, "hi": 2047},
        # the 64-sequence verify over contexts of 512 to 4096 tokens, k drawn from 3, 5, 7
        {"name": "attn_serving", "kind": "attn", "model": "8b", "batch": 64, "rows": 0, "lo": 512, "hi": 4096},
        # one token after a very long context
        {"name": "attn_long", "kind": "attn", "model": "8b", "batch": 1, "rows": 1, "lo": 131000, "hi": 131000},
        # an 8192-token prompt's prefill
        {"name": "attn_prefill", "kind": "attn", "model": "8b", "batch": 1, "rows": 8192, "lo": 0, "hi": 0},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["score", "score", "pages", "append", "read", "attn", "attn", "attn"])
    if kind == "score":
        return {"kind": "score", "rows": _log(rng, 1, 1700), "vocab": rng.choice([32000, 128256, _log(rng, 1000, 128256)]),
                "top": rng.choice([0, 1, 5, 20, rng.randint(1, 64)]), "greedy": rng.choice([0.0, 0.0, 0.25]),
                "masked": rng.choice([0.0, 0.0, 0.5, 0.995]), "coarse": rng.random() < 0.4}
    if kind == "pages":
        model = rng.choice(["tiny", "small", "1b", "8b"])
        pages = _log(rng, 32, 4096)
        sources = _log(rng, 1, pages // 2)
        return {"kind": "pages", "model": model, "layers": min(8, MODELS[model].n_layers), "bits": rng.choice([4, 16]), "pages": pages,
                "sources": sources, "copies": rng.randint(1, max(1, min(8, (pages - sources) // sources)))}
    if kind == "append":
        return {"kind": "append", "model": rng.choice(["tiny", "small", "1b", "8b"]), "rows": _log(rng, 1, 8000), "far": rng.choice([0, 500, 4096, 131072])}
    if kind == "read":
        return {"kind": "read", "model": rng.choice(["tiny", "small", "1b", "8b"]), "rows": _log(rng, 1, 8192)}
    model = rng.choice(["tiny", "small", "1b", "8b", "8b"])
    form = rng.choice(["verify", "verify", "long", "prefill"])
    if form == "verify":
        lo = _log(rng, 1, 4000)
        return {"kind": "attn", "model": model, "batch": _log(rng, 1, 64), "rows": rng.randint(0, 8), "lo": lo, "hi": _log(rng, lo, 4096)}
    if form == "long":
        lo = _log(rng, 8192, 120000)
        return {"kind": "attn", "model": model, "batch": rng.randint(1, 2), "rows": rng.randint(1, 6), "lo": lo, "hi": lo}
    lo = rng.choice([0, 0, rng.randint(1, 1000)])
    return {"kind": "attn", "model": model, "batch": rng.randint(1, 2), "rows": _log(rng, 16, 1024 if model == "tiny" else 3500), "lo": lo, "hi": lo}


# ---------------------------------------------------------------------------
# the 4-bit pages: for each of a (page, kv head) block's bytes, whose values it holds

def _block_bytes(hd):
    return 8 * hd + hd // 2


def _k_place(t, d, hd):
    """Byte and nibble of dim d of token t's key, and the byte of its block's scale."""
    s, g, i = d // 32, d // 8 % 4, d % 8
    h, j = t // 4 % 2, t % 4 + 4 * (t // 8)
    byte = ((h * 4 + g) * 8 + j) * 16 if hd == 128 else ((g * 8 + j) * 2 + h) * 8
    return byte + 4 * s + i // 2, i % 2, 8 * hd + (j * 2 + h) * (hd // 32) + s


def _v_place(t, d, hd):
    """The same of its value vector."""
    b, i = d // 32, d % 32
    byte = ((b // 2 * 2 + t // 8) * 16 + i % 16) * 16 + b % 2 * 8 + t % 8
    return byte, i // 16, 8 * hd + (t // 8 * (hd // 32) + b) * 8 + t % 8


def _tables(place, hd):
    """[16, hd] bytes, nibbles and scale bytes on the GPU."""
    got = np.array([[place(t, d, hd) for d in range(hd)] for t in range(16)], dtype=np.int64)
    return [torch.from_numpy(np.ascontiguousarray(got[:, :, i])).to(DEV) for i in range(3)]


def _exponents(x):
    """Exponent (biased by 127) of each block of 32 of x's last dim, repeated over the block."""
    m = x.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True)
    e = torch.frexp(m)[1]  # m = f 2^e with 0.5 <= f < 1, and the largest value held is 0.75 x 2^3
    e = torch.where(m > torch.ldexp(torch.full_like(m, 0.75), e), e - 2, e - 3)
    return (e.clamp(min=-126) + 127).expand(*m.shape[:-1], 32).flatten(-2)


def _codes(x, e):
    """4-bit codes of x with the exponents e: the nearest value, of two as near the one with an even code."""
    a = torch.ldexp(x, 127 - e).abs()
    n = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    return n + 8 * (x < 0)


def _numbers(codes, e):
    lut = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    return torch.ldexp(lut[codes.long()], e - 127)


def _pack(x, place):
    """Pages [P, Hkv, block bytes] that hold the vectors x fp32 [P, 16, Hkv, hd]."""
    hd = x.shape[-1]
    byte, nibble, scale = _tables(place, hd)
    e = _exponents(x)
    codes = (_codes(x, e).to(torch.uint8)).movedim(2, 1).flatten(2)  # [P, Hkv, 16 hd]
    pages = torch.empty(x.shape[0], x.shape[2], _block_bytes(hd), dtype=torch.uint8, device=DEV)
    order = torch.argsort((byte * 2 + nibble).flatten())  # values in the order of the bytes, low nibbles first
    codes = codes[:, :, order]
    pages[:, :, :8 * hd] = codes[:, :, 0::2] | (codes[:, :, 1::2] << 4)
    pages[:, :, scale.flatten()] = e.to(torch.uint8).movedim(2, 1).flatten(2)
    return pages


def _unpack(pages, page, token, tables):
    """fp32 vectors [..., Hkv, hd] of the tokens `token` of the pages `page` (index tensors of one shape)."""
    byte, nibble, scale = (t[token].unsqueeze(-2) for t in tables)
    head = torch.arange(pages.shape[1], device=DEV).unsqueeze(-1)
    page = page[..., None, None]
    codes = (pages[page, head, byte] >> (4 * nibble).to(torch.uint8)) & 15
    return _numbers(codes, pages[page, head, scale].int())


# ---------------------------------------------------------------------------
# inputs

def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_033 + tag)
    return g


def _dtype(sh):
    return torch.float32 if sh.dtype == "f32" else torch.bfloat16


def _vectors(n, sh, g, keys):
    """n tokens' keys or values [n, Hkv, hd]; a few of a key's dims are much larger than the others."""
    x = torch.randn(n, sh.n_kv_heads, sh.head_dim, generator=g, device=DEV)
    if keys:
        x = x * torch.where(torch.arange(sh.head_dim, device=DEV) % 17 == 3, 4.0, 1.0)
    return x


def _pages(n, sh, g):
    """n K and n V pages of one layer."""
    return [_pack(_vectors(16 * n, sh, g, p is _k_place).unflatten(0, (n, 16)), p) for p in (_k_place, _v_place)]


def _segments(case):
    """Rows of each sequence and the position of the first."""
    n, lo, hi = case["batch"], case["lo"], case["hi"]
    pos0 = [int(lo * (hi / lo) ** ((i + 0.5) / n)) if lo else 0 for i in range(n)]
    return [case["rows"] or (4, 6, 8)[i % 3] for i in range(n)], pos0


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    kind = case["kind"]
    g = _gen(seed, 1)
    rng = np.random.default_rng([int(seed) & 0x7FFFFFFF, 21])
    if kind == "score":
        R, V = case["rows"], case["vocab"]
        s.logits = torch.randn(R, V, generator=g, device=DEV) * 3.0
        if case["coarse"]:  # logits of a low-precision head: many are equal
            s.logits = torch.round(s.logits * 8) / 8
        tokens = rng.integers(0, V, R).astype(np.int32)
        tokens[::3] = s.logits[::3].argmax(1).int().cpu().numpy()  # what was drawn is often likely
        if case["masked"]:  # a grammar's mask; now and then it leaves a row nothing, or no token is asked for
            for r in range(0, R, 64):
                part = s.logits[r:r + 64]
                part[torch.rand(part.shape, generator=g, device=DEV) < case["masked"]] = -math.inf
            s.logits[11::97] = -math.inf
            tokens[5::31] = -1
        temps = np.array([0.0 if rng.uniform() < case["greedy"] else (0.3, 1.0, 1.5)[i % 3] for i in range(R)], dtype=np.float32)
        s.tokens, s.temps = torch.from_numpy(tokens).to(DEV), torch.from_numpy(temps).to(DEV)
    elif kind == "pages":
        sh = MODELS[case["model"]]
        s.page = sh.n_kv_heads * _block_bytes(sh.head_dim) if case["bits"] == 4 else sh.kv_dim * 16 * sh.bytes_per_elem()
        planes, P, n = 2 * case["layers"], case["pages"], case["sources"]
        s.pool = torch.empty(planes, P, s.page, dtype=torch.uint8, device=DEV)
        for p in s.pool:
            p.random_(0, 256, generator=g)
        # the sources, each copied to `copies` pages of the others
        perm = rng.permutation(P)
        s.src = np.tile(perm[:n], case["copies"]).astype(np.int32)
        s.dst = perm[n:n + len(s.src)].astype(np.int32)
    elif kind == "append":
        sh = MODELS[case["model"]]
        R = case["rows"]
        s.qkv = torch.randn(R, sh.qkv_rows, generator=g, device=DEV)
        pos = case["far"] + np.arange(R)
        s.P = (pos[-1] + 16) // 16
        s.pos = torch.from_numpy(pos.astype(np.int32)).to(DEV)
        table = rng.permutation(s.P)
        s.slot = torch.from_numpy((table[pos // 16] * 16 + pos % 16).astype(np.int32)).to(DEV)
        s.k_pages, s.v_pages = (torch.zeros(s.P, sh.n_kv_heads, _block_bytes(sh.head_dim), dtype=torch.uint8, device=DEV) for _ in range(2))
        s.q = torch.empty(R, sh.n_heads, sh.head_dim, dtype=_dtype(sh), device=DEV)
        s.k, s.v = (torch.empty(R, sh.n_kv_heads, sh.head_dim, dtype=_dtype(sh), device=DEV) for _ in range(2))
    elif kind == "read":
        sh = MODELS[case["model"]]
        R = case["rows"]
        s.P = (R + 15) // 16 + 3
        s.k_pages, s.v_pages = _pages(s.P, sh, g)
        pos = np.arange(R)
        table = rng.permutation(s.P)
        s.slot = torch.from_numpy((table[pos // 16] * 16 + pos % 16).astype(np.int32)).to(DEV)
        s.k, s.v = (torch.empty(R, sh.n_kv_heads, sh.head_dim, dtype=_dtype(sh), device=DEV) for _ in range(2))
    else:
        sh = MODELS[case["model"]]
        rows, pos0 = _segments(case)
        s.rows, s.pos0 = np.array(rows, dtype=np.int32), np.array(pos0, dtype=np.int32)
        need = (s.pos0 + s.rows + 15) // 16
        s.P = int(need.sum())
        perm = rng.permutation(s.P).astype(np.int32)
        s.table = np.zeros((len(rows), int(need.max())), dtype=np.int32)
        for i, o in enumerate(np.cumsum(need) - need):
            s.table[i, :need[i]] = perm[o:o + need[i]]
        s.q = torch.randn(int(s.rows.sum()), sh.n_heads, sh.head_dim, generator=g, device=DEV).to(_dtype(sh))
        s.k_pages, s.v_pages = _pages(s.P, sh, g)
        s.out = torch.zeros(s.q.shape[0], sh.q_dim, dtype=s.q.dtype, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass, in elementary operations

def _score(s):
    z, n = s.logits, s.case["top"]
    inv = torch.where(s.temps > 0, 1 / s.temps, 0.0).unsqueeze(1)
    m, best = z.max(1, keepdim=True)
    fine = torch.isfinite(m).squeeze(1)
    d = (z - m) * inv
    d = torch.where(torch.isfinite(z), d, -math.inf)
    w = torch.exp(d)
    total = w.sum(1, keepdim=True)
    log_total = total.log()
    entropy = (log_total - torch.where(w > 0, w * d, 0.0).sum(1, keepdim=True) / total).squeeze(1)
    greedy = (s.temps == 0).unsqueeze(1)
    first = (z == m).int().argmax(1, keepdim=True)  # the lowest id of the largest logit

    def of(ids):
        point = torch.where(ids == first, 0.0, -math.inf)
        return torch.where(greedy, point, d.gather(1, ids) - log_total)

    ids = s.tokens.long().unsqueeze(1)
    given = (ids >= 0) & (ids < z.shape[1])
    logp = torch.where(given, of(ids.clamp(0, z.shape[1] - 1)), -math.inf).squeeze(1)
    entropy = torch.where(greedy.squeeze(1), 0.0, entropy)
    top = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :n] if n else first[:, :0]
    top_logp = of(top) if n else d[:, :0]
    bad = ~fine.unsqueeze(1)
    nan = math.nan
    return (torch.where(fine, logp, nan), torch.where(fine, entropy, nan), torch.where(bad, -1, top).int(), torch.where(bad, nan, top_logp))


def _rotate(x, pos, theta):
    """fp64 [R, H, hd], rotated by its row's position."""
    half = x.shape[-1] // 2
    angle = pos.double()[:, None] * torch.exp(torch.arange(half, device=DEV, dtype=torch.float64) * (-math.log(theta) / half))
    cos, sin = angle.cos().unsqueeze(1), angle.sin().unsqueeze(1)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _append(s):
    sh = MODELS[s.case["model"]]
    x = s.qkv.unflatten(1, (-1, sh.head_dim))
    turned = _rotate(x[:, :sh.n_heads + sh.n_kv_heads].double(), s.pos, float(np.float32(sh.rope_theta))).float()
    k, v = turned[:, sh.n_heads:], x[:, sh.n_heads + sh.n_kv_heads:]
    held = [_numbers(_codes(y, _exponents(y)), _exponents(y)) for y in (k, v)]
    return tuple(y.to(s.q.dtype) for y in (turned[:, :sh.n_heads], *held))


def _read(s):
    hd = MODELS[s.case["model"]].head_dim
    page, token = s.slot.long() // 16, s.slot.long() % 16
    return tuple(_unpack(p, page, token, _tables(place, hd)).to(s.k.dtype) for p, place in ((s.k_pages, _k_place), (s.v_pages, _v_place)))


def _attend(s):
    """Every sequence's rows and keys padded to the longest."""
    sh = MODELS[s.case["model"]]
    hq, hkv, hd = sh.n_heads, sh.n_kv_heads, sh.head_dim
    rows, pos0 = torch.from_numpy(s.rows).to(DEV), torch.from_numpy(s.pos0).to(DEV)
    most, keys = int(s.rows.max()), int((s.pos0 + s.rows).max())
    at = torch.arange(most, device=DEV)
    valid = at < rows[:, None]
    row = ((rows.cumsum(0) - rows)[:, None] + at).clamp(max=s.q.shape[0] - 1)
    t = torch.arange(keys, device=DEV)
    page = torch.from_numpy(s.table).to(DEV).long()[:, t // 16]
    k, v = (_unpack(p, page, (t % 16).expand_as(page), _tables(place, hd)).transpose(1, 2).contiguous()
            for p, place in ((s.k_pages, _k_place), (s.v_pages, _v_place)))  # [n, Hkv, keys, hd]
    q = s.q[row].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [n, Hkv, G rows, hd]
    w = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(hd)
    seen = (t <= (pos0[:, None] + at)[..., None])[:, None, None]  # [n, 1, 1, rows, keys]
    w = torch.where(seen, w.unflatten(2, (hq // hkv, most)), -math.inf)
    w = torch.exp(w - w.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    o = torch.matmul(w.flatten(2, 3), v).unflatten(2, (hq // hkv, most))  # [n, Hkv, G, rows, hd]
    return o.permute(0, 3, 1, 2, 4).flatten(2)[valid].to(s.q.dtype)


def run(s):
    if own:
        return _run_own(s)
    kind = s.case["kind"]
    if kind == "pages":
        src, dst = torch.from_numpy(s.src).to(DEV).long(), torch.from_numpy(s.dst).to(DEV).long()
        s.pool[:, dst] = s.pool[:, src]
        return s.pool
    return {"score": _score, "append": _append, "read": _read, "attn": _attend}[kind](s)


# ---------------------------------------------------------------------------
# one pass, by the framework's calls

def _workspace(s, nbytes):
    """The caller's workspace, kept from pass to pass."""
    if not hasattr(s, "ws"):
        s.ws = torch.empty(max(256, nbytes), dtype=torch.uint8, device=DEV)
    return s.ws


def _run_own(s):
    from paper_2607_20507_amd import binding as B
    case = s.case
    kind = case["kind"]
    if kind == "score":
        R, V, n = case["rows"], case["vocab"], case["top"]
        if not hasattr(s, "logp"):
            s.logp, s.entropy = torch.empty(2, R, device=DEV)
            s.ids, s.top_logp = torch.empty(R, n, dtype=torch.int32, device=DEV), torch.empty(R, n, device=DEV)
            _workspace(s, B.spec_token_logprobs_workspace_bytes(R, V, n))
        B.spec_token_logprobs(s.logits, s.temps, s.tokens, s.logp, s.entropy, s.ids, s.top_logp, s.ws)
        return s.logp, s.entropy, s.ids, s.top_logp
    if kind == "pages":
        if not hasattr(s, "ws"):
            _workspace(s, B.spec_op_kv_copy_pages_workspace_bytes(len(s.src)))
        B.spec_op_kv_copy_pages(s.pool, s.src, s.dst, s.ws)
        return s.pool
    sh = MODELS[case["model"]]
    dt = B.SPEC_F32 if sh.dtype == "f32" else B.SPEC_BF16
    if kind == "append":
        B.spec_op_rope_kv4(dt, case["rows"], sh.n_heads, sh.n_kv_heads, sh.head_dim, sh.rope_theta, s.qkv, s.pos, s.slot, s.P, s.q, s.k_pages, s.v_pages)
        B.spec_op_kv4_read(dt, case["rows"], sh.n_kv_heads, sh.head_dim, s.slot, s.P, s.k_pages, s.v_pages, s.k, s.v)
        return s.q, s.k, s.v
    if kind == "read":
        B.spec_op_kv4_read(dt, case["rows"], sh.n_kv_heads, sh.head_dim, s.slot, s.P, s.k_pages, s.v_pages, s.k, s.v)
        return s.k, s.v
    if not hasattr(s, "ws"):
        _workspace(s, B.spec_op_attention_kv4_workspace_bytes(dt, s.rows, s.pos0, s.table.shape[1], sh.n_heads, sh.n_kv_heads, sh.head_dim))
    B.spec_op_attention_kv4(dt, s.rows, s.pos0, s.table, s.P, sh.n_heads, sh.n_kv_heads, sh.head_dim, s.q, s.k_pages, s.v_pages, s.out, s.ws)
    return s.out


# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "score":
        R, V = case["rows"], case["vocab"]
        return {"bytes": R * (4 * V + 16 + 8 * case["top"]), "flops": 4 * R * V}
    sh = MODELS[case["model"]]
    token = 2 * sh.n_kv_heads * _block_bytes(sh.head_dim) / 16  # a token's K and V in 4 bits
    if kind == "pages":
        page = sh.n_kv_heads * _block_bytes(sh.head_dim) if case["bits"] == 4 else sh.kv_dim * 16 * sh.bytes_per_elem()
        return {"bytes": 2 * case["layers"] * page * case["sources"] * (1 + case["copies"]), "flops": 0}
    e = sh.bytes_per_elem()
    if kind == "append":
        return {"bytes": case["rows"] * (4 * sh.qkv_rows + token + e * sh.qkv_rows), "flops": case["rows"] * 3 * sh.qkv_rows}
    if kind == "read":
        return {"bytes": case["rows"] * (token + 2 * e * sh.kv_dim), "flops": 0}
    rows, pos0 = _segments(case)
    seen = sum(r * p + r * (r + 1) // 2 for r, p in zip(rows, pos0))
    return {"bytes": sum(r + p for r, p in zip(rows, pos0)) * token + 2 * e * sum(rows) * sh.q_dim, "flops": 4 * sh.q_dim * seen}


# ---------------------------------------------------------------------------
# the definitions in 64 bits

_LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _held64(x):
    """What the cache holds of fp64 x: the nearest level of each value by its distance, on the host."""
    x = x.cpu().numpy()
    out = np.empty_like(x)
    flat, to = x.reshape(-1, 32), out.reshape(-1, 32)
    for i in range(0, len(flat), 1 << 16):
        b = flat[i:i + (1 << 16)]
        top = np.abs(b).max(1, keepdims=True)
        with np.errstate(divide="ignore"):
            e = np.where(top > 0, np.ceil(np.log2(top / 6.0)), -126)
        e = np.where(6.0 * np.exp2(e - 1) >= top, e - 1, np.where(6.0 * np.exp2(e) < top, e + 1, e))  # log2's own rounding
        unit = np.exp2(np.maximum(e, -126))
        r = np.abs(b) / unit
        n = np.searchsorted((_LEVELS[1:] + _LEVELS[:-1]) / 2, r)  # a tie stays with the lower level ...
        tie = (n < 7) & (r == (_LEVELS[np.minimum(n + 1, 7)] + _LEVELS[n]) / 2) & (n % 2 == 1)
        to[i:i + (1 << 16)] = np.sign(b) * _LEVELS[n + tie] * unit  # ... unless that one is odd
    return torch.from_numpy(out)


def _decode64(pages, slots, place, hd):
    """fp64 [n, Hkv, hd] of the listed slots, byte by byte on the host."""
    raw = pages.cpu().numpy()
    slots = np.asarray(slots)
    out = np.empty((len(slots), raw.shape[1], hd))
    signed = np.concatenate([_LEVELS, -_LEVELS])
    for t in range(16):
        rows = np.nonzero(slots % 16 == t)[0]
        blocks = raw[slots[rows] // 16]
        for d in range(hd):
            byte, nibble, scale = place(t, d, hd)
            out[rows, :, d] = signed[(blocks[:, :, byte] >> (4 * nibble)) & 15] * np.exp2(blocks[:, :, scale].astype(np.float64) - 127)
    return torch.from_numpy(out)


def _exact_score(case, seed):
    s = prepare(case, seed)
    n, got = case["top"], []
    for r in range(0, case["rows"], 128):
        z, t, tok = s.logits[r:r + 128].double(), s.temps[r:r + 128].double(), s.tokens[r:r + 128].long()
        ok = torch.isfinite(z.amax(1))
        p = torch.log_softmax(z / torch.where(t > 0, t, 1.0)[:, None], 1)
        h = torch.special.entr(p.exp()).sum(1)
        point = torch.full_like(p, -math.inf)
        point[torch.arange(len(z)), [int(torch.nonzero(x == x.max())[0]) if o else 0 for x, o in zip(z, ok)]] = 0.0
        p, h = torch.where((t > 0)[:, None], p, point), torch.where(t > 0, h, 0.0)
        lp = torch.where((tok >= 0) & (tok < z.shape[1]), p[torch.arange(len(z)), tok.clamp(0, z.shape[1] - 1)], -math.inf)
        top = p.topk(n, 1)[0]
        got.append([torch.where(ok, lp, math.nan), torch.where(ok, h, math.nan), torch.where(ok[:, None], top, math.nan)])
    lp, h, top = (torch.cat([x[i] for x in got]) for i in range(3))
    return lp, h, None, top


def exact(case, seed):
    kind = case["kind"]
    if kind == "score":
        return _exact_score(case, seed)
    if kind == "pages":
        return None  # bytes
    s = prepare(case, seed)
    sh = MODELS[case["model"]]
    hq, hkv, hd = sh.n_heads, sh.n_kv_heads, sh.head_dim
    if kind == "append":
        x = s.qkv.double().cpu().unflatten(1, (-1, hd))
        pos, half = s.pos.cpu().double(), hd // 2
        turn = torch.polar(torch.ones(half, dtype=torch.float64)[None].expand(len(pos), half), pos[:, None] * float(np.float32(sh.rope_theta)) ** (-torch.arange(half) / half).double())
        z = torch.complex(x[:, :hq + hkv, :half], x[:, :hq + hkv, half:]) * turn[:, None]
        z = torch.cat([z.real, z.imag], -1)
        return z[:, :hq].to(DEV), _held64(z[:, hq:].contiguous()).to(DEV), _held64(x[:, hq + hkv:].contiguous()).to(DEV)
    if kind == "read":
        slots = s.slot.cpu().numpy()
        return _decode64(s.k_pages, slots, _k_place, hd).to(DEV), _decode64(s.v_pages, slots, _v_place, hd).to(DEV)
    if sum(int(r) + int(p) for r, p in zip(s.rows, s.pos0)) * hkv * hd > 3e8:
        return None
    rows, pos0 = s.rows.tolist(), s.pos0.tolist()
    slots = [s.table[i][np.arange(r + p) // 16].astype(np.int64) * 16 + np.arange(r + p) % 16 for i, (r, p) in enumerate(zip(rows, pos0))]
    keys, values = (_decode64(x, np.concatenate(slots), place, hd).split([len(y) for y in slots]) for x, place in ((s.k_pages, _k_place), (s.v_pages, _v_place)))
    out, r0 = [], 0
    for r, p, k, v in zip(rows, pos0, keys, values):
        k, v = k.to(DEV), v.to(DEV)
        q = s.q[r0:r0 + r].double()
        o = torch.empty(r, hq, hd, dtype=torch.float64, device=DEV)
        hidden = torch.arange(r + p, device=DEV) > p + torch.arange(r, device=DEV)[:, None]
        for h in range(hq):
            kk, vv = k[:, h // (hq // hkv)].contiguous(), v[:, h // (hq // hkv)].contiguous()
            w = (q[:, h].contiguous() @ kk.t().contiguous() / hd ** 0.5).masked_fill(hidden, -math.inf)
            o[:, h] = torch.softmax(w, 1) @ vv
        out.append(o.flatten(1))
        r0 += r
    return torch.cat(out)
