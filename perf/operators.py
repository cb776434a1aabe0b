"""Performance cases of the 8-bit cache and of the block-sparse decode that reads it.

Every case is one use of entry points of ``paper_2607_07740_amd.api`` on the
shapes of a Qwen3-like layer (head dim 128, RoPE base 1e6, a 32768-token
pretraining window, a 4096-token local window): rows appended to an 8-bit
cache and read back, a decode step over all of it, the scores of its blocks, the
choice among them, and a decode step over the chosen ones.

The cache holds blocks of 64 tokens.  A block of one kv head is 64 x 128 e4m3
values with one power-of-two scale, in the order the decode kernel reads:
  K  key = 32 a + 16 t + r, channel = 64 p + 32 u + 8 g + j, as [a][t][u][g][r][j][p]
  V  key = 32 a + 16 t + 4 g + i, channel = 32 c + 16 e + m, as [a][c][g][m][e][t][i]
Beside them lie the scales (fp32) and each block's mean key (bf16).

Fields of a case
  op      append | decode | scores | select | blocks
  Hq, Hkv query and key/value heads (grouped-query attention)
  lens    sequence lengths, one per sequence, as a text.  append: before the call.
  n       append: rows appended per sequence.  select, blocks: blocks chosen per kv head.
  cap     tokens the cache can hold per sequence
  page    tokens per page of a paged cache, 0 for a dense one
  bifocal the paper's two views, or base rotations for every key
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
BLOCK = 64
THETA = 1e6
W_PRE = 32768
W_LOCAL = 4096
N_FIRST = 1     # blocks at the start of a sequence that are always chosen
K_OUTLIERS = 8  # channels of K that are 1.5x larger: attention as peaky as a trained layer's
E_MIN, E_MAX = -117, 119  # exponents of the scales


def _case(name, op, Hq, Hkv, lens, n=0, cap=0, page=0, bifocal=True):
    c = dict(op=op, Hq=Hq, Hkv=Hkv, lens=",".join(str(x) for x in lens), n=n, cap=cap, page=page,
             bifocal=bifocal)
    return dict(c, name=name) if name else c


CHAT = [517, 640, 801, 1000, 1024, 1250, 1501, 1777, 2048, 2049, 2300, 2700, 3001, 3333, 3900,
        4096, 4097, 4500, 5000, 5555, 6001, 6800, 7400, 8192, 8193, 9000, 10007, 11000, 12288,
        13001, 15000, 16384]
LONG = [32768, 32769, 65536, 65537, 98304, 98305, 131071, 131072]


def listed():
    return [
        # the keys and values of a prompt enter an empty cache, and come back for the next chunk
        _case("append_prompt_30k", "append", 32, 8, [0], n=30001, cap=32768),
        # one token each of a small batch whose blocks are partly filled: the smallest append
        _case("append_token_paged_b16", "append", 32, 8,
              [63, 64, 65, 100, 127, 1, 0, 200, 190, 33, 255, 128, 70, 17, 222, 250], n=1,
              cap=256, page=64),
        # one token of a chat that has only begun: latency, the smallest decode
        _case("decode_b1_2k", "decode", 16, 8, [1999], cap=4096),
        # one token of a single long document: streaming the whole cache once (G = 4)
        _case("decode_b1_128k", "decode", 32, 8, [131072], cap=131072),
        # a batch of long documents that reached different lengths (G = 1 .. 4): the largest
        _case("decode_b8_ragged", "decode", 32, 8, LONG, cap=131072),
        # an ordinary serving step: many sequences of chat length, paged, the base model's rotations
        _case("decode_paged_b32", "decode", 32, 8, CHAT, cap=16384, page=64, bifocal=False),
        # the blocks of one long document are scored ...
        _case("scores_b1_128k", "scores", 32, 8, [131072], cap=131072),
        # ... and those of a batch of them, on pages
        _case("scores_paged_b8", "scores", 64, 8, LONG, cap=131072, page=256),
        # 8192 of 131072 tokens are chosen for each kv head
        _case("select_b1_128k", "select", 32, 8, [131072], n=128, cap=131072),
        # the same for a batch
        _case("select_b8", "select", 32, 8, LONG, n=128, cap=131072),
        # one token of a long document over its chosen blocks
        _case("blocks_b1_128k", "blocks", 32, 8, [131072], n=128, cap=131072),
        # a batch of them, on pages
        _case("blocks_paged_b8", "blocks", 32, 8, LONG, n=160, cap=131072, page=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(16, 8), (32, 8), (32, 8), (64, 8), (28, 4), (8, 8)])
    op = rng.choice(["append", "decode", "decode", "scores", "select", "blocks"])
    page = rng.choice([0, 64, 128, 256])
    unit = page or BLOCK
    fit = lambda n: (n + unit - 1) // unit * unit  # noqa: E731
    bifocal = rng.random() < 0.75
    if op == "append":
        B = rng.choice([1, 2, 5, 16, 32])
        n = _log_int(rng, 1, 30000 // B)
        lens = [rng.randint(0, 3) and _log_int(rng, 1, 1000) for _ in range(B)]
        return _case("", op, *heads, lens, n=n, cap=fit(max(lens) + n), page=page)
    B = rng.choice([1, 1, 2, 4, 8, 16, 32] if op != "select" else [1, 1, 2, 4, 8])
    most = 655360 // B * 32 // max(32, heads[0])  # no larger a call than the largest listed one
    lens = [_log_int(rng, 100, min(131072, most)) for _ in range(B)]
    if op == "select":  # one at least that leaves a choice
        lens[0] = _log_int(rng, 20000, min(131072, most))
    n = 0
    if op in ("select", "blocks"):
        n = rng.randint(W_LOCAL // BLOCK + 2 + N_FIRST, 200)
    return _case("", op, *heads, lens, n=n, cap=fit(max(lens)), page=page, bifocal=bifocal)


def _lens(c):
    return [int(x) for x in c["lens"].split(",")]


# ------------------------------------------------------- the 8-bit cache
def _exponent(top):
    """The smallest e in [E_MIN, E_MAX] with top <= 448 * 2^e."""
    m, e = torch.frexp(top / 448.0)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(top == 0, torch.full_like(e, E_MIN), e).clamp(E_MIN, E_MAX)


def _power(e):
    """2^e as fp32, from its bits: a power function may be an ulp off."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _pack_k(y):
    """[..., 64 keys, 128] e4m3 -> the K image of each block, [..., 8192] bytes."""
    lead, n = y.shape[:-2], y.dim() - 2
    y = y.contiguous().view(torch.uint8).view(*lead, 2, 2, 16, 2, 2, 4, 8)  # a t r p u g j
    return y.permute(*range(n), n, n + 1, n + 4, n + 5, n + 2, n + 6, n + 3).reshape(*lead, -1)


def _unpack_k(image):
    lead, n = image.shape[:-1], image.dim() - 1
    y = image.view(*lead, 2, 2, 2, 4, 16, 8, 2)  # a t u g r j p
    return y.permute(*range(n), n, n + 1, n + 4, n + 6, n + 2, n + 3, n + 5).reshape(
        *lead, BLOCK, D).view(torch.float8_e4m3fn)


def _pack_v(y):
    lead, n = y.shape[:-2], y.dim() - 2
    y = y.contiguous().view(torch.uint8).view(*lead, 2, 2, 4, 4, 4, 2, 16)  # a t g i c e m
    return y.permute(*range(n), n, n + 4, n + 2, n + 6, n + 5, n + 1, n + 3).reshape(*lead, -1)


def _unpack_v(image):
    lead, n = image.shape[:-1], image.dim() - 1
    y = image.view(*lead, 2, 4, 4, 16, 2, 2, 4)  # a c g m e t i
    return y.permute(*range(n), n, n + 5, n + 2, n + 6, n + 1, n + 4, n + 3).reshape(
        *lead, BLOCK, D).view(torch.float8_e4m3fn)


def _images(pool, blocks):
    """The blocks' images of a pool [pages, Hkv, tokens, 128], as [pages, Hkv, blocks, 8192]."""
    return pool.view(pool.shape[0], pool.shape[1], blocks, BLOCK * D)


def _by_sequence(s, pool):
    """[pages, Hkv, blocks of a page, ...] -> [B, Hkv, blocks of a sequence, ...]."""
    if s["table"] is None:
        return pool
    x = pool[s["table"].long()]  # [B, pages, Hkv, blocks, ...]
    return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1, *x.shape[4:])


# ------------------------------------------------------------------ inputs
def _rows(gen, n, Hkv, outliers):
    """bf16 keys or values of n tokens: normals, each head at a size of its own."""
    x = torch.randn((n, Hkv, D), generator=gen, device="cuda")
    size = torch.exp2(torch.rand((Hkv, 1), generator=gen, device="cuda") * 2 - 1)
    if outliers:
        ch = torch.randperm(D, generator=gen, device="cuda")[:K_OUTLIERS]
        x[..., ch] *= 1.5
    return x.mul_(size).to(torch.bfloat16)


def _pools(c, gen):
    """Pools of one cache, each block filled with random rows that are quantised by
    its own scale; the mean key of a block is that of all of its rows."""
    B, Hkv = len(_lens(c)), c["Hkv"]
    page = c["page"] or c["cap"]
    pages = B * (c["cap"] // page) + (3 if c["page"] else 0)
    per = page // BLOCK
    k = torch.empty((pages, Hkv, page, D), dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    ks = torch.empty((pages, Hkv, per), device="cuda")
    vs = torch.empty_like(ks)
    mean = torch.empty((pages, Hkv, per, D), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 16) // page)
    for p in range(0, pages, step):
        n = min(step, pages - p)
        for pool, scale, pack, is_k in ((k, ks, _pack_k, True), (v, vs, _pack_v, False)):
            x = _rows(gen, n * page, Hkv, is_k).float()
            x = x.view(n, per, BLOCK, Hkv, D).permute(0, 3, 1, 2, 4)
            sc = _power(_exponent(x.abs().amax((-2, -1))))
            y = _e4m3(x / sc[..., None, None])
            pool[p:p + n] = pack(y).view(n, Hkv, page, D)
            scale[p:p + n] = sc
            if is_k:
                mean[p:p + n] = (y.float().sum(-2) * sc[..., None] / BLOCK).to(torch.bfloat16)
    return k, v, ks, vs, mean


def _pick(scores, lens, n_select):
    """Blocks of the first N_FIRST and of the local band, then by falling score with
    ties to the lowest index; ascending, -1 behind the last."""
    nb = scores.shape[-1]
    j = torch.arange(nb, device=scores.device)
    last = (lens.long()[:, None, None] + BLOCK - 1) // BLOCK
    always = (j < N_FIRST) | (BLOCK * j + BLOCK - 1 >= lens.long()[:, None, None] - 1 - W_LOCAL)
    inside = (j < last).expand(scores.shape)
    s = torch.where(always, torch.full_like(scores, math.inf), scores)
    s = torch.where(inside, s, torch.full_like(scores, -math.inf))
    order = torch.sort(s, dim=-1, descending=True, stable=True).indices[..., :n_select]
    order = torch.where(torch.gather(inside, -1, order), order, torch.full_like(order, nb))
    order = torch.sort(order, dim=-1).values
    order = torch.where(order < nb, order, torch.full_like(order, -1)).to(torch.int32)
    if order.shape[-1] < n_select:
        fill = order.new_full((*order.shape[:-1], n_select - order.shape[-1]), -1)
        order = torch.cat([order, fill], -1)
    return order.contiguous()


def _random_scores(c, lens, gen):
    """Scores as block_scores8 gives them: -inf past the end; some are equal."""
    nb = c["cap"] // BLOCK
    s = torch.randn((len(_lens(c)), c["Hkv"], nb), generator=gen, device="cuda")
    s = torch.round(s * 256) / 256
    j = torch.arange(nb, device="cuda")
    return s.masked_fill_(BLOCK * j >= lens[:, None, None], -math.inf)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, Hq, Hkv = len(_lens(c)), c["Hq"], c["Hkv"]
    lens = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
    s = dict(case=c, lens=lens, table=None)
    if c["op"] == "select":
        return dict(s, scores=_random_scores(c, lens, gen))
    k, v, ks, vs, mean = _pools(c, gen)
    if c["page"]:
        per = c["cap"] // c["page"]
        order = torch.randperm(k.shape[0], generator=gen, device="cuda")[:B * per]
        s["table"] = order.view(B, per).to(torch.int32)
    if c["op"] == "append":
        s.update(k_new=_rows(gen, B * c["n"], Hkv, True).view(B, c["n"], Hkv, D),
                 v_new=_rows(gen, B * c["n"], Hkv, False).view(B, c["n"], Hkv, D))
    else:
        s["q"] = torch.randn((B, Hq, D), generator=gen, device="cuda").to(torch.bfloat16)
    if c["op"] == "blocks":
        s["blocks"] = _pick(_random_scores(c, lens, gen), lens, c["n"])
    s.update(k=k, v=v, k_scale=ks, v_scale=vs, k_mean=mean)
    if own:  # the handle and the workspace that a decoding loop keeps
        from paper_2607_07740_amd import api
        s["cache"] = api.Cache8(k, v, ks, vs, mean)
        s["ws"] = api.decode8_workspace(Hq, Hkv, device="cuda")
    return s


# --------------------------------------------------------------- plain forms
def _groups(c, lens):
    """G = max(1, ceil(L / W_PRE)) of each sequence, or 1 with base rotations."""
    if not c["bifocal"]:
        return torch.ones_like(lens).long()
    return ((lens.long() + W_PRE - 1) // W_PRE).clamp(min=1)


def _angles(pos):
    """cos, sin of pos * theta^(-2i/d): in 64 bits, as far positions need, then in 32."""
    om = THETA ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device="cuda") / D)
    a = pos.double()[..., None] * om
    return a.cos().float(), a.sin().float()


def _rope(x, cs):
    lo, hi = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([lo * cs[0] - hi * cs[1], hi * cs[0] + lo * cs[1]], -1)


def _plain_append(s):
    c, n = s["case"], s["case"]["n"]
    B, Hkv, nb = len(_lens(c)), c["Hkv"], c["cap"] // BLOCK
    per = (c["page"] or c["cap"]) // BLOCK
    start = s["lens"].long()
    pos = start[:, None] + torch.arange(n, device="cuda")  # [B, n]
    at = torch.arange(c["cap"], device="cuda")
    old = (at < start[:, None]).view(B, 1, nb, BLOCK)
    new = ((at >= start[:, None]) & (at < start[:, None] + n)).view(B, 1, nb, BLOCK)
    touched = new.any(-1)  # [B, 1, nb]
    kept = (old & touched[..., None]).any(-1)
    out = []
    for image, rows, scale, unpack in (("k", "k_new", "k_scale", _unpack_k),
                                       ("v", "v_new", "v_scale", _unpack_v)):
        was = _by_sequence(s, s[scale])
        y = unpack(_by_sequence(s, _images(s[image], per))).float()  # [B, Hkv, nb, 64, D]
        x = torch.zeros((B, c["cap"], Hkv, D), device="cuda")
        x[torch.arange(B, device="cuda")[:, None], pos] = s[rows].float()
        x = x.view(B, nb, BLOCK, Hkv, D).permute(0, 3, 1, 2, 4)
        sc = _power(_exponent(x.abs().amax((-2, -1))))
        sc = torch.where(kept, torch.maximum(sc, was), sc)
        held = torch.where(old[..., None], y * (was / sc)[..., None, None], x / sc[..., None, None])
        held = torch.where((old | new)[..., None], _e4m3(held).float(), torch.zeros_like(held))
        sc = torch.where(touched, sc, was)
        y = torch.where(touched[..., None, None], held, y)
        if image == "k":
            rows_in = (old | new).sum(-1).float()  # [B, 1, nb]
            m = (y * (old | new)[..., None]).sum(-2) * sc[..., None] / rows_in.clamp(min=1)[..., None]
            mean = torch.where(touched[..., None], m.to(torch.bfloat16),
                               _by_sequence(s, s["k_mean"]))
        out.append((y * sc[..., None, None]).permute(0, 2, 3, 1, 4).reshape(
            B, c["cap"], Hkv, D).to(torch.bfloat16))
        out.append(_to_pool(s, s[scale], sc))
    return out[0], out[2], out[1], out[3], _to_pool(s, s["k_mean"], mean)


def _to_pool(s, pool, x):
    """A copy of the pool with the sequences' entries [B, Hkv, blocks, ...] put in."""
    if s["table"] is None:
        return x
    B, per = s["table"].shape
    x = x.reshape(B, x.shape[1], per, -1, *x.shape[3:]).transpose(1, 2)
    pool = pool.clone()
    pool[s["table"].long()] = x
    return pool


def _plain_attention(s, blocks):
    """One query per sequence over all keys, or over the listed blocks."""
    c = s["case"]
    B, Hkv, g = len(_lens(c)), c["Hkv"], c["Hq"] // c["Hkv"]
    per = (c["page"] or c["cap"]) // BLOCK
    k, v = (_by_sequence(s, _images(s[x], per)) for x in ("k", "v"))
    ks, vs = (_by_sequence(s, s[x]) for x in ("k_scale", "v_scale"))
    if blocks is None:
        pos = torch.arange(c["cap"], device="cuda").expand(B, 1, -1)
        valid = pos < s["lens"][:, None, None]
    else:
        j = blocks.long().clamp(min=0)  # [B, Hkv, n]
        k, v = (torch.gather(x, 2, j[..., None].expand(-1, -1, -1, BLOCK * D)) for x in (k, v))
        ks, vs = torch.gather(ks, 2, j), torch.gather(vs, 2, j)
        pos = (j[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(2)
        valid = (pos < s["lens"][:, None, None]) & (blocks >= 0).repeat_interleave(BLOCK, -1)
    k = (_unpack_k(k).float() * ks[..., None, None]).flatten(2, 3)  # [B, Hkv, S, D]
    v = (_unpack_v(v).float() * vs[..., None, None]).flatten(2, 3)
    G = _groups(c, s["lens"])[:, None, None]
    last = s["lens"].long()[:, None, None] - 1
    remote = (last - pos > W_LOCAL) & (G > 1)
    k = _rope(k, _angles(torch.where(remote, pos // G, pos)))
    q = s["q"].float().view(B, Hkv, g, D)
    near, far = (_rope(q, _angles(p)) for p in (last, last // G))
    score = torch.where(remote[..., None], torch.matmul(k, far.transpose(2, 3).contiguous()),
                        torch.matmul(k, near.transpose(2, 3).contiguous()))  # [B, Hkv, S, g]
    score = (score / math.sqrt(D)).masked_fill_(~valid[..., None], -math.inf)
    p = (score - score.amax(2, keepdim=True)).exp()
    p = (p / p.sum(2, keepdim=True)).transpose(2, 3).contiguous()
    v = torch.where(valid[..., None], v, torch.zeros_like(v))
    return torch.matmul(p, v).view(B, c["Hq"], D).to(torch.bfloat16)


def _plain_scores(s):
    c = s["case"]
    B, Hkv, g, nb = len(_lens(c)), c["Hkv"], c["Hq"] // c["Hkv"], c["cap"] // BLOCK
    G = _groups(c, s["lens"])[:, None, None]
    mid = (BLOCK * torch.arange(nb, device="cuda") + BLOCK // 2 - 1).view(1, 1, nb) // G
    m = _rope(_by_sequence(s, s["k_mean"]).float(), _angles(mid))
    last = s["lens"].long()[:, None, None] - 1
    q = _rope(s["q"].float().view(B, Hkv, g, D), _angles(last // G))
    x = torch.matmul(m, q.transpose(2, 3).contiguous()).amax(-1) / math.sqrt(D)
    j = torch.arange(nb, device="cuda")
    return x.masked_fill_(BLOCK * j >= s["lens"][:, None, None], -math.inf)


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "append":
            return _plain_append(s)
        if c["op"] == "decode":
            return _plain_attention(s, None)
        if c["op"] == "scores":
            return _plain_scores(s)
        if c["op"] == "select":
            return _pick(s["scores"], s["lens"], c["n"])
        return _plain_attention(s, s["blocks"])
    from paper_2607_07740_amd import api
    if c["op"] == "append":
        api.cache8_append(s["cache"], s["k_new"], s["v_new"], s["lens"], block_table=s["table"])
        k, v = api.cache8_read(s["cache"], c["cap"], block_table=s["table"])
        return k, v, s["k_scale"], s["v_scale"], s["k_mean"]
    if c["op"] == "select":
        return api.select_blocks(s["scores"], s["lens"], c["n"], w_local=W_LOCAL, n_first=N_FIRST)
    kw = dict(w_pretrained=W_PRE, rope_theta=THETA, bifocal=c["bifocal"], block_table=s["table"])
    if c["op"] == "scores":
        return api.block_scores8(s["q"], s["cache"], s["lens"], **kw)
    kw.update(w_local=W_LOCAL, workspace=s["ws"])
    if c["op"] == "decode":
        return api.decode8(s["q"], s["cache"], s["lens"], **kw)
    return api.decode8_blocks(s["q"], s["cache"], s["lens"], s["blocks"], **kw)


# ------------------------------------------------------- work and reference
def work(case):
    """append: each new row read once and held once in 8 bits, then the whole cache read
    back.  decode: each key and value that is attended to, its block's scales, query and
    output once; one score and one value product per (key, query head).  scores: each
    block's mean once.  select: each score once."""
    c, lens, g = case, _lens(case), case["Hq"] // case["Hkv"]
    B, Hkv = len(lens), c["Hkv"]
    if c["op"] == "append":
        new = B * c["n"] * Hkv
        blocks = sum((n + c["n"] + BLOCK - 1) // BLOCK - n // BLOCK for n in lens) * Hkv
        held = B * c["cap"] * Hkv
        return {"bytes": new * (512 + 256) + blocks * (8 + 2 * D) + held * (256 + 512),
                "flops": 3 * D * (new + held)}
    nb = sum((n + BLOCK - 1) // BLOCK for n in lens)
    qo = 2 * B * c["Hq"] * D
    if c["op"] == "scores":
        return {"bytes": nb * Hkv * (2 * D + 4) + qo, "flops": nb * Hkv * D * (3 + 2 * g)}
    if c["op"] == "select":
        return {"bytes": 4 * nb * Hkv + 4 * B * Hkv * c["n"], "flops": nb * Hkv}
    keys = [n if c["op"] == "decode" else min(n, c["n"] * BLOCK) for n in lens]
    return {"bytes": sum(keys) * Hkv * 256 + sum(k // BLOCK for k in keys) * Hkv * 8 + 2 * qo,
            "flops": 4 * D * c["Hq"] * sum(keys)}


def _exact_e4m3(x):
    """fp64 to the nearest e4m3 value, ties to the even one: steps of 2^-3 of a value's
    power of two, none below 2^-9."""
    x = x.clamp(-448.0, 448.0)
    _, e = torch.frexp(x)
    step = ((e.long() - 4).clamp(min=-9) + 1023 << 52).view(torch.float64)  # exact powers of two
    return torch.round(x / step) * step


def _exact_append(c, s):
    k, v = [], []
    ks, vs, mean = s["k_scale"].double(), s["v_scale"].double(), s["k_mean"].double()
    page = c["page"] or c["cap"]
    for b, n0 in enumerate(_lens(c)):
        n1 = n0 + c["n"]
        for pool, scale, unpack, rows, got in ((s["k"], ks, _unpack_k, s["k_new"], k),
                                               (s["v"], vs, _unpack_v, s["v_new"], v)):
            pages = [b] if s["table"] is None else s["table"][b].tolist()
            img = torch.stack([_images(pool, page // BLOCK)[p] for p in pages])
            x = unpack(img).double() * scale[pages][..., None, None]  # [pages, Hkv, per, 64, D]
            x = x.permute(0, 2, 3, 1, 4).reshape(c["cap"], c["Hkv"], D)
            j0, j1 = n0 // BLOCK, (n1 + BLOCK - 1) // BLOCK
            x[n0:n1] = rows[b].double()
            x[n1:j1 * BLOCK] = 0
            part = x[j0 * BLOCK:j1 * BLOCK].view(j1 - j0, BLOCK, c["Hkv"], D)
            lo = torch.arange(j0 * BLOCK, j1 * BLOCK, device="cuda").view(-1, BLOCK) >= n0
            top = (part.abs() * lo[..., None, None]).amax((1, 3))  # of the new rows
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448.0)).clamp(E_MIN, E_MAX)
            sc = (e.long() + 1023 << 52).view(torch.float64)
            idx = [(pages[j * BLOCK // page], j * BLOCK % page // BLOCK) for j in range(j0, j1)]
            pg = torch.tensor([i[0] for i in idx], device="cuda")
            bl = torch.tensor([i[1] for i in idx], device="cuda")
            if n0 % BLOCK:
                sc[0] = torch.maximum(sc[0], scale[pg[0], :, bl[0]])
            part = _exact_e4m3(part / sc[:, None, :, None]) * sc[:, None, :, None]
            x[j0 * BLOCK:j1 * BLOCK] = part.view(-1, c["Hkv"], D)
            scale[pg, :, bl] = sc
            if pool is s["k"]:
                rows_in = (n1 - BLOCK * torch.arange(j0, j1, device="cuda")).clamp(max=BLOCK)
                mean[pg, :, bl] = part.sum(1) / rows_in[:, None, None]
            got.append(x)
    return torch.stack(k), torch.stack(v), ks, vs, mean


def _turns(pos):
    """e^(i pos omega) for 64-bit positions."""
    om = THETA ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    return torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(
        *pos.shape, D // 2), pos.double()[..., None] * om)


def _pairs(x):
    return torch.complex(x[..., :D // 2].double().contiguous(), x[..., D // 2:].double().contiguous())


def _logits(q, k, rel):
    """Re <q, e^(i rel omega) k>: q [g, D] and k [n, D], rel [n] = key minus query position."""
    return (_pairs(k) * _turns(rel)) @ _pairs(q).conj().T


def exact(case, seed):
    c = case
    if c["op"] == "select":
        return None
    s = prepare(c, seed)
    if c["op"] == "append":
        return _exact_append(c, s)
    g, page = c["Hq"] // c["Hkv"], c["page"] or c["cap"]
    nb = c["cap"] // BLOCK
    out = torch.zeros((len(_lens(c)), c["Hq"], D), dtype=torch.float64, device="cuda")
    sco = torch.full((len(_lens(c)), c["Hkv"], nb), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lens(c)):
        G = max(1, -(-n // W_PRE)) if c["bifocal"] else 1
        pages = [b] if s["table"] is None else s["table"][b].tolist()
        for h in range(c["Hkv"]):
            q = s["q"][b, h * g:(h + 1) * g]
            if c["op"] == "scores":
                m = s["k_mean"][pages, h].reshape(nb, D)[:-(-n // BLOCK)]
                mid = (BLOCK * torch.arange(m.shape[0], device="cuda") + 31) // G
                sco[b, h, :m.shape[0]] = _logits(q, m, mid - (n - 1) // G).real.amax(1) / D ** 0.5
                continue
            img = [_images(s[x], page // BLOCK)[pages, h].reshape(nb, -1) for x in ("k", "v")]
            sc = [s[x][pages, h].reshape(nb) for x in ("k_scale", "v_scale")]
            sel = torch.arange(nb, device="cuda") if c["op"] == "decode" else s["blocks"][b, h]
            sel = sel[sel >= 0].long()
            pos = (sel[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten()
            k, v = (u(i[sel]).double() * f[sel].double()[:, None, None]
                    for u, i, f in zip((_unpack_k, _unpack_v), img, sc))
            keep = pos < n
            pos, k, v = pos[keep], k.view(-1, D)[keep], v.view(-1, D)[keep]
            rel = torch.where(n - 1 - pos > W_LOCAL, pos // G - (n - 1) // G, pos - (n - 1))
            w = (_logits(q, k, rel).real / D ** 0.5).softmax(0)
            out[b, h * g:(h + 1) * g] = w.T @ v
    return sco if c["op"] == "scores" else out
