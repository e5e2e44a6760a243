"""The operators that take prompts in: rows of many requests appended to the paged cache, their attention behind the
histories that are there, and the log probabilities of their tokens.

Kinds of case (heads and vocabularies of the repository's own workloads, other sizes of the same ranges by `draw`):

  append   the fused projection's rows of ragged chunks: per-head RMSNorm of q and k, rotary embedding (of one axis, or
           of time, height and width), q out, K/V into the paged cache, and into the direct rings where there are any
  prompt   attention of a chunk's rows over the paged cache, each up to its own place (or the last `window` of them);
           the plan of the call, which a server makes once for all layers of a step, is part of the pass
  cross    the same without a mask: rows against states of another length
  scores   log probability and rank of given tokens, entropy, the most probable alternatives

`run` computes them from elementary torch operations, or, where `own` is set, through paper_2609_20734_amd.  Sizes that
differ between requests are spread evenly over a case's range and dealt to the requests by the seed, so a case's work
does not depend on the seed.
"""
import math

import torch

own = False

BLOCK = 16
EPS = 1e-6
THETA = 1e6

_LLAMA = dict(Hq=32, Hkv=8, D=128)      # Llama-3-8B-shaped heads
_QWEN = dict(Hq=16, Hkv=8, D=128)       # Qwen3-1.7B-shaped heads
_HYBRID = dict(Hq=64, Hkv=8, D=128)     # the hybrid workload's heads


def listed():
    return [
        # one new token of each of eight chats: the smallest call, where latency counts
        dict(name="append-b8", kind="append", B=8, rows_lo=1, rows_hi=1, hist_lo=17, hist_hi=900, **_QWEN, type="f32", norm=True,
             axes=1, ring=0),
        # a chunk of a prompt, 2,048 tokens, from the decoder's own projection; rings of the windowed path kept current
        dict(name="append-chunk", kind="append", B=1, rows_lo=2048, rows_hi=2048, hist_lo=4099, hist_hi=4099, **_QWEN, type="f32",
             norm=True, axes=1, ring=1024),
        # sixteen prompts with images (time, height, width), projections in bf16, no norms
        dict(name="append-images", kind="append", B=16, rows_lo=201, rows_hi=1900, hist_lo=0, hist_hi=600, **_LLAMA, type="bf16",
             norm=False, axes=3, ring=0),
        # a short question of one request: the smallest attention
        dict(name="prompt-short", kind="prompt", B=1, rows_lo=33, rows_hi=33, hist_lo=0, hist_hi=0, **_QWEN, window=0, out="f32"),
        # a prompt of 8,192 tokens in one call
        dict(name="prompt-8k", kind="prompt", B=1, rows_lo=8192, rows_hi=8192, hist_lo=0, hist_hi=0, **_LLAMA, window=0, out="bf16"),
        # a chunk of 512 tokens behind 65,000: work that has to be split over the history
        dict(name="prompt-chunk-long", kind="prompt", B=1, rows_lo=512, rows_hi=512, hist_lo=65001, hist_hi=65001, **_LLAMA, window=0,
             out="bf16"),
        # sixteen requests of a mixed step, from single tokens to chunks, behind short and long histories
        dict(name="prompt-mixed", kind="prompt", B=16, rows_lo=1, rows_hi=900, hist_lo=0, hist_hi=6000, **_QWEN, window=0, out="f32"),
        # a chunk of a natively windowed layer
        dict(name="prompt-window", kind="prompt", B=1, rows_lo=2048, rows_hi=2048, hist_lo=6150, hist_hi=6150, **_HYBRID, window=4096,
             out="bf16"),
        # one new token of 32 requests against an encoder's states
        dict(name="cross-b32", kind="cross", B=32, rows_lo=1, rows_hi=1, hist_lo=375, hist_hi=1500, Hq=16, Hkv=16, D=64, window=0,
             out="f32"),
        # four requests' rows against longer states (none of one request)
        dict(name="cross-rows", kind="cross", B=4, rows_lo=449, rows_hi=1200, hist_lo=0, hist_hi=6001, **_QWEN, window=0, out="bf16"),
        # the next token of four requests, twenty alternatives
        dict(name="scores-b4", kind="scores", R=4, V=151936, top=20),
        # a prompt's 1,024 tokens scored, five alternatives, an odd vocabulary
        dict(name="scores-prompt", kind="scores", R=1024, V=50257, top=5),
    ]


def _log(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    """One more case of the ranges above (heads, batches, rows, histories, windows, types, vocabularies)."""
    kind = rng.choice(["append", "append", "prompt", "prompt", "prompt", "cross", "scores", "scores"])
    if kind == "scores":
        R = _log(rng, 1, 1024)
        return dict(kind=kind, R=R, V=min(_log(rng, 1000, 152000), 60_000_000 // R) | rng.randint(0, 1), top=rng.choice([0, 1, 5, 20, 32]))
    hkv = rng.choice([2, 4, 8])
    G, D = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128])
    B = _log(rng, 1, 32)
    a, b = _log(rng, 1, 4096), _log(rng, 1, 4096)
    h, i = _log(rng, 1, 32768) - 1, _log(rng, 1, 32768) - 1
    c = dict(kind=kind, B=B, rows_lo=min(a, b), rows_hi=max(a, b), hist_lo=min(h, i), hist_hi=max(h, i), Hq=hkv * G, Hkv=hkv, D=D)
    if kind == "append":
        c["rows_hi"] = max(1, min(c["rows_hi"], 32768 // B))
        c["rows_lo"] = min(c["rows_lo"], c["rows_hi"])
        c["hist_hi"] = min(c["hist_hi"], 65536 // B)
        c["hist_lo"] = min(c["hist_lo"], c["hist_hi"])
        return dict(c, type=rng.choice(["f32", "bf16"]), norm=rng.random() < 0.5, axes=rng.choice([1, 1, 3]),
                    ring=rng.choice([0, 0, 100, 1024]))
    # no more scores than the largest listed case has
    while B * c["Hq"] * c["rows_hi"] * (c["rows_hi"] + c["hist_hi"]) > 1 << 30:
        if c["rows_hi"] > c["hist_hi"]:
            c["rows_hi"] = c["rows_hi"] * 2 // 3
        else:
            c["hist_hi"] = c["hist_hi"] * 2 // 3
    c["rows_lo"], c["hist_lo"] = min(c["rows_lo"], c["rows_hi"]), min(c["hist_lo"], c["hist_hi"])
    return dict(c, window=rng.choice([0, 0, _log(rng, 1, 4096)]) if kind == "prompt" else 0, out=rng.choice(["f32", "bf16", "bf16"]))


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers, evenly spread over [lo, hi] (the last is hi)."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _sizes(c):
    """(rows, positions held before them, or states) of each request, before the seed deals them."""
    B = c["B"]
    step = next(m for m in range(max(1, B // 3), 2 * B + 2) if math.gcd(m, B) == 1)
    hist = _spread(c["hist_lo"], c["hist_hi"], B)
    return list(zip(_spread(c["rows_lo"], c["rows_hi"], B), [hist[i * step % B] for i in range(B)]))


def _attended(c, rows, hist):
    """(scored pairs, positions read) of a request."""
    if c["kind"] == "cross":
        return rows * hist, hist
    w = c["window"] or 1 << 60
    n, full = hist + rows, max(0, min(rows, w - hist))       # the first `full` rows see all that is before them
    return full * hist + full * (full + 1) // 2 + (rows - full) * min(w, n), min(n, w + rows - 1)


def work(case):
    c = case
    if c["kind"] == "scores":
        return dict(bytes=4.0 * c["R"] * (c["V"] + 4 + 2 * c["top"]), flops=4.0 * c["R"] * c["V"])
    total = sum(r for r, _ in _sizes(c))
    if c["kind"] == "append":
        elems = total * (c["Hq"] + 2 * c["Hkv"]) * c["D"]
        kept = sum(min(r, c["ring"]) for r, _ in _sizes(c)) * 2 * c["Hkv"] * c["D"]
        return dict(bytes=elems * ((4.0 if c["type"] == "f32" else 2.0) + 2) + 2.0 * kept + 12.0 * total * (c["axes"] > 1),
                    flops=6.0 * elems)
    pairs = keys = 0
    for r, h in _sizes(c):
        p, k = _attended(c, r, h)
        pairs, keys = pairs + p, keys + k
    return dict(bytes=4.0 * c["Hkv"] * c["D"] * keys + total * c["Hq"] * (c["D"] * (6.0 if c["out"] == "f32" else 4.0) + 4),
                flops=4.0 * c["Hq"] * c["D"] * pairs)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 1000003 + 41)
        self.cpu = torch.Generator()
        self.cpu.manual_seed(int(seed) * 1000003 + 41)

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        t = torch.empty(*shape, dtype=dtype, device="cuda")
        flat = t.view(-1)
        for s in range(0, flat.numel(), 1 << 28):
            flat[s:s + (1 << 28)].normal_(mean, std, generator=self.g)
        return t

    def perm(self, n):
        return torch.randperm(n, generator=self.cpu).tolist()


class _State:
    pass


def _i32(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


def _paged(c, r, s):
    """Rows and lengths of the requests, the paged cache, its table, and for the plain form each row's request and place."""
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    sizes, deal = _sizes(c), r.perm(B)
    s.rows, s.hist = [sizes[deal[b]][0] for b in range(B)], [sizes[deal[b]][1] for b in range(B)]
    s.n = s.hist if c["kind"] == "cross" else [h + n for n, h in zip(s.rows, s.hist)]
    s.starts = [0]
    for n in s.rows:
        s.starts.append(s.starts[-1] + n)
    s.R = s.starts[-1]
    need = [-(-n // BLOCK) for n in s.n]
    s.mb, s.nb = max(1, max(need)), max(1, sum(need))
    s.max_len = s.mb * BLOCK
    ids, at = r.perm(s.nb), 0
    table = torch.zeros(B, s.mb, dtype=torch.int32)
    for b in range(B):
        table[b, :need[b]] = torch.tensor(ids[at:at + need[b]], dtype=torch.int32)
        at += need[b]
    s.k = r.normal(s.nb, Hkv, D // 8, BLOCK, 8, dtype=torch.bfloat16)
    s.v = r.normal(s.nb, Hkv, D, BLOCK, dtype=torch.bfloat16)
    s.table, s.seq, s.start = table.cuda(), _i32(s.n), _i32(s.starts)
    s.row_request = torch.repeat_interleave(torch.arange(B), torch.tensor(s.rows)).cuda()
    s.row_place = torch.cat([torch.arange(n - k, n) for n, k in zip(s.n, s.rows)]).cuda() if c["kind"] != "cross" else None


def _prepare_append(c, r, s):
    _paged(c, r, s)
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    s.qkv = r.normal(s.R, (Hq + 2 * Hkv) * D, std=1.5, dtype=torch.float32 if c["type"] == "f32" else torch.bfloat16)
    s.q_gain = r.normal(D, std=0.02, mean=1.0) if c["norm"] else None
    s.k_gain = r.normal(D, std=0.02, mean=1.0) if c["norm"] else None
    s.positions, s.axis_pairs = None, None
    if c["axes"] == 3:
        # runs of text, where the axes agree, between images, whose rows and columns count on from their start
        s.axis_pairs = [D // 2 - 2 * (D // 6), D // 6, D // 6]
        i = torch.arange(s.R)
        side, run = 24, 700
        image, at = (i // run) % 2 == 1, i // run * run
        base = s.row_place.cpu() - (i - at)
        s.positions = torch.stack([torch.where(image, base, s.row_place.cpu()),
                                   torch.where(image, base + (i - at) // side, s.row_place.cpu()),
                                   torch.where(image, base + (i - at) % side, s.row_place.cpu())], 1).clamp(min=0).int().cuda()
    s.q = torch.zeros(s.R, Hq, D, dtype=torch.bfloat16, device="cuda")
    s.k_ring = s.v_ring = None
    s.sink = 4 if c["ring"] else 0
    if c["ring"]:
        sb, rb = -(-s.sink // BLOCK), -(-c["ring"] // BLOCK) + 2
        s.k_ring = r.normal(B, sb + rb, Hkv, D // 8, BLOCK, 8, dtype=torch.bfloat16)
        s.v_ring = r.normal(B, sb + rb, Hkv, D, BLOCK, dtype=torch.bfloat16)
        # the rows that the rings still hold, and the ring block of each
        block = s.row_place // BLOCK
        last = (torch.tensor(s.n).cuda()[s.row_request] - 1) // BLOCK
        s.ring_rows = torch.nonzero((block < sb) | (block > last - rb))[:, 0]
        s.ring_block = torch.where(block < sb, block, sb + block % rb)[s.ring_rows]


def _prepare_attn(c, r, s):
    _paged(c, r, s)
    s.q = r.normal(s.R, c["Hq"], c["D"], dtype=torch.bfloat16)
    s.out = torch.zeros(s.R, c["Hq"], c["D"], dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16, device="cuda")
    s.lse = torch.zeros(s.R, c["Hq"], device="cuda")
    # rows as a padded array [B][rows], and each row's place in it
    M = max(s.rows)
    s.pad = torch.tensor([[min(a + i, s.R - 1) for i in range(M)] for a in s.starts[:-1]]).cuda()
    s.unpad = torch.cat([b * M + torch.arange(n) for b, n in enumerate(s.rows)]).cuda()
    s.first = torch.tensor([n - k for n, k in zip(s.n, s.rows)]).cuda()


def _prepare_scores(c, r, s):
    # peaked distributions over a long tail; a grammar's mask on every eighth row
    s.z = r.normal(c["R"], c["V"], std=2.5)
    s.z[::8, ::2] = -math.inf
    s.tokens = torch.randint(0, c["V"], (c["R"],), generator=r.g, device="cuda").int()
    likely = torch.rand(c["R"], generator=r.g, device="cuda") < 0.7
    s.tokens = torch.where(likely, s.z.argmax(-1).int(), s.tokens)
    R, k = c["R"], c["top"]
    s.logprob, s.entropy = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda")
    s.rank = torch.zeros(R, dtype=torch.int32, device="cuda")
    s.top = torch.zeros(R, k, device="cuda") if k else None
    s.ids = torch.zeros(R, k, dtype=torch.int32, device="cuda") if k else None


_PREPARE = dict(append=_prepare_append, prompt=_prepare_attn, cross=_prepare_attn, scores=_prepare_scores)


def prepare(case, seed):
    s = _State()
    s.c = dict(case)
    with torch.no_grad():
        _PREPARE[case["kind"]](case, _Rand(seed), s)
    if own:      # descriptions, workspaces and prepared calls, which a server keeps from step to step
        s.calls, s.outputs = _calls(s.c, s)
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _zeros(n):
    return torch.zeros(max(256, n), dtype=torch.uint8, device="cuda")


def _calls(c, s):
    import paper_2609_20734_amd as P
    if c["kind"] == "scores":
        desc = P.logprob_desc(c["V"], c["top"], s.z, s.tokens)
        ws = _zeros(P.logprob_workspace_size(desc, c["R"]))
        outputs = [s.logprob, s.rank, s.entropy] + ([s.top, s.ids] if c["top"] else [])
        return [P.prepare_token_logprobs(desc, c["R"], s.logprob, s.rank, s.entropy, s.top, s.ids, ws)], outputs
    shape = P.Shape(1, c["B"], c["Hq"], c["Hkv"], c["D"], s.mb, s.max_len, s.nb)
    rows = P.prompt_rows(s.R, s.start)
    if c["kind"] == "append":
        desc = P.append_desc(s.qkv, s.q_gain, s.k_gain, EPS, THETA, s.positions, s.axis_pairs)
        rings = (s.k_ring, s.v_ring, s.sink, c["ring"]) if c["ring"] else ()
        outputs = [s.q, s.k, s.v] + ([s.k_ring, s.v_ring] if c["ring"] else [])
        return [P.prepare_append_qkv(shape, rows, desc, s.k, s.v, s.table, s.seq, s.q, *rings)], outputs
    inp = P.inputs(s.q, s.k, s.v, s.table, s.seq, 1.0 / math.sqrt(c["D"]))
    plan, ws = _zeros(P.prompt_plan_size(shape, rows)), _zeros(P.prompt_workspace_size(shape, rows))
    causal = c["kind"] == "prompt"
    return [P.prepare_prompt_plan(shape, rows, s.seq, causal, c["window"], plan),
            P.prepare_prompt_attn(shape, inp, rows, plan, s.out, s.lse, ws)], [s.out, s.lse]


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _append(c, s):
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    x = s.qkv.float().view(s.R, Hq + 2 * Hkv, D)
    qk, v = x[:, :Hq + Hkv], x[:, Hq + Hkv:]
    if c["norm"]:
        gain = torch.cat([s.q_gain.expand(Hq, D), s.k_gain.expand(Hkv, D)])
        qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS) * gain
    pair = torch.arange(D // 2, device="cuda")
    freq = THETA ** (-2.0 * pair.double() / D)
    place = s.row_place[:, None].double()
    if s.positions is not None:
        ends = torch.tensor(s.axis_pairs, device="cuda").cumsum(0)
        place = s.positions[:, (pair[:, None] >= ends).sum(1)].double()
    angle = place * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    lo, hi = qk[..., :D // 2], qk[..., D // 2:]
    qk = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).bfloat16()
    s.q.copy_(qk[:, :Hq])
    k, v = qk[:, Hq:].reshape(s.R, Hkv, D // 8, 8), v.bfloat16()
    blk, slot = s.table[s.row_request, s.row_place // BLOCK].long(), s.row_place % BLOCK
    s.k[blk, :, :, slot] = k
    s.v[blk, :, :, slot] = v
    if not c["ring"]:
        return [s.q, s.k, s.v]
    kept = s.ring_rows
    s.k_ring[s.row_request[kept], s.ring_block, :, :, slot[kept]] = k[kept]
    s.v_ring[s.row_request[kept], s.ring_block, :, :, slot[kept]] = v[kept]
    return [s.q, s.k, s.v, s.k_ring, s.v_ring]


def _attn(c, s):
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    G, M = Hq // Hkv, s.pad.shape[1]
    tab = s.table.long()
    k = s.k[tab].float().permute(0, 2, 3, 5, 1, 4).reshape(B, Hkv, D, -1)               # [B][Hkv][D][N]
    v = s.v[tab].float().permute(0, 2, 1, 4, 3).reshape(B, Hkv, -1, D)
    q = s.q[s.pad].float().view(B, M, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, M * G, D)
    z = torch.matmul(q, k).mul_(1.0 / math.sqrt(D))
    at = torch.arange(v.shape[2], device="cuda")
    if c["kind"] == "cross":
        seen = (at < s.seq[:, None])[:, None, :].expand(B, M, -1)
    else:
        place = s.first[:, None, None] + torch.arange(M, device="cuda")[:, None]
        seen = at <= place
        if c["window"]:
            seen = seen & (at > place - c["window"])
    # nothing of what is not attended counts, whatever it holds
    held = at < s.seq[:, None]
    v = torch.where(held[:, None, :, None], v, torch.zeros((), device="cuda"))
    seen = seen[:, None, :, None, :].expand(B, 1, M, G, -1).reshape(B, 1, M * G, -1)
    z = z.masked_fill_(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(z.sub_(m))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (m + torch.log(total))[..., 0]
    o = o.view(B, Hkv, M, G, D).permute(0, 2, 1, 3, 4).reshape(B * M, Hq, D)[s.unpad]
    lse = lse.view(B, Hkv, M, G).permute(0, 2, 1, 3).reshape(B * M, Hq)[s.unpad]
    return [o.to(s.out.dtype), lse]


def _scores(c, s):
    z = s.z.double()
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(-1, keepdim=True)
    log = z - m - torch.log(total)
    p = e / total
    t = s.tokens.long()[:, None]
    zt = s.z.gather(1, t)
    ahead = (s.z > zt) | ((s.z == zt) & (torch.arange(c["V"], device="cuda") < t))
    entropy = -torch.where(p > 0, p * log, torch.zeros_like(p)).sum(-1)
    outputs = [log.gather(1, t)[:, 0].float(), (ahead.sum(-1) + 1).int(), entropy.float()]
    if c["top"]:
        order = torch.sort(s.z, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
        outputs += [log.gather(1, order).float(), order.int()]
    return outputs


_PLAIN = dict(append=_append, prompt=_attn, cross=_attn, scores=_scores)


def run(s):
    if not own:
        with torch.no_grad():
            return _PLAIN[s.c["kind"]](s.c, s)
    for call in s.calls:
        call()
    return s.outputs


# ---------------------------------------------------------------------------
# the same in 64 bits, by definition
# ---------------------------------------------------------------------------

def _exact_append(c, s):
    """Row by row of each request: heads normed, pairs turned as complex numbers, then one copy per place."""
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    outs = [s.q, s.k, s.v] + ([s.k_ring, s.v_ring] if c["ring"] else [])
    outs = [o.double() for o in outs]
    axis = [0] * (D // 2) if s.positions is None else [a for a, n in enumerate(s.axis_pairs) for _ in range(n)]
    freq = torch.tensor([math.exp(-2.0 * i / D * math.log(THETA)) for i in range(D // 2)], dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        lo, n, h = s.starts[b], s.rows[b], s.hist[b]
        x = s.qkv[lo:lo + n].double().view(n, -1, D)
        heads = [x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]]
        if c["norm"]:
            for i, gain in ((0, s.q_gain), (1, s.k_gain)):
                heads[i] = heads[i] / (heads[i].square().mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
        place = torch.arange(h, h + n, device="cuda").double()
        if s.positions is None:
            turn = place[:, None] * freq
        else:
            turn = s.positions[lo:lo + n].double()[:, axis] * freq
        turn = torch.polar(torch.ones_like(turn), turn)[:, None]
        for i in (0, 1):
            y = torch.complex(heads[i][..., :D // 2].contiguous(), heads[i][..., D // 2:].contiguous()) * turn
            heads[i] = torch.cat([y.real, y.imag], -1)
        outs[0][lo:lo + n] = heads[0]
        last, sb, rb = (h + n - 1) // BLOCK, -(-s.sink // BLOCK), -(-c["ring"] // BLOCK) + 2
        for j in range(h // BLOCK, last + 1):                      # whole or partial blocks
            p0, p1 = max(h, j * BLOCK), min(h + n, (j + 1) * BLOCK)
            kk = heads[1][p0 - h:p1 - h].permute(1, 2, 0)          # [Hkv][D][places]
            vv = heads[2][p0 - h:p1 - h].permute(1, 2, 0)
            where = [(outs[1], outs[2], int(s.table[b, j]))]
            if c["ring"] and (j < sb or j > last - rb):
                where.append((outs[3][b], outs[4][b], j if j < sb else sb + j % rb))
            for ko, vo, blk in where:
                ko[blk][:, :, p0 - j * BLOCK:p1 - j * BLOCK] = kk.reshape(Hkv, D // 8, 8, p1 - p0).transpose(2, 3)
                vo[blk][:, :, p0 - j * BLOCK:p1 - j * BLOCK] = vv
    return outs


def _exact_attn(c, s):
    """Request by request and KV head by KV head, 256 rows at a time: the softmax over the attended positions."""
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    G = Hq // Hkv
    out = torch.zeros(s.R, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((s.R, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n, rows = s.n[b], s.rows[b]
        if n == 0:
            continue
        blocks = s.table[b, :-(-n // BLOCK)].long()
        k, v = s.k[blocks], s.v[blocks]
        for g in range(Hkv):
            kg = k[:, g].double().permute(1, 3, 0, 2).reshape(D, -1)[:, :n]
            vg = v[:, g].double().permute(1, 0, 2).reshape(D, -1)[:, :n].t()
            for r0 in range(0, rows, 256):
                r1 = min(rows, r0 + 256)
                lo, hi = s.starts[b] + r0, s.starts[b] + r1
                z = torch.matmul(s.q[lo:hi, g * G:(g + 1) * G].double(), kg) / math.sqrt(D)     # [rows][G][n]
                if c["kind"] == "prompt":
                    ahead = torch.arange(n, device="cuda") - torch.arange(n - rows + r0, n - rows + r1, device="cuda")[:, None]
                    out_of = (ahead > 0) | (ahead <= -(c["window"] or 1 << 40))
                    z = torch.where(out_of[:, None], torch.tensor(-math.inf, dtype=torch.float64, device="cuda"), z)
                l = torch.logsumexp(z, -1)
                out[lo:hi, g * G:(g + 1) * G] = torch.matmul(torch.exp(z - l[..., None]), vg)
                lse[lo:hi, g * G:(g + 1) * G] = l
    return [out, lse]


def _exact_scores(c, s):
    """Row by row, from the sorted logits."""
    logprob, entropy, top = [], [], []
    for r in range(c["R"]):
        z = s.z[r].double()
        log = torch.log_softmax(z, 0)
        p = torch.exp(log)
        logprob.append(log[int(s.tokens[r])])
        entropy.append(-(p * log)[p > 0].sum())
        top.append(log.sort(descending=True).values[:c["top"]])
    outputs = [torch.stack(logprob), None, torch.stack(entropy)]
    return outputs + [torch.stack(top), None] if c["top"] else outputs


def exact(case, seed):
    fn = dict(append=_exact_append, scores=_exact_scores).get(case["kind"], _exact_attn)
    with torch.no_grad():
        return fn(case, prepare(case, seed))
