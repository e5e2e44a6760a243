"""The operators of a decode step of many tenants: requests whose prompts begin alike, each tenant with its low-rank
adapter, each request with drafted tokens that one forward verifies.

Kinds of case (heads, widths and vocabularies of the repository's own workloads, other sizes of the same ranges by
`draw`):

  prefix   attention of L layers over a paged cache for groups of requests that share the first blocks of their
           histories; T current tokens per request (one, or one and its drafts), uncommitted candidates or already in
           the cache; the plan of the call, which a server makes once a step, is part of the pass
  lora     a dense layer with a low-rank adapter per row: fused projections in parts (query, key and value; gate and
           up), RMSNorm in front, SwiGLU or a residual behind
  verify   drafted tokens against the target's probabilities, by given random numbers: tokens accepted, next token
  commit   the accepted tokens' K/V of every layer into the paged cache

`run` computes them from elementary torch operations, or, where `own` is set, through paper_2609_20734_amd.  Sizes that
differ between requests are spread evenly over a case's range and dealt to the requests by the seed, so a case's work
does not depend on the seed.
"""
import math

import torch

own = False

BLOCK = 16
EPS = 1e-6

_LLAMA = dict(Hq=32, Hkv=8, D=128)      # Llama-3-8B-shaped heads
_QWEN = dict(Hq=16, Hkv=8, D=128)       # Qwen3-1.7B-shaped heads
_HYBRID = dict(Hq=64, Hkv=8, D=128)     # the hybrid workload's heads


def listed():
    return [
        # one layer of two chats behind a short system prompt: the smallest call, where latency counts
        dict(name="prefix-b2", kind="prefix", L=1, B=2, NG=1, T=1, **_QWEN, pre_lo=64, pre_hi=64, lo=17, hi=40, cur=True,
             ragged=False),
        # one layer of 32 chats of one assistant, 16K tokens of shared instructions and tools
        dict(name="prefix-b32", kind="prefix", L=1, B=32, NG=1, T=1, **_LLAMA, pre_lo=1024, pre_hi=1024, lo=40, hi=2100,
             cur=True, ragged=False),
        # eight requests of two tenants, up to four drafts each, four layers
        dict(name="prefix-drafts", kind="prefix", L=4, B=8, NG=2, T=5, **_QWEN, pre_lo=256, pre_hi=600, lo=33, hi=3000,
             cur=True, ragged=True),
        # 64 questions about one document of 64K tokens, heads of the hybrid workload, tokens in the cache already
        dict(name="prefix-b64-long", kind="prefix", L=2, B=64, NG=1, T=1, **_HYBRID, pre_lo=4096, pre_hi=4096, lo=3, hi=300,
             cur=False, ragged=False),
        # the fused query, key and value projection of a single request with an adapter
        dict(name="lora-qkv-b1", kind="lora", mode="plain", K=2048, parts="2048,1024,1024", r=16, B=1, adapters=8, none=0,
             norm=True, residual=False),
        # gate and up of 32 requests of 16 tenants, two requests without an adapter
        dict(name="lora-gu-b32", kind="lora", mode="swiglu", K=2048, parts="6144,6144", r=16, B=32, adapters=16, none=2,
             norm=True, residual=False),
        # the down projection of 32 requests with four drafts each, eight tenants of a larger rank
        dict(name="lora-down-b160", kind="lora", mode="plain", K=6144, parts="2048", r=64, B=160, adapters=8, none=0,
             norm=False, residual=True),
        # one request's four drafts, from a draft model's probabilities
        dict(name="verify-b1", kind="verify", B=1, K=4, V=151936, q=True, temps="one", masked=0),
        # a batch of 32 with mixed temperatures (greedy ones among them), some rows under a grammar's mask
        dict(name="verify-b32", kind="verify", B=32, K=4, V=151936, q=True, temps="mixed", masked=4),
        # drafts copied from the prompt (no draft probabilities), an odd vocabulary
        dict(name="verify-lookup-b8", kind="verify", B=8, K=7, V=50257, q=False, temps="mixed", masked=0),
        # one request's accepted tokens, the decoder's 28 layers
        dict(name="commit-b1", kind="commit", L=28, B=1, T=5, Hkv=8, D=128, lo=40, hi=40),
        # a batch of 32, 32 layers, up to eight tokens each
        dict(name="commit-b32", kind="commit", L=32, B=32, T=8, Hkv=8, D=128, lo=17, hi=400),
    ]


def _log(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    """One more case of the ranges above (heads, widths, batches, lengths, groups, drafts, ranks, vocabularies)."""
    kind = rng.choice(["prefix", "prefix", "prefix", "lora", "lora", "verify", "verify", "commit"])
    hkv = rng.choice([2, 4, 8])
    G, D = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128])
    if kind == "prefix":
        B, T, L = _log(rng, 1, 64), rng.choice([1, 1, 2, 3, 5, 8]), rng.choice([1, 1, 2, 4])
        top = min(4096, max(64, (1 << 24) // (B * T * G * hkv * L)))      # no more than the largest listed case
        a, b = _log(rng, 1, top), _log(rng, 1, top)
        lo, hi = _log(rng, 1, 2048), _log(rng, 1, 2048)
        return dict(kind=kind, L=L, B=B, NG=rng.randint(1, min(4, B)), T=T, Hq=hkv * G, Hkv=hkv, D=D, pre_lo=min(a, b),
                    pre_hi=max(a, b), lo=min(lo, hi), hi=max(lo, hi), cur=rng.random() < 0.7, ragged=rng.random() < 0.5)
    if kind == "lora":
        mode = rng.choice(["plain", "plain", "swiglu"])
        n = _log(rng, 256, 8192, 8) + rng.choice([0, 0, 1])
        parts = [n, n] if mode == "swiglu" else [n] if rng.random() < 0.5 else [n, max(1, n // 2), max(1, n // 2)]
        B = _log(rng, 1, 160)
        A = _log(rng, 1, 32)
        return dict(kind=kind, mode=mode, K=_log(rng, 256, 8192, 8), parts=",".join(map(str, parts)),
                    r=8 * rng.choice([1, 1, 2, 2, 3, 4, 8, 16]), B=B, adapters=A, none=rng.choice([0, 0, B // 4]),
                    norm=rng.random() < 0.5, residual=mode == "plain" and rng.random() < 0.5)
    if kind == "verify":
        B, K = _log(rng, 1, 48), rng.randint(0, 8)
        return dict(kind=kind, B=B, K=K, V=min(_log(rng, 1000, 152000), 24_000_000 // (B * (K + 1))), q=rng.random() < 0.6,
                    temps=rng.choice(["one", "mixed", "greedy"]), masked=rng.choice([0, 0, max(1, B // 4)]))
    lo, hi = _log(rng, 1, 600), _log(rng, 1, 600)
    return dict(kind=kind, L=rng.randint(1, 32), B=_log(rng, 1, 32), T=rng.randint(1, 8), Hkv=hkv, D=D, lo=min(lo, hi),
                hi=max(lo, hi))


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers, evenly spread over [lo, hi] (the last is hi)."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _group_sizes(B, NG):
    """NG uneven parts of B requests, none empty (they grow like the odd numbers)."""
    ends = [max(j + 1, min(B - (NG - 1 - j), round(B * (j + 1) ** 2 / NG ** 2))) for j in range(NG)]
    return [e - s for s, e in zip([0] + ends, ends)]


def _draft_counts(c):
    """Current tokens per request, ascending by request rank."""
    return [1 + i % c["T"] if c["ragged"] else c["T"] for i in range(c["B"])]


def _rows(c):
    """Output rows of each part, and all of them together."""
    parts = [int(p) for p in c["parts"].split(",")]
    return parts, sum(parts)


def _used_adapters(c):
    return min(c["adapters"], c["B"] - c["none"])


def work(case):
    c, k = case, case["kind"]
    if k == "prefix":
        pre = _spread(c["pre_lo"], c["pre_hi"], c["NG"])
        own_len, toks = _spread(c["lo"], c["hi"], c["B"]), _draft_counts(c)
        sizes = _group_sizes(c["B"], c["NG"])
        cached = sum(pre) * BLOCK + sum(n - 1 if c["cur"] else n - 1 + t for n, t in zip(own_len, toks))
        rows = sum(toks)
        # the operations count the mean tokens of a request with every prefix (which request is whose is dealt)
        scored = rows / c["B"] * (sum(p * BLOCK * m for p, m in zip(pre, sizes)) + sum(own_len)) + rows * c["T"] / 2
        kv = 4.0 * c["L"] * c["Hkv"] * c["D"]
        return dict(bytes=kv * (cached + (rows if c["cur"] else 0)) + c["L"] * rows * c["Hq"] * (6.0 * c["D"] + 4),
                    flops=4.0 * c["L"] * c["Hq"] * c["D"] * scored)
    if k == "lora":
        parts, n = _rows(c)
        out = n // 2 if c["mode"] == "swiglu" else n
        a = _used_adapters(c) * (c["K"] * len(parts) + n) * c["r"] * 2.0
        return dict(bytes=2.0 * n * c["K"] + a + 4.0 * c["B"] * (c["K"] + out * (2 if c["residual"] else 1)),
                    flops=2.0 * c["B"] * n * c["K"] + 2.0 * (c["B"] - c["none"]) * (c["K"] * len(parts) + n) * c["r"])
    if k == "verify":
        rows = c["B"] * (c["K"] + 1)
        # every target row, and the draft's row of the token that is drawn anew
        return dict(bytes=4.0 * c["V"] * (rows + (c["B"] if c["q"] else 0)) + 16.0 * rows, flops=4.0 * c["V"] * (rows + c["B"]))
    counts = [1 + i % c["T"] for i in range(c["B"])]
    return dict(bytes=2.0 * sum(counts) * c["L"] * c["Hkv"] * c["D"] * 4, flops=0)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 1000003 + 29)
        self.cpu = torch.Generator()
        self.cpu.manual_seed(int(seed) * 1000003 + 29)

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        t = torch.empty(*shape, dtype=dtype, device="cuda")
        flat = t.view(-1)
        for s in range(0, flat.numel(), 1 << 28):
            flat[s:s + (1 << 28)].normal_(mean, std, generator=self.g)
        return t

    def bf16(self, *shape, std=1.0):
        return self.normal(*shape, std=std, dtype=torch.bfloat16)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda")

    def perm(self, n):
        return torch.randperm(n, generator=self.cpu).tolist()


class _State:
    pass


def _i32(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


def _caches(c, r, s):
    s.k = r.bf16(c["L"], s.nb, c["Hkv"], c["D"] // 8, BLOCK, 8)
    s.v = r.bf16(c["L"], s.nb, c["Hkv"], c["D"], BLOCK)


def _prepare_prefix(c, r, s):
    L, B, T, NG, Hq, Hkv, D = (c[k] for k in ("L", "B", "T", "NG", "Hq", "Hkv", "D"))
    pre = _spread(c["pre_lo"], c["pre_hi"], NG)
    lens, toks = _spread(c["lo"], c["hi"], B), _draft_counts(c)
    deal, order = r.perm(B), r.perm(B)                       # lengths and tokens of a request; members in group order
    ends = torch.tensor(_group_sizes(B, NG)).cumsum(0).tolist()
    group = [0] * B
    for i, b in enumerate(order):
        group[b] = sum(i >= e for e in ends)
    s.n = [pre[group[b]] * BLOCK + lens[deal[b]] for b in range(B)]       # attended by the first current token
    s.tok = [toks[deal[b]] for b in range(B)]
    s.pre = [pre[group[b]] for b in range(B)]
    # a request's blocks beyond the prefix hold every current token too
    own_blocks = [-(-(s.n[b] + T) // BLOCK) - s.pre[b] for b in range(B)]
    s.mb = max(p + o for p, o in zip(s.pre, own_blocks))
    s.max_len = s.mb * BLOCK
    s.nb = sum(pre) + sum(own_blocks)
    ids, at = r.perm(s.nb), 0
    shared = []
    for p in pre:
        shared.append(ids[at:at + p])
        at += p
    table = torch.zeros(B, s.mb, dtype=torch.int32)
    for b in range(B):
        table[b, :s.pre[b]] = torch.tensor(shared[group[b]], dtype=torch.int32)
        table[b, s.pre[b]:s.pre[b] + own_blocks[b]] = torch.tensor(ids[at:at + own_blocks[b]], dtype=torch.int32)
        at += own_blocks[b]
    _caches(c, r, s)
    s.q = r.bf16(L, B, T, Hq, D)
    s.kc = s.vc = None
    if c["cur"]:
        s.kc, s.vc = r.bf16(L, B, T, Hkv, D), r.bf16(L, B, T, Hkv, D)
    s.table, s.seq, s.members = table.cuda(), _i32(s.n), _i32(order)
    s.start, s.prefix, s.n_tok = _i32([0] + ends), _i32(pre), _i32(s.tok)
    s.out = torch.zeros(L, B, T, Hq, D, device="cuda")
    s.lse = torch.zeros(L, B, T, Hq, device="cuda")
    # the groups as a padded array of members, the place of each request in it, and the blocks of both parts
    M = max(_group_sizes(B, NG))
    slots, place = [[0] * M for _ in range(NG)], [0] * B
    for j in range(NG):
        for i, b in enumerate(order[(ends[j - 1] if j else 0):ends[j]]):
            slots[j][i], place[b] = b, j * M + i
    s.slots, s.place = torch.tensor(slots).cuda(), torch.tensor(place).cuda()
    s.pre_table = torch.zeros(NG, max(pre), dtype=torch.long)
    for j in range(NG):
        s.pre_table[j, :pre[j]] = torch.tensor(shared[j])
    s.pre_table = s.pre_table.cuda()
    s.own_table = torch.zeros(B, max(own_blocks), dtype=torch.long)
    for b in range(B):
        s.own_table[b, :own_blocks[b]] = table[b, s.pre[b]:s.pre[b] + own_blocks[b]]
    s.own_table = s.own_table.cuda()
    s.first = torch.tensor(s.pre).cuda() * BLOCK             # the first position of a request's own blocks


def _prepare_lora(c, r, s):
    parts, n = _rows(c)
    K, B, R = c["K"], c["B"], c["r"]
    s.w = r.bf16(n, K, std=K ** -0.5)
    s.a = r.bf16(c["adapters"], len(parts) * R, K, std=K ** -0.5)
    s.b = r.bf16(c["adapters"], n, R, std=R ** -0.5)
    s.scale = 0.5 + r.uniform(c["adapters"])
    s.gain = r.normal(K, std=0.02, mean=1.0) if c["norm"] else None
    s.x = r.normal(B, K)
    out = n // 2 if c["mode"] == "swiglu" else n
    s.res = r.normal(B, out) if c["residual"] else None
    s.y = torch.zeros(B, out, device="cuda")
    order, names, used = r.perm(B), r.perm(c["adapters"]), max(1, _used_adapters(c))
    ids = [-1] * B
    for i, b in enumerate(order[c["none"]:]):
        ids[b] = names[i % used]
    s.ids = _i32(ids)
    s.part = torch.repeat_interleave(torch.arange(len(parts)), torch.tensor(parts)).cuda()


def _prepare_verify(c, r, s):
    B, K, V = c["B"], c["K"], c["V"]
    # peaked distributions: a few likely tokens over a long tail; the draft's are the target's with noise
    z = r.normal(B, K + 1, V, std=2.5)
    order = r.perm(B)
    temps = dict(one=[1.0], greedy=[0.0], mixed=[1.0, 0.0, 0.6, 1.3])[c["temps"]]
    s.temp = torch.tensor([temps[order[b] % len(temps)] for b in range(B)], device="cuda")
    s.n_drafts = _i32([K - (order[b] % 3 if K >= 3 and order[b] % 2 else 0) for b in range(B)])
    s.q = None
    s.tokens = torch.zeros(B, K, dtype=torch.int32, device="cuda")
    if K and c["q"]:
        t = torch.where(s.temp > 0, s.temp, torch.full_like(s.temp, 0.05))[:, None, None]
        s.q = torch.softmax((z[:, :K] + r.normal(B, K, V, std=0.4)) / t, -1)
        s.tokens = torch.multinomial(s.q.view(B * K, V), 1, generator=r.g).view(B, K).int()
    elif K:
        s.tokens = z[:, :K].argmax(-1).int()
        wild = r.uniform(B, K) < 0.2
        s.tokens = torch.where(wild, (r.uniform(B, K) * V).int().clamp(max=V - 1), s.tokens)
        z[:, :K].scatter_add_(2, s.tokens.long()[..., None], r.uniform(B, K, 1) * 9 + 3)
    masked = [b for b in range(B) if order[b] < c["masked"]]
    if masked:      # a grammar's mask: half the vocabulary out, by -infinity or by the type's lowest value
        out = r.uniform(len(masked), 1, V) < 0.5
        z[masked] = torch.where(out, torch.tensor(-math.inf, device="cuda"), z[masked])
        z[masked[0]] = z[masked[0]].clamp(min=torch.finfo(torch.float32).min)
    s.logits = z
    s.u = r.uniform(B, K + 1)
    s.accepted = torch.zeros(B, dtype=torch.int32, device="cuda")
    s.answer = torch.zeros(B, K + 1, dtype=torch.int32, device="cuda")


def _prepare_commit(c, r, s):
    L, B, T, Hkv, D = (c[k] for k in ("L", "B", "T", "Hkv", "D"))
    order = r.perm(B)
    lens = _spread(c["lo"], c["hi"], B)
    s.n = [lens[order[b]] for b in range(B)]
    need = [-(-(n + T - 1) // BLOCK) for n in s.n]
    s.mb, s.nb = max(need), sum(need)
    s.max_len = s.mb * BLOCK
    ids, at = r.perm(s.nb), 0
    table = torch.zeros(B, s.mb, dtype=torch.int32)
    for b in range(B):
        table[b, :need[b]] = torch.tensor(ids[at:at + need[b]], dtype=torch.int32)
        at += need[b]
    _caches(c, r, s)
    s.kc, s.vc = r.bf16(L, B, T, Hkv, D), r.bf16(L, B, T, Hkv, D)
    s.table, s.seq = table.cuda(), _i32(s.n)
    s.accepted = _i32([order[b] % T for b in range(B)])


_PREPARE = dict(prefix=_prepare_prefix, lora=_prepare_lora, verify=_prepare_verify, commit=_prepare_commit)


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
    B = c["B"]
    if c["kind"] == "prefix":
        shape = P.Shape(c["L"], B, c["Hq"], c["Hkv"], c["D"], s.mb, s.max_len, s.nb)
        inp = P.inputs(s.q, s.k, s.v, s.table, s.seq, 1.0 / math.sqrt(c["D"]), s.kc, s.vc)
        groups = P.prefix_groups(c["NG"], c["T"], s.start, s.members, s.prefix, s.n_tok if c["ragged"] else None)
        plan = _zeros(P.prefix_plan_size(shape, groups))
        ws = _zeros(P.prefix_workspace_size(shape, groups))
        return [P.prepare_prefix_plan(shape, inp, groups, plan),
                P.prepare_prefix_decode_attn(shape, inp, groups, plan, s.out, s.lse, ws)], [s.out, s.lse]
    if c["kind"] == "lora":
        parts, n = _rows(c)
        swiglu = c["mode"] == "swiglu"
        desc = P.dense_desc(c["K"], n // 2 if swiglu else n, P.DENSE_SWIGLU if swiglu else P.DENSE_PLAIN, s.w, s.gain, EPS)
        lora = P.lora_desc(c["adapters"], c["r"], parts, s.a, s.b, s.scale)
        ws = _zeros(P.lora_workspace_size(lora, B))
        return [P.prepare_dense_lora(desc, lora, B, s.x, s.res, s.y, s.ids, ws)], [s.y]
    if c["kind"] == "verify":
        desc = P.verify_desc(c["V"], c["K"], s.logits, s.tokens, s.u, s.q, s.n_drafts, s.temp)
        ws = _zeros(P.verify_workspace_size(B, c["V"], c["K"]))
        return [P.prepare_verify_drafts(desc, B, s.accepted, s.answer, ws)], [s.accepted, s.answer]
    shape = P.Shape(c["L"], B, c["Hkv"], c["Hkv"], c["D"], s.mb, s.max_len, s.nb)
    return [P.prepare_commit_drafts(shape, c["T"], s.k, s.v, s.table, s.seq, s.kc, s.vc, s.accepted, advance=False)], [s.k, s.v]


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _heads(kv, Hkv, keys):
    """Gathered blocks [L][X][blocks][Hkv][..] in fp32 as [L][X][Hkv][positions][D]."""
    L, X, N = kv.shape[:3]
    if keys:      # [D/8][16][8]
        return kv.permute(0, 1, 3, 2, 5, 4, 6).reshape(L, X, Hkv, N * BLOCK, -1).float()
    return kv.permute(0, 1, 3, 2, 5, 4).reshape(L, X, Hkv, N * BLOCK, -1).float()      # [D][16]


def _prefix(c, s):
    L, B, T, NG, Hq, Hkv, D = (c[k] for k in ("L", "B", "T", "NG", "Hq", "Hkv", "D"))
    G, M, scale = Hq // Hkv, s.slots.shape[1], 1.0 / math.sqrt(D)
    no = torch.tensor(-math.inf, device="cuda")
    q = s.q.float().view(L, B, T, Hkv, G, D).permute(0, 1, 3, 2, 4, 5)                 # [L][B][Hkv][T][G][D]
    # the prefix: a group's members side by side against its blocks
    kp, vp = _heads(s.k[:, s.pre_table], Hkv, True), _heads(s.v[:, s.pre_table], Hkv, False)
    qp = q[:, s.slots].permute(0, 1, 3, 2, 4, 5, 6).reshape(L, NG, Hkv, M * T * G, D)
    zp = torch.matmul(qp, kp.transpose(-1, -2)).mul_(scale)
    here = torch.arange(kp.shape[3], device="cuda") < s.prefix[:, None] * BLOCK
    zp = torch.where(here[:, None, None, :], zp, no)
    # the rest: each request against its own blocks, then its candidates
    ko, vo = _heads(s.k[:, s.own_table], Hkv, True), _heads(s.v[:, s.own_table], Hkv, False)
    t = torch.arange(T, device="cuda")
    at = s.first[:, None] + torch.arange(ko.shape[3], device="cuda")
    if c["cur"]:
        seen = (at < s.seq[:, None] - 1)[:, None, :].expand(B, T, -1)
        ko = torch.cat([ko, s.kc.float().permute(0, 1, 3, 2, 4)], 3)
        vo = torch.cat([vo, s.vc.float().permute(0, 1, 3, 2, 4)], 3)
        seen = torch.cat([seen, (t[None, :] <= t[:, None]).expand(B, T, T)], 2)
    else:
        seen = at[:, None, :] < s.seq[:, None, None] + t[:, None]
    zo = torch.matmul(q.reshape(L, B, Hkv, T * G, D), ko.transpose(-1, -2)).mul_(scale)
    zo = torch.where(seen[:, None, :, None, :].expand(B, 1, T, G, -1).reshape(B, 1, T * G, -1), zo, no)
    # one softmax over both
    mp = zp.amax(-1).view(L, NG, Hkv, M, T * G).permute(0, 1, 3, 2, 4).reshape(L, NG * M, Hkv, T * G)
    m = torch.maximum(mp[:, s.place], zo.amax(-1))                                     # [L][B][Hkv][T G]
    mg = m[:, s.slots].permute(0, 1, 3, 2, 4).reshape(L, NG, Hkv, M * T * G)
    zp = torch.exp(zp.sub_(mg[..., None]))
    zo = torch.exp(zo.sub_(m[..., None]))

    def per_request(x):
        return x.view(L, NG, Hkv, M, T * G, -1).permute(0, 1, 3, 2, 4, 5).reshape(L, NG * M, Hkv, T * G, -1)[:, s.place]

    total = per_request(zp.sum(-1))[..., 0] + zo.sum(-1)
    o = (per_request(torch.matmul(zp, vp)) + torch.matmul(zo, vo)) / total[..., None]
    valid = (t < s.n_tok[:, None])[None, :, :, None]
    out = o.view(L, B, Hkv, T, G, D).permute(0, 1, 3, 2, 4, 5).reshape(L, B, T, Hq, D)
    lse = (m + torch.log(total)).view(L, B, Hkv, T, G).permute(0, 1, 3, 2, 4).reshape(L, B, T, Hq)
    return [torch.where(valid[..., None], out, torch.zeros_like(out)), torch.where(valid, lse, torch.zeros_like(lse))]


def _lora(c, s):
    parts, n = _rows(c)
    x = s.x
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s.gain
    ids = s.ids.clamp(min=0).long()
    scale = torch.where(s.ids >= 0, s.scale[ids], torch.zeros_like(s.scale[ids]))
    t = torch.matmul(s.a[ids].float(), x[..., None])[..., 0] * scale[:, None]          # [B][parts r]
    t = t.view(c["B"], len(parts), c["r"])[:, s.part]                                  # [B][n][r]
    y = torch.matmul(x, s.w.float().t()) + (s.b[ids].float() * t).sum(-1)
    if c["mode"] == "swiglu":
        g, up = y[:, :n // 2], y[:, n // 2:]
        y = g / (1 + torch.exp(-g)) * up
    return [y + s.res if c["residual"] else y]


def _verify(c, s):
    B, K, V = c["B"], c["K"], c["V"]
    z = s.logits.double()
    m = z.amax(-1, keepdim=True)
    hot = torch.arange(V, device="cuda") == z.argmax(-1, keepdim=True)
    temp = s.temp.double()[:, None, None]
    e = torch.where(temp > 0, torch.exp((z - m) / torch.where(temp > 0, temp, torch.ones_like(temp))), hot.double())
    p = e / e.sum(-1, keepdim=True)
    i = torch.arange(K + 1, device="cuda")
    n = s.n_drafts.long()
    count = torch.zeros(B, dtype=torch.long, device="cuda")
    q = torch.zeros(B, K + 1, V, dtype=torch.float64, device="cuda")
    if K:
        x = s.tokens.long()
        q[:, :K] = s.q.double() if s.q is not None else torch.arange(V, device="cuda") == x[..., None]
        px = p[:, :K].gather(2, x[..., None])[..., 0]
        qx = q[:, :K].gather(2, x[..., None])[..., 0]
        ok = (s.u[:, :K].double() * qx < px) & (i[:K] < n[:, None])
        count = ok.long().cumprod(1).sum(1)
    b = torch.arange(B, device="cuda")
    row = p[b, count]
    w = torch.where((count < n)[:, None], (row - q[b, count]).clamp(min=0), row)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, row)
    cum = w.cumsum(-1)
    last = torch.where(w > 0, torch.arange(V, device="cuda"), torch.zeros(1, dtype=torch.long, device="cuda")).amax(-1)
    token = torch.minimum((cum <= s.u[:, K:].double() * cum[:, -1:]).sum(-1), last)
    drafts = torch.cat([s.tokens.long(), torch.zeros(B, 1, dtype=torch.long, device="cuda")], 1)
    answer = torch.where(i < count[:, None], drafts, torch.where(i == count[:, None], token[:, None], torch.full_like(drafts, -1)))
    return [count.int(), answer.int()]


def _commit(c, s):
    T, D = c["T"], c["D"]
    t = torch.arange(T, device="cuda")
    pos = (s.seq[:, None] - 1 + t).long()                                              # [B][T]
    blk, slot = s.table.long().gather(1, pos // BLOCK), pos % BLOCK
    keep = (t <= s.accepted[:, None])[None, :, :, None]
    k = s.kc.view(c["L"], c["B"], T, c["Hkv"], D // 8, 8)
    s.k[:, blk, :, :, slot] = torch.where(keep[..., None, None], k, s.k[:, blk, :, :, slot].permute(2, 0, 1, 3, 4, 5)) \
        .permute(1, 2, 0, 3, 4, 5)
    s.v[:, blk, :, :, slot] = torch.where(keep[..., None], s.vc, s.v[:, blk, :, :, slot].permute(2, 0, 1, 3, 4)) \
        .permute(1, 2, 0, 3, 4)
    return [s.k, s.v]


_PLAIN = dict(prefix=_prefix, lora=_lora, verify=_verify, commit=_commit)


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

def _exact_prefix(c, s):
    """Request by request: each row's softmax over its whole history, read through the request's own table."""
    L, B, T, Hq, Hkv, D = (c[k] for k in ("L", "B", "T", "Hq", "Hkv", "D"))
    out = torch.zeros(L, B, T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(L, B, T, Hq, dtype=torch.float64, device="cuda")
    for l in range(L):
        for b in range(B):
            n = s.n[b] - 1 if c["cur"] else s.n[b] + s.tok[b] - 1
            blocks = s.table[b, :-(-n // BLOCK)].long()
            k = s.k[l][blocks].double().permute(1, 2, 4, 0, 3).reshape(Hkv, D, -1)[..., :n]
            v = s.v[l][blocks].double().permute(1, 0, 3, 2).reshape(Hkv, -1, D)[:, :n]
            if c["cur"]:
                k = torch.cat([k, s.kc[l, b].double().permute(1, 2, 0)], 2)
                v = torch.cat([v, s.vc[l, b].double().permute(1, 0, 2)], 1)
            for t in range(s.tok[b]):
                e = s.n[b] + t
                z = torch.matmul(s.q[l, b, t].double().view(Hkv, -1, D), k[..., :e]) / math.sqrt(D)
                top = z.amax(-1, keepdim=True)
                w = torch.exp(z - top)
                norm = w.sum(-1, keepdim=True)
                out[l, b, t] = (torch.matmul(w, v[:, :e]) / norm).reshape(Hq, D)
                lse[l, b, t] = (top + torch.log(norm)).reshape(Hq)
    return [out, lse]


def _exact_lora(c, s):
    parts, n = _rows(c)
    y = torch.zeros_like(s.y, dtype=torch.float64)
    for b, a in enumerate(s.ids.tolist()):
        x = s.x[b].double()
        if c["norm"]:
            x = x / (x.square().mean() + EPS).sqrt() * s.gain.double()
        rows = s.w.double() @ x
        if a >= 0:
            low, at = s.a[a].double() @ x, 0
            for j, m in enumerate(parts):
                rows[at:at + m] += s.scale[a].double() * (s.b[a, at:at + m].double() @ low[j * c["r"]:(j + 1) * c["r"]])
                at += m
        if c["mode"] == "swiglu":
            rows = rows[:n // 2] * torch.sigmoid(rows[:n // 2]) * rows[n // 2:]
        y[b] = rows + s.res[b].double() if c["residual"] else rows
    return [y]


def exact(case, seed):
    fn = dict(prefix=_exact_prefix, lora=_exact_lora).get(case["kind"])
    if fn is None:
        return None      # tokens are whole numbers, the commit moves bytes
    with torch.no_grad():
        return fn(case, prepare(case, seed))
