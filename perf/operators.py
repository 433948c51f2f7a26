"""The language-model operators around the verify step, as cases that can be timed and checked.

A decoding iteration's attention needs its keys and values in the cache, and its context has
to come from somewhere:

"append"  the queries and keys of new rows (a prompt's tokens, or the nodes of candidate trees)
          normalised per head where the model does that, rotated by their positions, and the keys
          and values written to the cache rows after each sequence's context;
"prompt"  causal attention of a batch's new tokens over their contexts and themselves: whole
          prompts packed without padding, chunks of long ones, or one token per sequence;
"prefix"  the verification attention of candidate trees whose sequences share a long prefix (a
          system prompt, or samples of one prompt), which is stored once.

With `own` false the operators are computed in plain torch operations, in 32 bits (angles in 64),
rounded once at the end; with `own` true by the package's functions.
"""

import math
import random

import torch

own = False

CHAIN = 16
DEPTH = 4
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _append(name, dtype, batch, rows_min, rows_max, ctx_min, ctx_max, hq, hkv, d, rot, tree=False, norm=False,
            interleaved=False, fused=False, far=0, mscale=1.0):
    return dict(name=name, kind="append", dtype=dtype, batch=batch, rows_min=rows_min, rows_max=rows_max,
                ctx_min=ctx_min, ctx_max=ctx_max, hq=hq, hkv=hkv, d=d, rot=rot, tree=tree, norm=norm,
                interleaved=interleaved, fused=fused, far=far, mscale=mscale)


def _prompt(name, dtype, batch, rows_min, rows_max, ctx_min, ctx_max, hq, hkv, d):
    return dict(name=name, kind="prompt", dtype=dtype, batch=batch, rows_min=rows_min, rows_max=rows_max,
                ctx_min=ctx_min, ctx_max=ctx_max, hq=hq, hkv=hkv, d=d)


def _prefix(name, dtype, batch, rows_min, rows_max, ctx_min, ctx_max, prefix, hq, hkv, d):
    return dict(name=name, kind="prefix", dtype=dtype, batch=batch, rows_min=rows_min, rows_max=rows_max,
                ctx_min=ctx_min, ctx_max=ctx_max, prefix=prefix, hq=hq, hkv=hkv, d=d)


def listed():
    return [
        # One interactive user's step: the 32 nodes of a candidate tree at 2k context. All latency.
        _append("append_tree_b1", "bf16", 1, 32, 32, 2048, 2048, 32, 8, 128, 128, tree=True),
        # A serving batch's trees of 20 to 48 nodes, a model that normalises queries and keys per
        # head, positions beyond its trained length (amplitude above one).
        _append("append_tree_norm_b16", "bf16", 16, 20, 48, 1024, 4096, 32, 8, 128, 128, tree=True, norm=True,
                far=100000, mscale=1.1386),
        # Prompts of a batch, read in place from the fused projection's output, interleaved pairs
        # over half the head.
        _append("append_prompt_b8", "bf16", 8, 501, 4001, 0, 0, 32, 8, 128, 64, interleaved=True, fused=True),
        # A small fp32 model's prompts, odd lengths, after some context.
        _append("append_f32_b3", "f32", 3, 37, 701, 11, 300, 12, 2, 64, 64, norm=True),
        # The smallest prompt call: a short fp32 prompt, four heads. All latency.
        _prompt("prompt_tiny_f32", "f32", 1, 101, 101, 0, 0, 4, 4, 64),
        # One long prompt.
        _prompt("prompt_8k_b1", "bf16", 1, 8192, 8192, 0, 0, 32, 8, 128),
        # A batch of prompts of different lengths, packed: the ordinary start of a serving batch.
        _prompt("prompt_ragged_b16", "bf16", 16, 1, 2048, 0, 0, 32, 8, 128),
        # Chunks of long prompts scheduled beside other work, head dim 64.
        _prompt("prompt_chunk_b4", "bf16", 4, 256, 512, 2000, 16000, 32, 8, 64),
        # One new token per sequence over long contexts: plain decoding.
        _prompt("prompt_token_b8", "bf16", 8, 1, 1, 4096, 32768, 32, 8, 128),
        # Verification of 48-node trees that share an 8k prefix and have short turns of their own.
        _prefix("prefix_tree_b16", "bf16", 16, 40, 48, 100, 1000, 8192, 32, 8, 128),
        # Many samples of one long prompt, one token at a time, head dim 64.
        _prefix("prefix_token_b32", "bf16", 32, 1, 1, 1, 500, 16384, 32, 8, 64),
        # Full-precision verification over a shared prefix.
        _prefix("prefix_f32_b4", "f32", 4, 12, 32, 50, 400, 2001, 32, 8, 128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: 1 to 32 sequences, 1 to 48 tree nodes or 1 to 8192 new tokens each,
    contexts of up to 32k tokens, prefixes of 100 to 16k, 1 to 32 heads over 1 to 8, head dims 64 and 128
    (and multiples of 16 up to 256 where no attention is computed)."""
    kind = rng.choice(["append", "prompt", "prompt", "prefix"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (32, 4), (16, 16), (8, 1), (12, 2), (20, 4), (28, 4)])
    d = rng.choice([64, 128])
    f32 = dtype == "f32"
    batch = _log_int(rng, 1, 16)
    case = dict(kind=kind, dtype=dtype, batch=batch, hq=hq, hkv=hkv)
    if kind == "append":
        d = rng.choice([64, 80, 96, 128, 128, 128, 256])
        tree = rng.random() < 0.5
        hi = 48 if tree else max(2, min(8192, 16000 * 128 * 48 // (d * (hq + 2 * hkv) * batch * (2 if f32 else 1))))
        a, b = sorted((_log_int(rng, 1, hi), _log_int(rng, 1, hi)))
        c, e = sorted((_log_int(rng, 1, 4096) - 1, _log_int(rng, 1, 4096) - 1))
        rot = rng.choice([d, d, d // 32 * 16])
        case.update(rows_min=a, rows_max=b, ctx_min=c, ctx_max=e, d=d, rot=rot, tree=tree, norm=rng.random() < 0.5,
                    interleaved=rng.random() < 0.5, fused=rng.random() < 0.5, far=rng.choice([0, 0, 30000, 1000000]),
                    mscale=rng.choice([1.0, 1.0, 1.25]))
    elif kind == "prompt":
        # At most about the largest listed case's products (8192 tokens of 32 heads of 128; an
        # eighth of them in fp32), and its cache rows.
        ctx = _log_int(rng, 1, 32768) - 1 if rng.random() < 0.5 else 0
        pairs = 8192 * 8192 // 2 * 32 * 128 // (hq * d * batch * (8 if f32 else 1))
        hi = int(math.sqrt(float(ctx) * ctx + 2.0 * pairs) - ctx)
        hi = max(1, min(8192, hi))
        ctx = min(ctx, 8 * 32768 * 8 // (batch * hkv) // (2 if f32 else 1))
        a, b = sorted((_log_int(rng, 1, hi), _log_int(rng, 1, hi)))
        case.update(rows_min=a, rows_max=b, ctx_min=ctx // 4, ctx_max=ctx, d=d)
    else:
        batch = _log_int(rng, 2, 32)
        hi = 48 if rng.random() < 0.7 else 1
        a, b = sorted((rng.randint(1, hi), rng.randint(1, hi)))
        most = 16 * 48 * 8192 * 32 * 128 // (batch * b * hq * d * (8 if f32 else 1))
        c, e = sorted((_log_int(rng, 1, 1000), _log_int(rng, 1, 1000)))
        case.update(batch=batch, rows_min=a, rows_max=b, ctx_min=c, ctx_max=e,
                    prefix=_log_int(rng, 100, max(101, min(16384, most))), d=d)
    return case


def _spread(lo, hi, n, phase):
    """n whole numbers spread over [lo, hi], the ends among them where there is room."""
    if n == 1:
        return [hi]
    mid = [lo + int((hi - lo) * (((i + 1) * 0.6180339887498949 + phase) % 1.0)) for i in range(n - 2)]
    return [hi] + mid + [lo]


def _sizes(case):
    """New rows and context lengths of the case's sequences."""
    rows = _spread(case["rows_min"], case["rows_max"], case["batch"], 0.0)
    ctx = _spread(case["ctx_min"], case["ctx_max"], case["batch"], 0.37)
    return rows, ctx


def _parents(rows, n_max, seed):
    """Trees of up to n_max nodes: a chain with branches of four nodes hung off random chain nodes."""
    rng = random.Random(seed)
    out = []
    for n in rows:
        p = list(range(-1, min(n, CHAIN) - 1))
        while len(p) < n:
            p.append(rng.randint(-1, CHAIN - 1) if (len(p) - CHAIN) % DEPTH == 0 else len(p) - 1)
        out.append(p + [-1] * (n_max - n))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], _DTYPES[case["dtype"]]
    batch, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    rows, ctx = _sizes(case)
    prefix = case.get("prefix", 0)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    def ints(v, t=torch.int32):
        return torch.tensor(v, dtype=t, device="cuda")

    # Each sequence's region of the cache: its context, its new rows and some room, in mixed order.
    regions = [c + n + 5 for c, n in zip(ctx, rows)]
    order = list(range(batch))
    random.Random(seed).shuffle(order)
    at, kv_off = prefix, [0] * batch
    for b in order:
        kv_off[b] = at
        at += regions[b]
    s = dict(case, kv_off=ints(kv_off, torch.int64), ctx_len=ints(ctx), n_rows=ints(rows), host_ctx=ctx, host_rows=rows,
             k_cache=normal(at, hkv, d), v_cache=normal(at, hkv, d), scale=1.0 / math.sqrt(d))
    n_max = max(rows)
    if kind == "prefix" or case.get("tree"):
        s["parent"] = ints(_parents(rows, n_max, seed))
        shape = (batch, n_max)
    else:
        off = [0]
        for n in rows:
            off.append(off[-1] + n)
        s["row_off"] = ints(off[:-1], torch.int64)
        shape = (off[-1],)
    if kind == "append":
        if case["fused"]:
            both = normal(*shape, hq + 2 * hkv, d)
            s["q"], s["k"], s["v"] = both.split([hq, hkv, hkv], dim=-2)
        else:
            s["q"], s["k"], s["v"] = normal(*shape, hq, d), normal(*shape, hkv, d), normal(*shape, hkv, d)
        half = case["rot"] // 2
        s["inv_freq"] = torch.tensor([500000.0 ** (-i / half) for i in range(half)], dtype=torch.float32, device="cuda")
        s["pos_off"] = ints([case["far"] + 7 * b for b in range(batch)]) if case["far"] else None
        s["q_weight"] = normal(d, std=0.1) + 1 if case["norm"] else None
        s["k_weight"] = normal(d, std=0.1) + 1 if case["norm"] else None
        s["out"] = torch.zeros(*shape, hq, d, dtype=dtype, device="cuda")
    else:
        s["q"] = normal(*shape, hq, d, std=1.5)
        s["out"] = torch.zeros(*shape, hq, d, dtype=dtype, device="cuda")
    return s


# --- the plain forms -----------------------------------------------------------------------------

def _closure(parent, live):
    """anc[b, n, m]: node m is node n or one of its ancestors (repeated squaring of the parent relation)."""
    n_max = parent.shape[1]
    eye = torch.eye(n_max, device=parent.device)
    step = torch.zeros(*parent.shape, n_max + 1, device=parent.device).scatter_(
        2, torch.where(live & (parent >= 0), parent, n_max).long().unsqueeze(2), 1.0)
    anc = eye + step[..., :n_max]
    for _ in range(max(1, (n_max - 1).bit_length())):
        anc = (anc @ anc).clamp_(max=1.0)
    return anc > 0


def _live(s, n_max):
    return torch.arange(n_max, device="cuda").unsqueeze(0) < s["n_rows"].unsqueeze(1)


def _plain_append(s):
    q, k, v, rot = s["q"], s["k"], s["v"], s["rot"]
    first = s["ctx_len"].long() if s["pos_off"] is None else s["ctx_len"].long() + s["pos_off"].long()
    if s["tree"]:
        batch, n_max = q.shape[:2]
        live = _live(s, n_max)
        depth = _closure(s["parent"], live).sum(2) - 1
        seq, step = live.nonzero(as_tuple=True)
        pos = first[seq] + depth[seq, step]
        flat = seq * n_max + step
        q, k, v = (x.reshape(batch * n_max, x.shape[-2], x.shape[-1])[flat] for x in (q, k, v))
    else:
        seq = torch.repeat_interleave(torch.arange(s["batch"], device="cuda"), s["n_rows"].long(), output_size=q.shape[0])
        step = torch.arange(q.shape[0], device="cuda") - s["row_off"][seq]
        pos, flat = first[seq] + step, torch.arange(q.shape[0], device="cuda")
    angle = pos.double().unsqueeze(1) * s["inv_freq"].double()
    cos, sin = (angle.cos() * s["mscale"]).float().unsqueeze(1), (angle.sin() * s["mscale"]).float().unsqueeze(1)

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
        if s["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
        else:
            a, b = x[..., : rot // 2], x[..., rot // 2: rot]
            y = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
        return torch.cat((y, x[..., rot:]), dim=-1).to(s["q"].dtype)

    out = s["out"]
    out.view(-1, out.shape[-2], out.shape[-1])[flat] = turned(q, s["q_weight"])
    slot = (s["kv_off"] + s["ctx_len"])[seq] + step
    s["k_cache"][slot] = turned(k, s["k_weight"])
    s["v_cache"][slot] = v
    return dict(q=out, k_cache=s["k_cache"], v_cache=s["v_cache"], status=torch.zeros(s["batch"], dtype=torch.int32, device="cuda"))


def _rows_by_head(x, hkv):
    """[batch, rows, hq, d] -> [batch, hkv, rows * group, d] in 32 bits."""
    b, n, hq, d = x.shape
    return x.float().view(b, n, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * (hq // hkv), d)


def _attend(q, k, v, visible, group, scale):
    """softmax(scale q k') v over the visible keys: q [b, h, rows * group, d], k and v [b, h, keys, d],
    visible [b, rows, keys]; a row that sees nothing gives zeros."""
    hidden = ~visible.repeat_interleave(group, dim=1).unsqueeze(1)
    x = (q @ k.transpose(2, 3)).mul_(scale).masked_fill_(hidden, -math.inf)
    x = x.sub_(x.amax(3, keepdim=True).clamp_(min=-1e30)).exp_()
    return (x @ v) / x.sum(3, keepdim=True).clamp_(min=1e-30)


def _heads_last(o, hq, rows):
    b, hkv, _, d = o.shape
    return o.view(b, hkv, rows, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(b, rows, hq, d)


def _plain_prompt(s):
    q, hq, hkv = s["q"], s["hq"], s["hkv"]
    n_max, t_max = max(s["host_rows"]), max(c + n for c, n in zip(s["host_ctx"], s["host_rows"]))
    live = _live(s, n_max)
    step = torch.arange(n_max, device="cuda")
    flat = (s["row_off"].unsqueeze(1) + step).clamp_(max=q.shape[0] - 1)
    tok = torch.arange(t_max, device="cuda")
    slot = (s["kv_off"].unsqueeze(1) + tok).clamp_(max=s["k_cache"].shape[0] - 1)
    last = s["ctx_len"].unsqueeze(1) + step
    visible = tok <= last.unsqueeze(2)
    k, v = (c[slot].float().transpose(1, 2).contiguous() for c in (s["k_cache"], s["v_cache"]))
    o = _attend(_rows_by_head(q[flat], hkv), k, v, visible, hq // hkv, s["scale"])
    s["out"][flat[live]] = _heads_last(o, hq, n_max)[live].to(q.dtype)
    return dict(o=s["out"])


def _plain_prefix(s):
    q, hq, hkv, prefix = s["q"], s["hq"], s["hkv"], s["prefix"]
    batch, n_max = q.shape[:2]
    live = _live(s, n_max)
    own_max = max(s["host_ctx"]) + n_max
    tok = torch.arange(own_max, device="cuda")
    slot = torch.cat((torch.arange(prefix, device="cuda").expand(batch, prefix),
                      (s["kv_off"].unsqueeze(1) + tok).clamp_(max=s["k_cache"].shape[0] - 1)), dim=1)
    node = tok - s["ctx_len"].unsqueeze(1)                     # node index of each own row, negative in the context
    anc = _closure(s["parent"], live)
    in_tree = anc.gather(2, node.clamp(0, n_max - 1).unsqueeze(1).expand(batch, n_max, own_max))
    own_visible = (node < 0).unsqueeze(1) | (in_tree & (node < n_max).unsqueeze(1))
    visible = torch.cat((torch.ones(batch, n_max, prefix, dtype=torch.bool, device="cuda"), own_visible), dim=2)
    k, v = (c[slot].float().transpose(1, 2).contiguous() for c in (s["k_cache"], s["v_cache"]))
    o = _heads_last(_attend(_rows_by_head(q, hkv), k, v, visible, hq // hkv, s["scale"]), hq, n_max)
    s["out"][live] = o[live].to(q.dtype)
    return dict(o=s["out"], status=torch.zeros(batch, dtype=torch.int32, device="cuda"))


# --- the package's calls -------------------------------------------------------------------------

def _own(s):
    import paper_2608_00531_amd as pc
    if s["kind"] == "append":
        q, status = pc.cure_rope_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["kv_off"], s["ctx_len"],
                                        s["n_rows"], s["inv_freq"], parent=s.get("parent"), row_off=s.get("row_off"),
                                        pos_off=s["pos_off"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6,
                                        interleaved=s["interleaved"], mscale=s["mscale"], n_max=max(s["host_rows"]),
                                        out=s["out"])
        return dict(q=q, k_cache=s["k_cache"], v_cache=s["v_cache"], status=status)
    if s["kind"] == "prompt":
        o, _ = pc.cure_prompt_attn(s["q"], s["k_cache"], s["v_cache"], s["row_off"], s["n_rows"], s["kv_off"],
                                   s["ctx_len"], s["host_rows"], s["host_ctx"], s["scale"], with_lse=False, out=s["out"])
        return dict(o=o)
    o, _, status = pc.cure_prefix_attn(s["q"], s["k_cache"], s["v_cache"], 0, s["prefix"], s["kv_off"], s["ctx_len"],
                                       s["n_rows"], s["parent"], s["host_ctx"], s["host_rows"], s["scale"],
                                       with_lse=False, out=s["out"])
    return dict(o=o, status=status)


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "prompt": _plain_prompt, "prefix": _plain_prefix}[state["kind"]](state)


def _pairs(case):
    """Sum over the query rows of the keys that they see (trees: the context and about half the chain and a branch)."""
    rows, ctx = _sizes(case)
    if case["kind"] == "prompt":
        return sum(n * c + n * (n + 1) // 2 for n, c in zip(rows, ctx))
    seen = 0
    for n, c, p in zip(rows, ctx, _parents(rows, max(rows), 0)):
        depth = []
        for m in range(n):
            depth.append(1 + (depth[p[m]] if p[m] >= 0 else 0))
        seen += n * (case["prefix"] + c) + sum(depth)
    return seen


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    rows, ctx = _sizes(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "append":
        values = sum(rows) * (hq + 2 * hkv) * d
        return {"bytes": 2 * values * size, "flops": 10 * values}
    keys = case.get("prefix", 0) + sum(n + c for n, c in zip(rows, ctx))
    return {"bytes": (2 * sum(rows) * hq + 2 * keys * hkv) * d * size, "flops": 4 * d * hq * _pairs(case)}


# --- the definitions, in 64 bits -----------------------------------------------------------------

def _tree_paths(parent, n):
    """Every node's root path (itself last), on the host."""
    paths = []
    for m in range(n):
        p = int(parent[m])
        paths.append((paths[p] if p >= 0 else []) + [m])
    return paths


def _exact_append(s):
    rows, ctx, rot = s["host_rows"], s["host_ctx"], s["rot"]
    out, kc, vc = s["out"].double(), s["k_cache"].double(), s["v_cache"].double()
    freq = s["inv_freq"].double()
    for b in range(s["batch"]):
        n, base = rows[b], ctx[b] + (int(s["pos_off"][b]) if s["pos_off"] is not None else 0)
        if s["tree"]:
            depth = [len(p) - 1 for p in _tree_paths(s["parent"][b].tolist(), n)]
            x = {c: s[c][b, :n].double() for c in "qkv"}
        else:
            depth = list(range(n))
            r0 = int(s["row_off"][b])
            x = {c: s[c][r0:r0 + n].double() for c in "qkv"}
        theta = torch.outer(torch.tensor(depth, dtype=torch.float64, device="cuda") + base, freq)
        turn = torch.polar(torch.full_like(theta, s["mscale"]), theta).unsqueeze(1)
        for c, w in (("q", s["q_weight"]), ("k", s["k_weight"])):
            y = x[c]
            if w is not None:
                y = y / ((y ** 2).mean(dim=-1, keepdim=True) + 1e-6).sqrt() * w.double()
            if s["interleaved"]:
                z = torch.complex(y[..., 0:rot:2].contiguous(), y[..., 1:rot:2].contiguous()) * turn
                y = torch.cat((torch.view_as_real(z).reshape(*y.shape[:-1], rot), y[..., rot:]), dim=-1)
            else:
                z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
                y = torch.cat((z.real, z.imag, y[..., rot:]), dim=-1)
            x[c] = y
        if s["tree"]:
            out[b, :n] = x["q"]
        else:
            out[r0:r0 + n] = x["q"]
        at = int(s["kv_off"][b]) + ctx[b]
        kc[at:at + n], vc[at:at + n] = x["k"], x["v"]
    return dict(q=out, k_cache=kc, v_cache=vc, status=None)


def _exact_rows(q, k, v, seen, scale):
    """One sequence: q [n, hq, d], k and v [keys, hkv, d] in 64 bits, seen [n, keys]; a head at a time."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    o = torch.empty_like(q)
    for h in range(hq):
        kh, vh = k[:, h // group].contiguous(), v[:, h // group].contiguous()
        x = torch.mm(q[:, h].contiguous(), kh.t().contiguous()) * scale
        x[~seen] = -math.inf
        o[:, h] = torch.softmax(x, dim=1) @ vh
    return o


def _exact_attention(s):
    rows, ctx = s["host_rows"], s["host_ctx"]
    out = s["out"].double()
    for b in range(s["batch"]):
        n, at = rows[b], int(s["kv_off"][b])
        span = slice(at, at + ctx[b] + n)
        k, v = s["k_cache"][span].double(), s["v_cache"][span].double()
        own_seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril_()
        if s["kind"] == "prefix":
            own_seen.zero_()
            for m, path in enumerate(_tree_paths(s["parent"][b].tolist(), n)):
                own_seen[m, torch.tensor(path, device="cuda")] = True
            k = torch.cat((s["k_cache"][:s["prefix"]].double(), k))
            v = torch.cat((s["v_cache"][:s["prefix"]].double(), v))
        seen = torch.cat((torch.ones(n, k.shape[0] - n, dtype=torch.bool, device="cuda"), own_seen), dim=1)
        if s["kind"] == "prefix":
            out[b, :n] = _exact_rows(s["q"][b, :n].double(), k, v, seen, s["scale"])
        else:
            r0 = int(s["row_off"][b])
            out[r0:r0 + n] = _exact_rows(s["q"][r0:r0 + n].double(), k, v, seen, s["scale"])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    o = _exact_attention(s)
    return dict(o=o) if case["kind"] == "prompt" else dict(o=o, status=None)
