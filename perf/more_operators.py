"""Operators of long sampled decoding around the verify step, as cases that can be timed and checked.

The context of a long conversation is held in 8 bits, the step's attention reads it there, and each
tree node's target token is drawn rather than the largest taken:

"pack"    committed rows of keys and values made blocks of 64 tokens with one scale for each block and
          head (in every layer, where the cache holds several), and blocks made rows again, as for a
          sequence that is opened for more tokens;
"attend"  attention of candidate trees, single tokens or chunks of prompts over a packed context, the
          rows behind it that are not packed yet, and themselves;
"sample"  one token drawn for each logits row with temperature, top-k, top-p and min-p, from given
          uniform numbers.

With `own` false the operators are computed in plain torch operations, in 32 bits (borders of roundings
and the sums that a drawn token depends on in 64), rounded once at the end; with `own` true by the
package's functions.
"""

import math
import random

import torch

own = False

BLOCK = 64
CHAIN = 16
DEPTH = 4
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _pack(name, dtype, layers, batch, rows_min, rows_max, done_max, hkv, d):
    return dict(name=name, kind="pack", dtype=dtype, layers=layers, batch=batch, rows_min=rows_min, rows_max=rows_max,
                done_max=done_max, hkv=hkv, d=d)


def _attend(name, dtype, batch, rows_min, rows_max, packed_min, packed_max, open_min, open_max, hq, hkv, d, tree):
    return dict(name=name, kind="attend", dtype=dtype, batch=batch, rows_min=rows_min, rows_max=rows_max,
                packed_min=packed_min, packed_max=packed_max, open_min=open_min, open_max=open_max, hq=hq, hkv=hkv, d=d,
                tree=tree)


def _sample(name, dtype, batch, rows_min, rows_max, vocab, filters):
    return dict(name=name, kind="sample", dtype=dtype, batch=batch, rows_min=rows_min, rows_max=rows_max, vocab=vocab,
                filters=filters)


def listed():
    return [
        # One interactive user has filled a block: its 64 rows in all 32 layers.
        _pack("pack_block_l32_b1", "bf16", 32, 1, 64, 64, 2048, 8, 128),
        # A batch's prompts, one layer, right after their attention; the last block of each is partly filled.
        _pack("pack_prompt_b8", "bf16", 1, 8, 501, 4001, 0, 8, 128),
        # A small fp32 model's contexts, odd lengths.
        _pack("pack_f32_b3", "f32", 4, 3, 37, 701, 640, 2, 64),
        # One interactive user's step: the 32 nodes of a candidate tree at 2k context, some of it not packed yet.
        _attend("attend_tree_b1", "bf16", 1, 32, 32, 2048, 2048, 21, 21, 32, 8, 128, True),
        # A serving batch's trees of 20 to 48 nodes.
        _attend("attend_tree_b16", "bf16", 16, 20, 48, 1024, 4096, 0, 63, 32, 8, 128, True),
        # Long contexts, 32 nodes each.
        _attend("attend_tree_32k_b4", "bf16", 4, 32, 32, 32768, 32768, 0, 63, 32, 8, 128, True),
        # One new token per sequence over long contexts: plain decoding.
        _attend("attend_token_b8", "bf16", 8, 1, 1, 4096, 32768, 0, 63, 32, 8, 128, False),
        # Chunks of new turns on packed contexts, head dim 64, the last block partly filled.
        _attend("attend_chunk_b4", "bf16", 4, 256, 512, 2000, 16000, 0, 100, 32, 8, 64, False),
        # A small fp32 model's trees.
        _attend("attend_f32_b2", "f32", 2, 7, 12, 100, 640, 3, 30, 4, 4, 64, True),
        # One row, the usual filters. All latency.
        _sample("sample_b1", "bf16", 1, 1, 1, 128256, "k_p"),
        # The target's tokens for every node of a serving batch's trees, each sequence with settings of its own.
        _sample("sample_tree_b16", "bf16", 16, 20, 48, 128256, "mixed"),
        # fp32 logits of an odd vocabulary, the nucleus alone.
        _sample("sample_f32_b4", "f32", 4, 9, 17, 50257, "p"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: 1 to 16 sequences; 1 to 4001 rows to pack in 1 to 32 layers; 1 to 48 tree nodes,
    single tokens or 1 to 512 new ones on up to 32k packed tokens; 1 to 768 logits rows of 1000 to 262144 entries."""
    kind = rng.choice(["pack", "attend", "attend", "sample"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (32, 4), (16, 16), (8, 1), (12, 2), (20, 4), (28, 4)])
    d = rng.choice([64, 128])
    f32 = dtype == "f32"
    batch = _log_int(rng, 1, 16)
    case = dict(kind=kind, dtype=dtype, batch=batch)
    if kind == "pack":
        layers = rng.choice([1, 1, 4, 32])
        hi = max(2, min(4001, 18000 * 8 * 128 // (hkv * d * batch * layers * (2 if f32 else 1))))
        a, b = sorted((_log_int(rng, 1, hi), _log_int(rng, 1, hi)))
        case.update(layers=layers, rows_min=a, rows_max=b, done_max=BLOCK * rng.randint(0, 20), hkv=hkv, d=d)
    elif kind == "attend":
        form = rng.choice(["tree", "tree", "token", "chunk"])
        hi = {"tree": 48, "token": 1, "chunk": 512}[form]
        a, b = sorted((_log_int(rng, 1, hi), _log_int(rng, 1, hi)))
        # At most the largest listed case's products (an eighth in fp32) and its packed tokens.
        most = 4 * 512 * 16000 * 32 * 64 // (batch * b * hq * d * (16 if f32 else 1))
        most = max(2, min(32768, most, 4 * 32768 * 8 * 128 // (batch * hkv * d)))
        c, e = sorted((_log_int(rng, 1, most) - 1, _log_int(rng, 1, most) - 1))
        o, p = sorted((rng.randint(0, 63), rng.randint(0, 130)))
        case.update(rows_min=a, rows_max=b, packed_min=c, packed_max=e, open_min=o, open_max=p, hq=hq, hkv=hkv, d=d,
                    tree=form == "tree")
    else:
        vocab = rng.choice([_log_int(rng, 1000, 262144), 32000, 128256])
        hi = max(1, min(48, 16 * 48 * 128256 // (vocab * batch * (4 if f32 else 1))))
        a, b = sorted((rng.randint(1, hi), rng.randint(1, hi)))
        case.update(rows_min=a, rows_max=b, vocab=vocab, filters=rng.choice(["k_p", "p", "min_p", "none", "mixed", "mixed"]))
    return case


def _spread(lo, hi, n, phase):
    """n whole numbers spread over [lo, hi], the ends among them where there is room."""
    if n == 1:
        return [hi]
    mid = [lo + int((hi - lo) * (((i + 1) * 0.6180339887498949 + phase) % 1.0)) for i in range(n - 2)]
    return [hi] + mid + [lo]


def _sizes(case):
    """New rows, packed tokens and open rows of the case's sequences."""
    rows = _spread(case["rows_min"], case["rows_max"], case["batch"], 0.0)
    if case["kind"] == "pack":
        return rows, [n // BLOCK * BLOCK for n in _spread(0, case["done_max"], case["batch"], 0.37)], None
    if case["kind"] == "sample":
        return rows, None, None
    return (rows, _spread(case["packed_min"], case["packed_max"], case["batch"], 0.37),
            _spread(case["open_min"], case["open_max"], case["batch"], 0.71))


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


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


def _places(sizes, seed, first=0):
    """Where each sequence's region begins when they lie in mixed order, and the end of them all."""
    order = list(range(len(sizes)))
    random.Random(seed).shuffle(order)
    at, off = first, [0] * len(sizes)
    for b in order:
        off[b] = at
        at += sizes[b]
    return off, at


#: Temperature, top-k (0: all), top-p and min-p that sequences of a mixed batch ask for in turn.
_MIXED = [(0.7, 50, 0.9, 0.0), (1.0, 0, 0.95, 0.0), (0.0, 0, 1.0, 0.0), (0.6, 20, 0.95, 0.0), (1.0, 0, 1.0, 0.0), (1.3, 0, 1.0, 0.05),
          (0.8, 1000, 0.99, 0.02)]


def _settings(case):
    """The sampling settings of the case's sequences; None: the call goes without that filter."""
    n, filters = case["batch"], case["filters"]
    mix = [_MIXED[b % len(_MIXED)] for b in range(n)]
    if filters == "k_p":
        return [0.6 + 0.1 * (b % 5) for b in range(n)], [20 + 15 * (b % 3) for b in range(n)], [0.8 + 0.05 * (b % 4) for b in range(n)], None
    if filters == "p":
        return [1.0] * n, None, [0.9 + 0.02 * (b % 4) for b in range(n)], None
    if filters == "min_p":
        return [1.0 + 0.25 * (b % 3) for b in range(n)], None, None, [0.02 + 0.03 * (b % 4) for b in range(n)]
    if filters == "none":
        return [0.8 + 0.2 * (b % 3) for b in range(n)], None, None, None
    return tuple([m[i] for m in mix] for i in range(4))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], _DTYPES[case["dtype"]]
    batch = case["batch"]
    rows, packed, ctx = _sizes(case)

    def normal(*shape, std=1.0, dtype=dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    def device(v, t=torch.int32):
        return None if v is None else torch.tensor(v, dtype=t, device="cuda")

    s = dict(case, n_rows=device(rows), host_rows=rows)
    if kind == "sample":
        n_max, vocab = max(rows), case["vocab"]
        # A broad body, and some dozens of tokens that the model holds for likely.
        x = normal(batch, n_max, vocab, std=2.0, dtype=torch.float32)
        few = min(64, vocab // 4)
        at = torch.randint(vocab, (batch, n_max, few), device="cuda", generator=gen)
        x.scatter_(2, at, 4.0 + 12.0 * torch.rand(batch, n_max, few, device="cuda", generator=gen) ** 2)
        t, k, p, m = _settings(case)
        s.update(logits=x.to(dtype), uniform=torch.rand(batch, n_max, device="cuda", generator=gen), temperature=device(t, torch.float32),
                 top_k=device(k), top_p=device(p, torch.float32), min_p=device(m, torch.float32))
        return s
    hkv, d = case["hkv"], case["d"]
    if kind == "pack":
        layers = (case["layers"],) if case["layers"] > 1 else ()
        kv_off, end = _places([n + 3 for n in rows], seed)
        blk_off, blocks = _places([_blocks(p) + _blocks(n) for p, n in zip(packed, rows)], seed + 1)
        # Heads of different sizes, and some columns that are always large.
        loud = 1.0 + 4.0 * (torch.rand(hkv, d, device="cuda", generator=gen) < 0.03)
        k = (normal(*layers, end, hkv, d, dtype=torch.float32) * loud * torch.linspace(0.5, 2.0, hkv, device="cuda").unsqueeze(1)).to(dtype)
        s.update(k=k, v=normal(*layers, end, hkv, d), kv_off=device(kv_off, torch.int64), blk_off=device(blk_off, torch.int64),
                 packed_len=device(packed), packed=packed,
                 pk=torch.zeros(*layers, blocks, hkv, BLOCK * d, dtype=torch.int8, device="cuda"),
                 pv=torch.zeros(*layers, blocks, hkv, BLOCK * d, dtype=torch.int8, device="cuda"),
                 k_scale=torch.zeros(*layers, blocks, hkv, device="cuda"), v_scale=torch.zeros(*layers, blocks, hkv, device="cuda"),
                 k_back=torch.zeros(*layers, end, hkv, d, dtype=dtype, device="cuda"),
                 v_back=torch.zeros(*layers, end, hkv, d, dtype=dtype, device="cuda"))
        return s
    blk_off, blocks = _places([_blocks(p) + 1 for p in packed], seed + 1)
    kv_off, end = _places([c + n + 5 for c, n in zip(ctx, rows)], seed)

    def bytes_(std):
        return normal(blocks, hkv, BLOCK * d, std=std, dtype=torch.float32).round_().clamp_(-127, 127).to(torch.int8)

    def scales():
        return (4.0 + torch.rand(blocks, hkv, device="cuda", generator=gen)) / 127

    hq, n_max = case["hq"], max(rows)
    s.update(pk=bytes_(32.0), pv=bytes_(32.0), k_scale=scales(), v_scale=scales(), blk_off=device(blk_off, torch.int64),
             packed_len=device(packed), packed=packed, k=normal(end, hkv, d), v=normal(end, hkv, d), kv_off=device(kv_off, torch.int64),
             ctx_len=device(ctx), ctx=ctx, scale=1.0 / math.sqrt(d))
    if case["tree"]:
        s["parent"] = device(_parents(rows, n_max, seed))
        shape = (batch, n_max)
    else:
        off = [0]
        for n in rows:
            off.append(off[-1] + n)
        s["row_off"] = device(off[:-1], torch.int64)
        shape = (off[-1],)
    s["q"] = normal(*shape, hq, d, std=1.5)
    s["out"] = torch.zeros(*shape, hq, d, dtype=dtype, device="cuda")
    return s


# --- the plain forms -----------------------------------------------------------------------------

def _token_major(bytes_, d, values):
    """Blocks' bytes [..., hkv, 64 d] as tokens [..., hkv, 64, d].

    A block of keys holds, for its two halves of 32 tokens and each 32 columns, 1 KB that 64 lanes of 16
    bytes make: lane 32 h + t the columns 16 h .. 16 h + 15 of token t. One of values has, for the same
    pieces, lane 32 h + m column m of the tokens 8 a + 4 h + c (a, c < 4), in the order (a, c).
    """
    lead = bytes_.shape[:-1]
    n = len(lead)
    if values:
        x = bytes_.view(*lead, 2, d // 32, 2, 32, 4, 4)               # half, columns / 32, h, m, a, c
        order = (0, 4, 2, 5, 1, 3)
    else:
        x = bytes_.view(*lead, 2, d // 32, 2, 32, 16)                 # half, columns / 32, h, token, column
        order = (0, 3, 1, 2, 4)
    return x.permute(*range(n), *(n + i for i in order)).reshape(*lead, BLOCK, d)


def _rows_of(s):
    """Sequence and place within it of every row to pack."""
    seq = torch.repeat_interleave(torch.arange(s["batch"], device="cuda"), s["n_rows"].long(), output_size=sum(s["host_rows"]))
    step = torch.arange(seq.shape[0], device="cuda") - (s["n_rows"].cumsum(0) - s["n_rows"])[seq]
    return seq, step


def _plain_pack(s):
    layered = s["k"].dim() == 4
    seq, step = _rows_of(s)
    src = s["kv_off"][seq] + step
    blk = s["blk_off"][seq] + (s["packed_len"][seq] + step) // BLOCK
    out = dict(status=torch.zeros(s["batch"], dtype=torch.int32, device="cuda"))
    touched = torch.zeros(s["k_scale"].shape[-2], dtype=torch.bool, device="cuda")
    touched[blk] = True

    def one(x, scale, back):
        if not layered:
            x, scale, back = x.unsqueeze(0), scale.unsqueeze(0), back.unsqueeze(0)
        rows = x[:, src].float()
        high = torch.zeros_like(scale).index_reduce_(1, blk, rows.abs().amax(3), "amax")
        scale[:, touched] = high[:, touched] / 127
        # Borders between two integers in 64 bits.
        top = high[:, blk].unsqueeze(3).double()
        q = torch.where(top > 0, (rows.double() * 127 / top).round(), 0.0).float()
        back[:, src] = (q * scale[:, blk].unsqueeze(3)).to(back.dtype)

    one(s["k"], s["k_scale"], s["k_back"])
    one(s["v"], s["v_scale"], s["v_back"])
    return dict(out, k=s["k_back"], v=s["v_back"], k_scale=s["k_scale"], v_scale=s["v_scale"])


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


def _plain_attend(s):
    q, hq, hkv, d = s["q"], s["hq"], s["hkv"], s["d"]
    group, n_max = hq // hkv, max(s["host_rows"])
    step = torch.arange(n_max, device="cuda")
    live = step < s["n_rows"].unsqueeze(1)
    flat = (torch.arange(s["batch"], device="cuda").unsqueeze(1) * n_max if s["tree"] else s["row_off"].unsqueeze(1)) + step
    flat = flat.clamp_(max=q.numel() // (hq * d) - 1)
    packed_max = max(s["packed"])
    own_max = max(c + n for c, n in zip(s["ctx"], s["host_rows"]))
    old, tok = torch.arange(packed_max, device="cuda"), torch.arange(own_max, device="cuda")
    node = tok - s["ctx_len"].unsqueeze(1)                     # index among the new rows, negative in the context
    if s["tree"]:
        anc = _closure(s["parent"], live)
        seen = anc.gather(2, node.clamp(0, n_max - 1).unsqueeze(1).expand(-1, n_max, own_max)) & (node < n_max).unsqueeze(1)
        seen = seen | (node < 0).unsqueeze(1)
    else:
        seen = node.unsqueeze(1) <= step.unsqueeze(1)
    visible = torch.cat(((old < s["packed_len"].unsqueeze(1)).unsqueeze(1).expand(-1, n_max, packed_max), seen), dim=2)
    old_slot = (s["blk_off"].unsqueeze(1) * BLOCK + old).clamp_(max=s["pk"].shape[0] * BLOCK - 1)
    own_slot = (s["kv_off"].unsqueeze(1) + tok).clamp_(max=s["k"].shape[0] - 1)

    def keys(bytes_, scale, rows, values):
        x = _token_major(bytes_, d, values).float() * scale.view(*scale.shape, 1, 1)
        x = x.transpose(1, 2).reshape(-1, hkv, d)
        return torch.cat((x[old_slot], rows[own_slot].float()), dim=1).transpose(1, 2).contiguous()

    k, v = keys(s["pk"], s["k_scale"], s["k"], False), keys(s["pv"], s["v_scale"], s["v"], True)
    x = q.view(-1, hq, d)[flat].float().view(-1, n_max, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(-1, hkv, n_max * group, d)
    x = (x @ k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~visible.repeat_interleave(group, dim=1).unsqueeze(1), -math.inf)
    x = x.sub_(x.amax(3, keepdim=True).clamp_(min=-1e30)).exp_()
    o = (x @ v) / x.sum(3, keepdim=True).clamp_(min=1e-30)
    o = o.view(-1, hkv, n_max, group, d).permute(0, 2, 1, 3, 4).reshape(-1, n_max, hq, d)
    s["out"].view(-1, hq, d)[flat[live]] = o[live].to(q.dtype)
    return dict(o=s["out"], status=torch.zeros(s["batch"], dtype=torch.int32, device="cuda"))


def _plain_sample(s):
    """Entries in the order (value descending, index ascending). Weights exp((x - max) / T); what lies more than
    64 T below the largest has none. Kept is a run from the front: top-k, of that the fewest whose weight
    reaches top-p of the whole, of those what has at least min-p of the largest's weight."""
    x, order = torch.sort(s["logits"].float(), dim=2, descending=True, stable=True)
    x, vocab = x.double(), x.shape[2]
    each = lambda name, other: torch.full((s["batch"], 1, 1), other, dtype=torch.float64, device="cuda") if s[name] is None \
        else s[name].double().view(-1, 1, 1)  # noqa: E731
    t, top_k, top_p, min_p = each("temperature", 1.0), each("top_k", 0.0), each("top_p", 1.0), each("min_p", 0.0)
    below = x[..., :1] - x
    greedy = t == 0
    w = torch.exp(-below / torch.where(greedy, 1.0, t))
    rank = torch.arange(vocab, device="cuda")
    keep = (below <= 64 * t) & ~(greedy & (rank > 0)) & ((rank < top_k) | (top_k <= 0))
    w = w.masked_fill_(~keep, 0.0)
    upto = w.cumsum(2)
    keep &= ((upto - w < top_p * upto[..., -1:]) | (top_p >= 1) | (rank == 0)) & ((w >= min_p) | (rank == 0))
    n = keep.sum(2)
    whole = upto.gather(2, n.unsqueeze(2) - 1)
    at = torch.minimum((upto <= s["uniform"].double().unsqueeze(2) * whole).sum(2), n - 1).unsqueeze(2)
    live = torch.arange(x.shape[1], device="cuda") < s["n_rows"].unsqueeze(1)
    return dict(token=torch.where(live, order.gather(2, at).squeeze(2), -2).int(),
                logprob=torch.where(live, (w.gather(2, at) / whole).log().squeeze(2), -math.inf).float(),
                kept=torch.where(live, n, 0).int())


# --- the package's calls -------------------------------------------------------------------------

def _own(s):
    import paper_2608_00531_amd as pc
    if s["kind"] == "sample":
        return pc.cure_sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                              min_p=s["min_p"], n_rows=s["n_rows"])
    if s["kind"] == "pack":
        status = pc.cure_kv_pack(s["k"], s["v"], s["kv_off"], s["n_rows"], s["pk"], s["pv"], s["k_scale"], s["v_scale"], s["blk_off"],
                                 s["packed_len"], n_max=max(s["host_rows"]))
        pc.cure_kv_unpack(s["pk"], s["pv"], s["k_scale"], s["v_scale"], s["blk_off"], s["packed_len"], s["k_back"], s["v_back"],
                          s["kv_off"], s["n_rows"], n_max=max(s["host_rows"]))
        return dict(status=status, k=s["k_back"], v=s["v_back"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    o, _, status = pc.cure_packed_attn(s["q"], s["pk"], s["pv"], s["k_scale"], s["v_scale"], s["blk_off"], s["packed_len"], s["k"],
                                       s["v"], s["kv_off"], s["ctx_len"], s["n_rows"], s["packed"], s["ctx"], s["host_rows"],
                                       s["scale"], parent=s.get("parent"), row_off=s.get("row_off"), with_lse=False, out=s["out"])
    return dict(o=o, status=status)


def run(state):
    if own:
        return _own(state)
    return {"pack": _plain_pack, "attend": _plain_attend, "sample": _plain_sample}[state["kind"]](state)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    rows, packed, ctx = _sizes(case)
    if case["kind"] == "sample":
        n = sum(rows) * case["vocab"]
        return {"bytes": n * size, "flops": 2 * n}
    hkv, d = case["hkv"], case["d"]
    if case["kind"] == "pack":
        n = 2 * case["layers"] * sum(rows) * hkv * d               # read, packed, read again, written
        scales = 2 * case["layers"] * sum(_blocks(r) for r in rows) * hkv * 4
        return {"bytes": n * (2 * size + 2) + 2 * scales, "flops": 4 * n}
    seen = 0
    for n, p, c, par in zip(rows, packed, ctx, _parents(rows, max(rows), 0)):
        depth = []
        for m in range(n):
            depth.append(1 + (m if not case["tree"] else depth[par[m]] if par[m] >= 0 else 0))
        seen += n * (p + c) + sum(depth)
    values = (2 * sum(rows) * case["hq"] + 2 * (sum(rows) + sum(ctx)) * hkv) * d * size + 2 * sum(packed) * hkv * d
    return {"bytes": values + 2 * sum(_blocks(p) for p in packed) * hkv * 4, "flops": 4 * d * case["hq"] * seen}


# --- the definitions, in 64 bits -----------------------------------------------------------------

def _exact_pack(s):
    out = dict(status=None)
    for name in "kv":
        x, back, scale = s[name].double(), s[name + "_back"].double(), s[name + "_scale"].double()
        if x.dim() == 3:
            x, back, scale = x.unsqueeze(0), back.unsqueeze(0), scale.unsqueeze(0)
        for b, n in enumerate(s["host_rows"]):
            src, blk = int(s["kv_off"][b]), int(s["blk_off"][b]) + s["packed"][b] // BLOCK
            for i in range(0, n, BLOCK):
                rows = x[:, src + i:src + min(i + BLOCK, n)]
                step = rows.abs().amax(dim=(1, 3)) / 127
                scale[:, blk + i // BLOCK] = step
                step = step.view(step.shape[0], 1, -1, 1)
                back[:, src + i:src + i + rows.shape[1]] = torch.round(rows / step) * step
        out[name], out[name + "_scale"] = (back, scale) if s[name].dim() == 4 else (back[0], scale[0])
    return out


def _places_in_block(d, device):
    """Byte of (token, column) in a block of keys and in one of values."""
    t, c = torch.arange(BLOCK, device=device).unsqueeze(1), torch.arange(d, device=device)
    piece = ((t // 32) * (d // 32) + c // 32) * 1024
    k = piece + (c % 32) // 16 * 512 + (t % 32) * 16 + c % 16
    v = piece + (t // 4) % 2 * 512 + (c % 32) * 16 + (t % 32) // 8 * 4 + t % 4
    return k, v


def _exact_attend(s):
    out, d, group = s["out"].double(), s["d"], s["hq"] // s["hkv"]
    at_k, at_v = _places_in_block(d, "cuda")
    for b, n in enumerate(s["host_rows"]):
        packed, ctx, at, blk = s["packed"][b], s["ctx"][b], int(s["kv_off"][b]), int(s["blk_off"][b])
        span, open_ = slice(blk, blk + _blocks(packed)), slice(at, at + ctx + n)
        seen = torch.ones(n, packed + ctx + n, dtype=torch.bool, device="cuda")
        if s["tree"]:
            seen[:, packed + ctx:] = False
            paths = []
            for m, p in enumerate(s["parent"][b, :n].tolist()):
                paths.append((paths[p] if p >= 0 else []) + [m])
                seen[m, packed + ctx + torch.tensor(paths[m], device="cuda")] = True
            dst = out[b, :n]
            q = s["q"][b, :n].double()
        else:
            seen[:, packed + ctx:].tril_()
            r0 = int(s["row_off"][b])
            dst, q = out[r0:r0 + n], s["q"][r0:r0 + n].double()
        for h in range(s["hkv"]):
            k, v = (torch.cat(((p[span, h].double()[:, at_] * c[span, h].double().view(-1, 1, 1)).reshape(-1, d)[:packed],
                               r[open_, h].double()))
                    for p, at_, c, r in ((s["pk"], at_k, s["k_scale"], s["k"]), (s["pv"], at_v, s["v_scale"], s["v"])))
            kt = k.t().contiguous()
            for g in range(h * group, (h + 1) * group):
                x = torch.mm(q[:, g].contiguous(), kt) * s["scale"]
                x[~seen] = -math.inf
                dst[:, g] = torch.softmax(x, dim=1) @ v
    return dict(o=out, status=None)


def _exact_sample(s):
    batch, n_max, vocab = s["logits"].shape
    token = torch.full((batch, n_max), -2, dtype=torch.int32, device="cuda")
    logprob = torch.full((batch, n_max), -math.inf, dtype=torch.float64, device="cuda")
    kept = torch.zeros(batch, n_max, dtype=torch.int32, device="cuda")
    value = lambda name, b, other: other if s[name] is None else s[name][b].item()  # noqa: E731
    for b, n in enumerate(s["host_rows"]):
        t, k, p, m = (value(a, b, o) for a, o in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)))
        for r in range(n):
            x = s["logits"][b, r].double()
            order = torch.argsort(-x, stable=True)
            order = order[:1] if t == 0 else order[:k] if k > 0 else order
            y = (x[order] - x[order[0]]) / (t or 1.0)
            y = y[y >= -64]
            if p < 1:
                share = torch.softmax(y, 0)
                before = torch.cat((share.new_zeros(1), share.cumsum(0)[:-1]))
                y = y[:max(1, int((before < p).sum()))]
            if m > 0:
                y = y[:max(1, int((y.exp() >= m).sum()))]
            share = torch.softmax(y, 0)
            j = min(int(torch.searchsorted(share.cumsum(0), s["uniform"][b, r].double(), right=True)), y.shape[0] - 1)
            token[b, r], logprob[b, r], kept[b, r] = order[j], share[j].log(), y.shape[0]
    return dict(token=token, logprob=logprob, kept=kept)


def exact(case, seed):
    return {"pack": _exact_pack, "attend": _exact_attend, "sample": _exact_sample}[case["kind"]](prepare(case, seed))
