"""The operators of the paged KV cache, and what is measured of them.

Four operators, each over the range that serving suspended agents meets (8 KV heads of 128, contexts
of 1,024 to 131,072 tokens as in ``workloads.py``, and other head layouts):

``rotary``     kvr_rotary: rotary positions of queries or keys, both layouts, part of the head, and
               the adjoint (the gradient, or a rotation back)
``write``      kvr_cache_write: keys (rotated on the way) and values into the pages of a cache, kept
               in 16 bits or quantised as they are written, then kvr_cache_read of the same rows
``read``       kvr_cache_read: rows of a cache back in their order, dequantised
``attention``  kvr_tree_attention: one new token, or a tree of drafted tokens, of each sequence over
               its pages of the cache

A quantised row is cut into blocks of 32; a block keeps one power of two (a byte: its exponent + 127)
and 32 codes of 8 bits (e4m3) or 4 bits (e2m1, the even element in the low half of the byte).
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LARGEST = {"fp8": 448.0, "fp4": 6.0}     # the largest code of each format
MIN_EXP = -110                           # the smallest block exponent


def listed():
    return [
        # the queries of one decoded token: the smallest call, latency only
        dict(name="rotary-1-token", op="rotary", tokens=1, heads=32, dim=128, rot=128, dtype="bf16",
             interleaved=False, adjoint=False, positions=131072),
        # the queries of a whole 32,768-token context recomputed after its copy was discarded
        dict(name="rotary-32k", op="rotary", tokens=32768, heads=32, dim=128, rot=128, dtype="bf16",
             interleaved=False, adjoint=False, positions=32768),
        # interleaved pairs, half of the head rotated, odd sizes, the gradient
        dict(name="rotary-4097-part-adjoint", op="rotary", tokens=4097, heads=9, dim=192, rot=96,
             dtype="fp16", interleaved=True, adjoint=True, positions=8192),
        # one new token of each of 64 sequences into an 8-bit cache
        dict(name="write-64-fp8", op="write", fmt="fp8", tokens=64, heads=8, dim=128, rot=128,
             dtype="bf16", out="bf16", interleaved=False, page=16, positions=131072, skip=0),
        # a context of 32,768 tokens quantised to 4 bits for retention, odd length, some rows padding
        dict(name="write-32k-fp4", op="write", fmt="fp4", tokens=32749, heads=8, dim=128, rot=128,
             dtype="bf16", out="bf16", interleaved=False, page=64, positions=32768, skip=100),
        # a prompt kept in 16 bits, a part of each key rotated in interleaved pairs
        dict(name="write-8191-fp16", op="write", fmt="fp16", tokens=8191, heads=4, dim=192, rot=64,
             dtype="fp16", out="fp16", interleaved=True, page=32, positions=8192, skip=0),
        # a suspended context of 131,072 tokens restored from 8 bits
        dict(name="read-128k-fp8", op="read", fmt="fp8", tokens=131072, heads=8, dim=128, out="bf16",
             page=64),
        # a short one of odd length from 4 bits
        dict(name="read-1021-fp4", op="read", fmt="fp4", tokens=1021, heads=8, dim=128, out="fp16",
             page=16),
        # one resumed agent, one token, a short context in 16 bits: latency
        dict(name="attention-1x1000-bf16", op="attention", fmt="bf16", dtype="bf16", seqs=1,
             kv_lo=1000, kv_hi=1000, q_lo=1, q_hi=1, tree=False, heads=8, group=4, dim=128, page=16,
             shape_seed=1),
        # the decode step of 64 agents of 8,192 tokens each in 8 bits
        dict(name="attention-64x8192-fp8", op="attention", fmt="fp8", dtype="bf16", seqs=64,
             kv_lo=8192, kv_hi=8192, q_lo=1, q_hi=1, tree=False, heads=8, group=4, dim=128, page=64,
             shape_seed=2),
        # one agent of the longest context in 4 bits, a small tree of drafted tokens
        dict(name="attention-1x128k-tree7-fp4", op="attention", fmt="fp4", dtype="bf16", seqs=1,
             kv_lo=131071, kv_hi=131071, q_lo=7, q_hi=7, tree=True, heads=8, group=8, dim=128,
             page=64, shape_seed=3),
        # sixteen agents of 2,048 to 32,768 tokens with trees of up to 64 drafted tokens in 16 bits
        dict(name="attention-16-ragged-tree64", op="attention", fmt="bf16", dtype="bf16", seqs=16,
             kv_lo=2048, kv_hi=32768, q_lo=17, q_hi=64, tree=True, heads=8, group=8, dim=128,
             page=32, shape_seed=4),
    ]


def log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "write", "read", "attention", "attention"])
    dim = rng.choice([64, 96, 128, 128, 192, 256])
    if op == "rotary":
        heads = rng.randint(1, 64)
        tokens = log_int(rng, 1, min(32768, 32768 * 32 * 128 // (heads * dim)))
        return dict(op=op, tokens=tokens, heads=heads, dim=dim, rot=dim // rng.choice([1, 1, 2]),
                    dtype=rng.choice(["bf16", "fp16", "fp32"]) if tokens <= 8192 else "bf16",
                    interleaved=rng.random() < 0.5, adjoint=rng.random() < 0.5, positions=32768)
    if op == "write":
        heads = rng.randint(1, 16)
        fmt = rng.choice(["bf16", "fp16", "fp8", "fp8", "fp4", "fp4"])
        tokens = log_int(rng, 1, min(65536, 32749 * 8 * 128 // (heads * dim)))
        dtype = fmt if fmt in DTYPES else rng.choice(["bf16", "fp16"])
        return dict(op=op, fmt=fmt, tokens=tokens, heads=heads, dim=dim,
                    rot=dim // rng.choice([1, 1, 2]), dtype=dtype, out=dtype,
                    interleaved=rng.random() < 0.5, page=rng.choice([16, 32, 64, 256]),
                    positions=65536, skip=tokens // 50 if rng.random() < 0.5 else 0)
    if op == "read":
        heads = rng.randint(1, 16)
        fmt = rng.choice(["bf16", "fp16", "fp8", "fp8", "fp4", "fp4"])
        out = fmt if fmt in DTYPES else rng.choice(["bf16", "fp16", "fp32"])
        tokens = log_int(rng, 1, min(131072, 131072 * 8 * 128 // (heads * dim)) // (1 + (out == "fp32")))
        return dict(op=op, fmt=fmt, tokens=tokens, heads=heads, dim=dim, out=out,
                    page=rng.choice([16, 32, 64, 256]))
    fmt = rng.choice(["bf16", "fp16", "fp8", "fp8", "fp4", "fp4"])
    heads, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 3, 4, 8, 8, 16])
    seqs = log_int(rng, 1, 64)
    q_hi = rng.choice([1, 1, log_int(rng, 2, 64)])
    # no dearer than the listed ones: cache elements, and products of rows and elements
    rows = q_hi * group
    elements = min(64 * 8192 * 8 * 128, 16 * 20000 * 8 * 128 * 512 // rows)
    kv_hi = log_int(rng, q_hi, max(q_hi, min(131072, elements // (seqs * heads * dim))))
    return dict(op=op, fmt=fmt, dtype=fmt if fmt in DTYPES else rng.choice(["bf16", "fp16"]),
                seqs=seqs, kv_lo=max(q_hi, kv_hi // rng.choice([1, 4, 16])), kv_hi=kv_hi,
                q_lo=rng.choice([q_hi, max(1, q_hi // 3)]), q_hi=q_hi,
                tree=q_hi > 1 and rng.random() < 0.7, heads=heads, group=group, dim=dim,
                page=rng.choice([16, 32, 64, 256]), shape_seed=rng.randint(0, 10 ** 6))


def lengths(case):
    """Each sequence's tokens in the cache, its newest ones among them, and how many those are."""
    rng = random.Random(case["shape_seed"])
    kv = [log_int(rng, case["kv_lo"], case["kv_hi"]) for _ in range(case["seqs"])]
    return kv, [min(n, rng.randint(case["q_lo"], case["q_hi"])) for n in kv]


def row_bytes(fmt, dim):
    """A row of the cache: one token's key or value of one head."""
    return {"bf16": 2 * dim, "fp16": 2 * dim, "fp8": dim + dim // 32, "fp4": dim // 2 + dim // 32}[fmt]


def work(case):
    c = case
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    if c["op"] == "rotary":
        values = c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": 2 * values * size[c["dtype"]] + c["tokens"] * (4 * c["rot"] + 4),
                "flops": 3 * c["tokens"] * c["heads"] * c["rot"]}
    if c["op"] in ("write", "read"):
        rows = 2 * c["tokens"] * c["heads"]
        cache = rows * row_bytes(c["fmt"], c["dim"])
        read = cache + rows * c["dim"] * size[c["out"]] + 8 * c["tokens"]
        if c["op"] == "read":
            return {"bytes": read, "flops": rows * c["dim"]}
        write = cache + rows * c["dim"] * size[c["dtype"]] + c["tokens"] * (4 * c["rot"] + 12)
        return {"bytes": read + write, "flops": 4 * rows * c["dim"]}
    kv, nq = lengths(c)
    q_heads = c["heads"] * c["group"]
    values = sum(nq) * q_heads * c["dim"]
    return {"bytes": 2 * sum(kv) * c["heads"] * row_bytes(c["fmt"], c["dim"])
            + 2 * values * size[c["dtype"]] + 4 * sum(nq) * q_heads,
            "flops": sum(4 * n * q_heads * c["dim"] * (t - (n - 1) / 2) for t, n in zip(kv, nq))}


# ---- inputs -------------------------------------------------------------------------------------

def rotary_table(positions, rot):
    """cos and sin of position * 500000^(-2i / rot), [positions, 2, rot / 2]."""
    freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], 1).float()


def activations(gen, shape, dtype):
    """Projections of a hidden state: near normal, some channels of the head several times larger."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    wide = 1 + 4 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.05)
    return (x * wide).to(dtype)


def filled_cache(gen, case, pages):
    """The cache's tensors, every row of it written: [pages, heads, page, row]."""
    shape = (pages, case["heads"], case["page"], case["dim"])
    out = []
    for _ in range(2):
        if case["fmt"] in DTYPES:
            out.append([activations(gen, shape, DTYPES[case["fmt"]]), None])
            continue
        step = max(1, (1 << 26) // math.prod(shape[1:]))
        parts = [encode(activations(gen, (min(step, pages - p),) + shape[1:], torch.bfloat16), case["fmt"])
                 for p in range(0, pages, step)]
        out.append([torch.cat(x) for x in zip(*parts)])
    return dict(k=out[0][0], v=out[1][0], k_scale=out[0][1], v_scale=out[1][1])


def empty_cache(case, pages):
    shape = (pages, case["heads"], case["page"])
    if case["fmt"] in DTYPES:
        new = lambda: torch.zeros(shape + (case["dim"],), dtype=DTYPES[case["fmt"]], device="cuda")  # noqa: E731
        return dict(k=new(), v=new(), k_scale=None, v_scale=None)
    new = lambda n: torch.zeros(shape + (n,), dtype=torch.uint8, device="cuda")  # noqa: E731
    row = case["dim"] if case["fmt"] == "fp8" else case["dim"] // 2
    return dict(k=new(row), v=new(row), k_scale=new(case["dim"] // 32), v_scale=new(case["dim"] // 32))


def handle(cache):
    """The framework's handle of the cache, which a program makes once."""
    import paper_2608_30830_amd as kvr
    return kvr.KvCache(cache["k"], cache["v"], cache["k_scale"], cache["v_scale"])


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    c = dict(case)
    s = {"case": c}
    if c["op"] in ("rotary", "write"):
        s["table"] = rotary_table(c["positions"], c["rot"])
        # a decoded token's position is anywhere, a context's tokens follow one another
        first = torch.randint(0, max(1, c["positions"] - c["tokens"]), (1,), generator=gen, device="cuda")
        s["positions"] = ((first + torch.arange(c["tokens"], device="cuda")) % c["positions"]).int()
    if c["op"] == "rotary":
        s["x"] = activations(gen, (c["tokens"], c["heads"], c["dim"]), DTYPES[c["dtype"]])
        return s
    if c["op"] in ("write", "read"):
        used = -(-c["tokens"] // c["page"])
        pages = used + 1 + used // 8
        order = torch.randperm(pages, generator=gen, device="cuda")[:used]
        slots = (order[:, None] * c["page"] + torch.arange(c["page"], device="cuda")).reshape(-1)
        s["slots"] = slots[:c["tokens"]].clone()
        if c["op"] == "write":
            s["k"], s["v"] = (activations(gen, (c["tokens"], c["heads"], c["dim"]), DTYPES[c["dtype"]])
                              for _ in range(2))
            if c["skip"]:   # padding of the batch: written nowhere
                s["slots"][torch.randperm(c["tokens"], generator=gen, device="cuda")[:c["skip"]]] = -1
        s["cache"] = empty_cache(c, pages) if c["op"] == "write" else filled_cache(gen, c, pages)
    else:
        kv, nq = lengths(c)
        need = [-(-n // c["page"]) for n in kv]
        pages = sum(need) + 1
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        table = torch.full((c["seqs"], max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        s["page_table"] = table
        s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
        cu = [0]
        for n in nq:
            cu.append(cu[-1] + n)
        s["cu_q"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
        s["max_q"], s["max_kv"] = max(nq), max(kv)
        s["q"] = activations(gen, (cu[-1], c["heads"] * c["group"], c["dim"]), DTYPES[c["dtype"]])
        s["scale"] = c["dim"] ** -0.5
        s["mask"] = None
        if c["tree"]:
            rng, words = random.Random(seed), []
            for n in nq:
                seen = []
                for i in range(n):   # a drafted token sees itself and what its parent sees
                    parent = rng.randint(max(-1, i - 8), i - 1)
                    seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
                words += seen
            words = [w - (1 << 64) if w >> 63 else w for w in words]
            s["mask"] = torch.tensor(words, dtype=torch.int64, device="cuda")[:, None]
        s["cache"] = filled_cache(gen, c, pages)
    if own:
        s["handle"] = handle(s["cache"])
    return s


# ---- the plain forms ----------------------------------------------------------------------------

def rotate(x, positions, table, interleaved, adjoint):
    """Rotary positions in 32 bits; x is [tokens, heads, dim] in 32 bits."""
    rot = 2 * table.shape[-1]
    rows = table[positions.long()][:, :, None, :]
    cos, sin = rows[:, 0], rows[:, 1]
    if adjoint:
        sin = -sin
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    y, z = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([y, z], -1).flatten(-2) if interleaved else torch.cat([y, z], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def encode(x, fmt):
    """Codes and scale bytes of rows [..., dim]."""
    blocks = x.float().unflatten(-1, (-1, 32))
    bits = blocks.abs().amax(-1).view(torch.int32)
    # the smallest k with amax <= M 2^k: one more than the floor where the mantissa is beyond M's
    over, top = (0x7FFFFF - 0x600000, 8) if fmt == "fp8" else (0x7FFFFF - 0x400000, 2)
    k = (((bits + over) >> 23) - 127 - top).clamp(min=MIN_EXP)
    bad = ~(blocks.abs() < math.inf).all(-1)
    k = torch.where(bad, 128, k)
    y = blocks * ((127 - k.clamp(max=126)) << 23).view(torch.float32)[..., None]
    y = torch.where(bad[..., None], 0.0, y).flatten(-2)
    if fmt == "fp8":
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        a = y.abs()   # between two levels to the nearer one, halfway to the even code
        n = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
        n = n + 8 * (y.view(torch.int32) < 0)
        codes = (n[..., 0::2] + 16 * n[..., 1::2]).to(torch.uint8)
    return codes, (k + 127).to(torch.uint8)


def decode(codes, scale):
    """The values of rows of the cache in 32 bits."""
    if scale is None:
        return codes.float()
    if codes.shape[-1] == 32 * scale.shape[-1]:
        y = codes.view(torch.float8_e4m3fn).float()
    else:
        levels = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=codes.device)
        y = torch.stack([levels[(codes & 15).int()], levels[(codes >> 4).int()]], -1).flatten(-2)
    s = (scale.int() << 23).view(torch.float32)
    s = torch.where(scale == 255, math.nan, s)
    return (y.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def put(cache, name, rows, slots):
    """Rows [tokens, heads, dim] in 32 bits into the pages; slots below 0 are dropped."""
    page = cache[name].shape[2]
    keep = slots >= 0
    at, off = slots[keep] // page, slots[keep] % page
    rows = rows[keep]
    if cache[name + "_scale"] is None:
        cache[name][at, :, off] = rows.to(cache[name].dtype)
    else:
        fmt = "fp8" if cache[name].shape[-1] == rows.shape[-1] else "fp4"
        codes, scale = encode(rows, fmt)
        cache[name][at, :, off] = codes
        cache[name + "_scale"][at, :, off] = scale


def get(cache, name, slots, dtype):
    """Rows back, zeros where the slot is below 0."""
    page = cache[name].shape[2]
    at, off = slots.clamp(min=0) // page, slots.clamp(min=0) % page
    scale = cache[name + "_scale"]
    rows = decode(cache[name][at, :, off], None if scale is None else scale[at, :, off])
    return torch.where((slots >= 0)[:, None, None], rows, 0.0).to(dtype)


def attend(s):
    cache, q, cu, kv_len = s["cache"], s["q"], s["cu_q"].long(), s["kv_len"].long()
    seqs, total = len(kv_len), q.shape[0]
    heads, mq, length = cache["k"].shape[1], s["max_q"], s["max_kv"]
    table = s["page_table"].clamp(min=0).long()

    def rows(name):   # [seqs, heads, length, dim]
        scale = cache[name + "_scale"]
        x = decode(cache[name][table], None if scale is None else scale[table])
        return x.transpose(1, 2).flatten(2, 3)[:, :, :length]

    nq = cu[1:] - cu[:-1]
    i = torch.arange(mq, device=q.device)
    at = (cu[:-1, None] + i).clamp(max=total - 1)
    group = q.shape[1] // heads
    x = q.float()[at].unflatten(2, (heads, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    score = torch.matmul(x, rows("k").transpose(2, 3)).mul_(s["scale"]).unflatten(2, (mq, group))
    t = torch.arange(length, device=q.device)
    newest = t - (kv_len - nq)[:, None]                       # [seqs, length], from 0 for drafted ones
    if s["mask"] is None:
        seen = newest[:, None] <= i[:, None]
    else:
        bits = ((s["mask"][at][..., 0][..., None] >> i) & 1).bool()      # [seqs, mq, mq]
        m = newest.clamp(0, mq - 1)[:, None].expand(-1, mq, -1)
        seen = torch.gather(bits, 2, m) | (newest < 0)[:, None]
    seen = (seen & (t < kv_len[:, None])[:, None])[:, None, :, None]     # [seqs, 1, mq, 1, length]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total_p = p.sum(-1)
    v = torch.where((t < kv_len[:, None])[:, None, :, None], rows("v"), 0.0)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (mq, group))
    out = out / torch.where(total_p > 0, total_p, 1.0)[..., None]
    lse = top[..., 0] + torch.log(total_p)
    # [seqs, heads, mq, group, ...] back to the rows of q
    r = torch.arange(total, device=q.device)
    b = (cu[1:, None] <= r).sum(0)
    out = out.permute(0, 2, 1, 3, 4)[b, r - cu[b]].flatten(1, 2)
    lse = lse.permute(0, 2, 1, 3)[b, r - cu[b]].flatten(1, 2)
    return {"out": out.to(q.dtype), "lse": lse}


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2608_30830_amd as kvr
        if c["op"] == "rotary":
            return kvr.kvr_rotary(s["x"], s["positions"], s["table"], interleaved=c["interleaved"],
                                  adjoint=c["adjoint"], check=False)
        if c["op"] == "write":
            kvr.kvr_cache_write(s["handle"], s["k"], s["v"], s["slots"], s["positions"], s["table"],
                                interleaved=c["interleaved"], check=False)
        if c["op"] in ("write", "read"):
            k, v = kvr.kvr_cache_read(s["handle"], s["slots"], DTYPES[c["out"]], check=False)
            return {"k": k, "v": v}
        out, lse = kvr.kvr_tree_attention(s["handle"], s["q"], s["cu_q"], s["kv_len"], s["page_table"],
                                          s["max_q"], s["max_kv"], tree_mask=s["mask"],
                                          scale=s["scale"], want_lse=True, check=False)
        return {"out": out, "lse": lse}
    if c["op"] == "rotary":
        return rotate(s["x"].float(), s["positions"], s["table"], c["interleaved"],
                      c["adjoint"]).to(s["x"].dtype)
    if c["op"] == "write":
        put(s["cache"], "k", rotate(s["k"].float(), s["positions"], s["table"], c["interleaved"], False),
            s["slots"])
        put(s["cache"], "v", s["v"].float(), s["slots"])
    if c["op"] in ("write", "read"):
        return {x: get(s["cache"], x, s["slots"], DTYPES[c["out"]]) for x in ("k", "v")}
    return attend(s)


# ---- the definitions in 64 bits -----------------------------------------------------------------

def rotated64(x, angles, interleaved, sign):
    """Each pair as a complex number, turned by multiplication."""
    rot = 2 * angles.shape[-1]
    x = x.double()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else x[..., :rot].chunk(2, -1)
    z = torch.complex(a, b) * torch.conj_physical(angles)[:, None] if sign < 0 else \
        torch.complex(a, b) * angles[:, None]
    y = x.clone()
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def power64(k):
    """2^k exactly, for whole k in the range of normal numbers."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def quantised64(x, fmt):
    """The values that blocks of 32 along the head keep: each rounded to the format's spacing at its
    own magnitude, halves to the even multiple."""
    blocks = x.double().reshape(x.shape[:-1] + (-1, 32))
    most = blocks.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(most.clamp(min=1e-300) / LARGEST[fmt])).clamp(min=-900)
    k = torch.where(most > LARGEST[fmt] * power64(k), k + 1, k)
    k = torch.where(most <= LARGEST[fmt] * power64(k - 1), k - 1, k).clamp(min=MIN_EXP)
    y = blocks / power64(k)
    low, bits = (-6, 3) if fmt == "fp8" else (0, 1)
    step = power64((torch.frexp(y.abs())[1] - 1).clamp(min=low) - bits)
    return (torch.round(y / step) * step * power64(k)).reshape(x.shape)


def dequantised64(rows, scale):
    if scale is None:
        return rows.double()
    bytes_ = rows.int()
    if rows.shape[-1] == 32 * scale.shape[-1]:
        e, m = (bytes_ >> 3) & 15, bytes_ & 7
        y = torch.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * power64(e - 7))
        y = torch.where(bytes_ >= 128, -y, y)
    else:
        n = torch.stack([bytes_ & 15, bytes_ >> 4], -1).reshape(rows.shape[:-1] + (-1,))
        e, m = (n >> 1) & 3, n & 1
        y = torch.where(e == 0, m / 2.0, (1 + m / 2.0) * power64(e - 1))
        y = torch.where(n >= 8, -y, y)
    return y * power64(scale.long() - 127).repeat_interleave(32, -1)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] in ("rotary", "write"):
        t = s["table"].double()[s["positions"].long()]
        angles = torch.complex(t[:, 0], t[:, 1])
    if c["op"] == "rotary":
        return rotated64(s["x"], angles, c["interleaved"], -1 if c["adjoint"] else 1)
    if c["op"] == "write":
        out = {"k": rotated64(s["k"], angles, c["interleaved"], 1), "v": s["v"].double()}
        for x in out:
            if c["fmt"] not in DTYPES:
                out[x] = quantised64(out[x], c["fmt"])
            out[x][s["slots"] < 0] = 0.0
        return out
    page = c["page"]
    if c["op"] == "read":
        at, off = s["slots"] // page, s["slots"] % page
        out = {}
        for x in ("k", "v"):
            scale = s["cache"][x + "_scale"]
            out[x] = dequantised64(s["cache"][x][at, :, off], None if scale is None else scale[at, :, off])
        return out
    kv, nq = lengths(c)
    q, group = s["q"].double(), c["group"]
    out, lse, first = torch.zeros_like(q), q.new_zeros(q.shape[:2]), 0
    for b, (t, n) in enumerate(zip(kv, nq)):
        pages = s["page_table"][b, :-(-t // page)].long()
        seen = torch.ones(n, t, dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            seen[:, t - n:] = torch.tril(seen[:, t - n:])
        else:
            word = s["mask"][first:first + n]
            seen[:, t - n:] = ((word >> torch.arange(n, device="cuda")) & 1).bool()
        for h in range(c["heads"]):
            k, v = (dequantised64(s["cache"][x][pages, h],
                                  None if s["cache"][x + "_scale"] is None else s["cache"][x + "_scale"][pages, h])
                    .reshape(-1, c["dim"])[:t] for x in ("k", "v"))
            own_heads = slice(h * group, (h + 1) * group)
            x = q[first:first + n, own_heads].reshape(n * group, -1)
            e = (x @ k.T.contiguous() * s["scale"]).reshape(n, group, t)
            e = e.masked_fill(~seen[:, None], -math.inf)
            total = torch.logsumexp(e, -1)
            lse[first:first + n, own_heads] = total
            p = torch.exp(e - total[..., None])
            out[first:first + n, own_heads] = (p.reshape(n * group, t) @ v).reshape(n, group, -1)
        first += n
    return {"out": out, "lse": lse}
