"""Performance cases of the 8-bit operators: block quantisation, the matrix
product of block-scaled 8-bit operands, the merge of fresh keys and values
into an 8-bit cache, and the attention over that cache.

Eight-bit values are e4m3; a block's scale is a power of two, 2^(e - 127) for
the stored byte e, the least one with which the block's largest magnitude is
at most 448 (and e >= 1).  Matrices have a scale for each row and 128 columns
(activations) or for each 128 x 128 tile (weights); scales are stored with the
column blocks outermost, [column block][row block], rows padded to 16 bytes.
The cache holds, for each chain, head and block of 64 tokens, 64 keys and then
64 values of 72 dims, with a scale for each of the two.

Sizes are those of the framework's model and grids: hidden 1152, 16 heads of
72, MLP 4608, 120 text tokens of 4096 features, 32 to 128 patches a side,
5-20 % of the tokens active in an edit; the odd ones are generic.
"""
import math
import types

import torch

own = False

HEADS, D, BLOCK, KEYS = 16, 72, 128, 64
C = HEADS * D


def _quantize(rows, cols, tile, dtype):
    return dict(kind="quantize", rows=rows, cols=cols, tile=tile, dtype=dtype)


def _gemm(m, n, k, gelu=False, out="bf16", bias=True):
    return dict(kind="gemm", m=m, n=n, k=k, gelu=gelu, out=out, bias=bias)


def _store(gh, gw, h, w, batch=1, dtype="bf16"):
    """An h x w rectangle of a gh x gw token grid, moved from chain to chain."""
    return dict(kind="store", gh=gh, gw=gw, h=h, w=w, batch=batch, dtype=dtype)


def _attention(tokens, queries, keys=""):
    """queries, keys: counts of each chain, separated by commas; no keys: all tokens of every chain."""
    return dict(kind="attention", tokens=tokens, queries=queries, keys=keys)


def listed():
    def case(name, c):
        c["name"] = name
        return c

    return [
        # normalised activations of a 1024 px edit's rows, before the MLP
        case("quantize_rows", _quantize(723, 1152, 1, "bf16")),
        # an MLP weight matrix as loaded, once per model
        case("quantize_weight", _quantize(4608, 1152, 128, "f32")),
        # a single active token through the MLP's first product: the smallest call
        case("gemm_token", _gemm(1, 4608, 1152, gelu=True)),
        # the MLP's second product of a 1024 px edit: few tiles, a long sum
        case("gemm_down_723", _gemm(723, 1152, 4608)),
        # ragged sizes: 219 rows, columns and sum that end inside a block of 128
        case("gemm_ragged", _gemm(219, 1000, 1072, out="f32", bias=False)),
        # the MLP's first product of the dense step at 2048 px: the largest product
        case("gemm_up_16384", _gemm(16384, 4608, 1152, gelu=True)),
        # keys and values of a 1024 px edit (27 x 27 patches) into the cache
        case("store_1024", _store(64, 64, 27, 27)),
        # those of every token of a 2048 px grid in float32, two chains: the dense step
        case("store_dense_2048", _store(128, 128, 128, 128, batch=2, dtype="f32")),
        # one query over a long cache: latency and the split of the keys
        case("attention_token", _attention(16384, "1")),
        # the benchmark's edit: 723 queries of 4096 keys
        case("attention_723", _attention(4096, "723")),
        # a served batch with ragged regions and valid lengths, one chain with no key and one without query
        case("attention_ragged", _attention(4096, "410,1,77,655,0,233", "4096,3001,0,65,4096,1")),
        # every query and key of the 2048 px grid: the largest
        case("attention_dense_2048", _attention(16384, "16384")),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["quantize", "gemm", "gemm", "store", "attention", "attention"])
    if kind == "quantize":
        cols = 16 * log(1, 288)
        return _quantize(min(log(1, 16384), (1 << 26) // cols), cols, rng.choice([1, 1, 128]), rng.choice(["bf16", "f32"]))
    if kind == "gemm":
        n, k = rng.choice([log(1, 4608), 1152, 4608, 3456]), rng.choice([16 * log(1, 288), 1152, 4608])
        return _gemm(min(log(1, 16384), 16384 * 4608 * 1152 // (n * k)), n, k, gelu=rng.random() < 0.3,
                     out=rng.choice(["bf16", "bf16", "f32"]), bias=rng.random() < 0.8)
    if kind == "store":
        gh, gw = 8 * rng.randint(1, 16), 8 * rng.randint(1, 16)
        return _store(gh, gw, min(gh, log(1, gh)), min(gw, log(1, gw)), batch=rng.choice([1, 1, 2, 4]),
                      dtype=rng.choice(["bf16", "f32"]))
    batch = rng.choice([1, 1, 2, 3, 5])
    tokens = 64 * log(1, 256)
    most = (1 << 28) // (tokens * batch)
    queries = [min(most, rng.choice([1, log(1, 16384), log(1, 16384)])) if rng.random() < 0.9 else 0 for _ in range(batch)]
    queries[0] = max(queries[0], 1)
    keys = ""
    if rng.random() < 0.5:
        keys = ",".join(str(rng.choice([0, tokens, rng.randint(1, tokens), rng.randint(1, tokens)])) for _ in range(batch))
    return _attention(tokens, ",".join(map(str, queries)), keys)


# ------------------------------------------------------------------ inputs

def _ints(text):
    return [int(t) for t in text.split(",")] if text else []


def _tokens(case):
    """Active tokens of each chain, ascending."""
    out = []
    for b in range(case["batch"]):
        y0 = (case["gh"] - case["h"]) * (b + 1) // (case["batch"] + 1)
        x0 = (case["gw"] - case["w"]) * (b + 1) // (case["batch"] + 1)
        out.append([(y0 + y) * case["gw"] + x0 + x for y in range(case["h"]) for x in range(case["w"])])
    return out


def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * std


def _activations(gen, rows, cols):
    """Normalised rows with a few columns that are much larger, as modulated activations have."""
    x = _normal(gen, rows, cols)
    big = torch.rand(cols, generator=gen, device="cuda") < 0.01
    return x * torch.where(big, 12.0, 1.0)


def prepare(case, seed):
    gen = torch.Generator("cuda")
    gen.manual_seed(int(seed))
    kind = case["kind"]
    st = types.SimpleNamespace(kind=kind, case=dict(case))
    if kind == "quantize":
        x = _activations(gen, case["rows"], case["cols"]) if case["tile"] == 1 else _normal(gen, case["rows"], case["cols"], std=0.02)
        st.x = x.to(_TYPES[case["dtype"]])
    elif kind == "gemm":
        st.a, st.a_scale = _to_blocks(_activations(gen, case["m"], case["k"]), 1)
        st.w, st.w_scale = _to_blocks(_normal(gen, case["n"], case["k"], std=0.02), 128)
        st.bias = _normal(gen, case["n"], std=0.02) if case["bias"] else None
    else:
        batch = case["batch"] if kind == "store" else len(_ints(case["queries"]))
        n = case["gh"] * case["gw"] if kind == "store" else case["tokens"]
        kv = _normal(gen, batch, HEADS, n // KEYS, 2, KEYS, D)
        kv[:, :, :, 0] *= 2.0
        kv[:, :, :, 1] *= 0.7
        st.data, st.scale = _to_cache(kv)
        if kind == "store":
            per = _tokens(case)
            rows = sum(map(len, per))
            kv = _normal(gen, rows, 2 * C).to(_TYPES[case["dtype"]])  # one product's output: keys beside values
            st.k, st.v = kv[:, :C], kv[:, C:]
            st.idx = torch.tensor(sum(per, []), dtype=torch.int32, device="cuda")
            counts = [len(p) for p in per]
        else:
            counts = _ints(case["queries"])
            st.q = _normal(gen, sum(counts), C, std=2.0).to(torch.bfloat16)  # logits of standard deviation 4
            st.key_len = torch.tensor(_ints(case["keys"]), dtype=torch.int32, device="cuda") if case["keys"] else None
            st.idx = torch.zeros(sum(counts), dtype=torch.int32, device="cuda")
        st.offsets_host = [0]
        for c in counts:
            st.offsets_host.append(st.offsets_host[-1] + c)
        st.offsets = torch.tensor(st.offsets_host, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    return st


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ plain forms

def _exponents(amax):
    """Stored scale byte of a block whose largest finite magnitude is amax (float32)."""
    bits = amax.view(torch.int32)
    e = (bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000)
    return e.clamp(1, 254).to(torch.uint8)


def _factor(e):
    return torch.ldexp(torch.ones((), device=e.device), e.to(torch.int32) - 127)


def _encode(x, e):
    """x in units of the scale byte e's step, rounded to e4m3 (non-finite: NaN)."""
    y = torch.ldexp(x, 127 - e.to(torch.int32))
    return torch.where(torch.isfinite(x), y, math.nan).to(torch.float8_e4m3fn)


def _to_blocks(x, tile):
    """x [rows][cols] -> e4m3 [rows][cols], scale bytes [column blocks][row blocks, padded to 16]."""
    rows, cols = x.shape
    x = x.float()
    rb, cb = -(-rows // tile), -(-cols // BLOCK)
    padded = torch.nn.functional.pad(x, (0, cb * BLOCK - cols, 0, rb * tile - rows)).view(rb, tile, cb, BLOCK)
    mag = torch.where(torch.isfinite(padded), padded.abs(), 0.0)
    e = _exponents(mag.amax(dim=(1, 3)))
    q = _encode(padded, e[:, None, :, None]).view(torch.uint8).reshape(rb * tile, cb * BLOCK)[:rows, :cols].contiguous()
    scale = torch.zeros(cb, rb + -rb % 16, dtype=torch.uint8, device=x.device)
    scale[:, :rb] = e.t()
    return q.view(torch.float8_e4m3fn), scale


def _of_blocks(q, scale, tile):
    rows, cols = q.shape
    f = _factor(scale[:, :-(-rows // tile)].t())
    f = f.repeat_interleave(tile, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]
    return q.float() * f


def _to_cache(kv):
    """kv [batch][heads][blocks][2][64][72] float32 -> e4m3 of that shape, scale bytes [batch][heads][blocks][2]."""
    mag = torch.where(torch.isfinite(kv), kv.abs(), 0.0)
    e = _exponents(mag.amax(dim=(4, 5)))
    return _encode(kv, e[..., None, None]), e


def _of_cache(data, scale):
    return data.float() * _factor(scale)[..., None, None]


def _chain_of_row(st, rows):
    return torch.searchsorted(st.offsets[1:].long(), torch.arange(rows, device="cuda"), right=True)


def _plain_quantize(st):
    q, scale = _to_blocks(st.x, st.case["tile"])
    return {"q": q, "scale": scale[:, :-(-st.case["rows"] // st.case["tile"])]}


def _gelu(y):
    return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))


def _plain_gemm(st):
    y = _of_blocks(st.a, st.a_scale, 1) @ _of_blocks(st.w, st.w_scale, 128).t()
    if st.bias is not None:
        y = y + st.bias
    if st.case["gelu"]:
        y = _gelu(y)
    return {"y": y.to(_TYPES[st.case["out"]])}


def _plain_store(st):
    kv = _of_cache(st.data, st.scale)
    chain, tok = _chain_of_row(st, st.idx.numel()), st.idx.long()
    for which, rows in ((0, st.k), (1, st.v)):
        kv[chain, :, tok // KEYS, which, tok % KEYS] = rows.float().view(-1, HEADS, D)
    touched = torch.zeros(st.scale.shape[0], st.scale.shape[2], dtype=torch.bool, device="cuda")
    touched[chain, tok // KEYS] = True
    q, e = _to_cache(kv)
    keep = ~touched[:, None, :, None]
    st.data.copy_(torch.where(keep[..., None, None], st.data.view(torch.uint8), q.view(torch.uint8)).view(torch.float8_e4m3fn))
    st.scale.copy_(torch.where(keep, st.scale, e))
    return {"data": st.data, "scale": st.scale}


def _plain_attention(st):
    kv = _of_cache(st.data, st.scale)
    batch, n = kv.shape[0], st.case["tokens"]
    k = kv[:, :, :, 0].reshape(batch * HEADS, n, D)
    v = kv[:, :, :, 1].reshape(batch * HEADS, n, D)
    rows, most = st.q.shape[0], max(_ints(st.case["queries"]))
    chain = _chain_of_row(st, rows)
    at = torch.arange(rows, device="cuda") - st.offsets.long()[chain]
    q = torch.zeros(batch, most, HEADS, D, device="cuda")
    q[chain, at] = st.q.float().view(rows, HEADS, D)
    s = torch.bmm(q.permute(0, 2, 1, 3).reshape(batch * HEADS, most, D), k.transpose(1, 2).contiguous())
    s = s.mul_(1.0 / math.sqrt(D)).view(batch, HEADS, most, n)
    if st.key_len is not None:
        s.masked_fill_((torch.arange(n, device="cuda") >= st.key_len[:, None])[:, None, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    den = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(batch * HEADS, most, n), v).view(batch, HEADS, most, D) / torch.where(den == 0.0, 1.0, den)
    return {"o": o.permute(0, 2, 1, 3)[chain, at].reshape(rows, C).to(torch.bfloat16)}


# ------------------------------------------------------------------ the framework's calls

def _own(st):
    from paper_2608_29809_amd import quant
    from paper_2608_29809_amd.runtime import ActiveSet

    if st.kind == "quantize":
        m = quant.quantize(st.x, st.case["tile"])
        return {"q": m.data, "scale": m.scales[:, :-(-st.case["rows"] // st.case["tile"])]}
    if st.kind == "gemm":
        y = quant.qgemm(quant.QuantMatrix(st.a, st.a_scale, 1), quant.QuantMatrix(st.w, st.w_scale, 128), st.bias,
                        gelu=st.case["gelu"], dtype=_TYPES[st.case["out"]])
        return {"y": y}
    cache = quant.QuantCache(st.data, st.scale)
    rows = ActiveSet(st.idx, st.offsets, st.offsets_host)
    if st.kind == "store":
        quant.qcache_store(cache, rows, st.k, st.v)
        return {"data": st.data, "scale": st.scale}
    return {"o": quant.qcache_attention(cache, rows, st.q, key_len=st.key_len)}


def run(state):
    if own:
        return _own(state)
    return {"quantize": _plain_quantize, "gemm": _plain_gemm, "store": _plain_store, "attention": _plain_attention}[state.kind](state)


# ------------------------------------------------------------------ work

def _size(name):
    return {"bf16": 2, "f32": 4}[name]


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        scales = -(-case["rows"] // case["tile"]) * -(-case["cols"] // BLOCK)
        return {"bytes": n * (_size(case["dtype"]) + 1) + scales, "flops": 2 * n}
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        scales = (m + -(-n // 128)) * -(-k // BLOCK)
        return {"bytes": m * k + n * k + scales + (4 * n if case["bias"] else 0) + m * n * _size(case["out"]), "flops": 2 * m * n * k}
    if kind == "store":
        rows = case["batch"] * case["h"] * case["w"]
        blocks = sum(len({t // KEYS for t in per}) for per in _tokens(case))
        kept = blocks * KEYS - rows  # tokens of touched blocks that stay: read and written
        return {"bytes": 2 * C * (rows * _size(case["dtype"]) + kept + blocks * KEYS) + 4 * HEADS * blocks + 4 * rows,
                "flops": 4 * C * blocks * KEYS}
    queries = _ints(case["queries"])
    keys = _ints(case["keys"]) or [case["tokens"]] * len(queries)
    read = sum(k for q, k in zip(queries, keys) if q)
    return {"bytes": 2 * C * read + 2 * HEADS * -(-read // KEYS) + 4 * C * sum(queries),
            "flops": 4 * C * sum(q * k for q, k in zip(queries, keys))}


# ------------------------------------------------------------------ 64 bits

def _exact_scale(mag):
    """log2 of the least power of two s, at least 2^-126, with mag <= 448 s."""
    frac, ex = torch.frexp(mag)  # mag = frac 2^ex, 0.5 <= frac < 1
    return torch.where(mag > 0, ex - 9 + (frac > 0.875).int(), -126).clamp(min=-126).double()


def _exact_codes(x, log2s):
    """Nearest e4m3 number to x / 2^log2s, ties to the even one."""
    y = x * torch.exp2(-log2s)
    low = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(low - 3.0)
    return torch.round(y / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        x, tile = st.x.double(), case["tile"]
        q = torch.empty_like(x)
        bytes_ = torch.empty(-(-case["cols"] // BLOCK), -(-case["rows"] // tile), dtype=torch.uint8, device="cuda")
        for j in range(0, case["cols"], BLOCK):
            part = x[:, j:j + BLOCK].abs().amax(1)
            part = torch.nn.functional.pad(part, (0, -case["rows"] % tile)).view(-1, tile).amax(1)
            log2s = _exact_scale(part)
            bytes_[j // BLOCK] = (log2s + 127).to(torch.uint8)
            q[:, j:j + BLOCK] = _exact_codes(x[:, j:j + BLOCK], log2s.repeat_interleave(tile)[:case["rows"], None])
        return {"q": q, "scale": bytes_}
    if kind == "gemm":
        def value(q, scale, tile):
            s = torch.exp2(scale.double() - 127.0)
            i = torch.arange(q.shape[0], device="cuda") // tile
            j = torch.arange(q.shape[1], device="cuda") // BLOCK
            return q.double() * s[j][:, i].t()

        y = value(st.a, st.a_scale, 1) @ value(st.w, st.w_scale, 128).t()
        if st.bias is not None:
            y += st.bias.double()
        if case["gelu"]:
            y = y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
        return {"y": y}
    value = st.data.double() * torch.exp2(st.scale.double() - 127.0)[..., None, None]
    if kind == "store":
        codes, log2s = st.data.double(), st.scale.double() - 127.0
        for b, tokens in enumerate(_tokens(case)):
            r0 = st.offsets_host[b]
            for blk in sorted({t // KEYS for t in tokens}):
                at = [(r0 + i, t % KEYS) for i, t in enumerate(tokens) if t // KEYS == blk]
                src = torch.tensor([a for a, _ in at], device="cuda")
                dst = torch.tensor([t for _, t in at], device="cuda")
                for which, fresh in ((0, st.k), (1, st.v)):
                    v = value[b, :, blk, which]
                    v[:, dst] = fresh[src].double().view(-1, HEADS, D).transpose(0, 1)
                    s = _exact_scale(v.abs().amax((1, 2)))
                    codes[b, :, blk, which] = _exact_codes(v, s[:, None, None])
                    log2s[b, :, blk, which] = s
        return {"data": codes, "scale": (log2s + 127).to(torch.uint8)}
    out = torch.zeros(st.q.shape[0], HEADS, D, dtype=torch.float64, device="cuda")
    for b in range(len(st.offsets_host) - 1):
        r0, r1 = st.offsets_host[b], st.offsets_host[b + 1]
        n = case["tokens"] if st.key_len is None else int(st.key_len[b])
        for h in range(HEADS if r1 > r0 and n else 0):
            k, v = value[b, h, :, 0].reshape(-1, D)[:n], value[b, h, :, 1].reshape(-1, D)[:n]
            p = torch.softmax(st.q[r0:r1, h * D:(h + 1) * D].double() @ k.t() / math.sqrt(D), -1)
            out[r0:r1, h] = p @ v
    return {"o": out.view(-1, C)}
