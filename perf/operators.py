"""Operators around the decode attention, as cases that can be timed: rotary positions, the rotated append to a cache, the
residual's addition with the root-mean-square norm, and products with 4-bit weights.

Where `own` is false, run() computes them in elementary torch operations; where it is true it calls the library."""
import math

import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0


def listed():
    return [
        # rotary positions: the query of one new token of a layer without keys and values (latency)
        dict(name="rope_token", op="rope", tokens=1, heads=32, d=128, rot=128, interleaved=False, fp32=False, positions=4096, fused=False),
        # rotary positions: queries of eight 4096-token prompts inside a fused projection, half of each head rotated, pairs interleaved
        dict(name="rope_prompt_part", op="rope", tokens=32768, heads=32, d=128, rot=64, interleaved=True, fp32=False, positions=4096, fused=True),
        # tables of a model stretched to 131072 positions, frequencies scaled by parts
        dict(name="rope_tables_long", op="tables", positions=131072, rot=128, kind=3, base=500000.0, factor=8.0, original=8192.0),
        # rotated append: a decode step of the TinyLlama shape (4 kv heads of 64), q, k, v are views of a fused projection
        dict(name="append_step_gqa", op="append", batch=128, new=1, hq=32, hkv=4, d=64, rot=64, interleaved=False, lo=512, hi=1536, page=64, fused=True),
        # rotated append: 8 drafted tokens for each of 64 sequences of the Llama-7B shape
        dict(name="append_drafts_7b", op="append", batch=64, new=8, hq=32, hkv=32, d=128, rot=128, interleaved=False, lo=256, hi=2048, page=128, fused=False),
        # rotated append: ragged prompts of up to 4096 tokens, Llama-7B shape (the largest)
        dict(name="append_prompts_7b", op="prompt", batch=8, longest=4096, hq=32, hkv=32, d=128, rot=128, interleaved=False, page=128, fused=False),
        # norm: the hidden states of 16 decoding sequences, Llama-7B width, bf16 out
        dict(name="norm_step", op="norm", rows=16, width=4096, res=True, x32=False, r32=False, out="bf16", group=0),
        # norm: prompts, Llama-7B width, residual kept in fp32, 8-bit out with one scale per 128 columns
        dict(name="norm_prompt_e4m3", op="norm", rows=16384, width=4096, res=True, x32=False, r32=True, out="e4m3", group=128),
        # norm: a large decode batch at the 30B width, 8-bit out with one scale per row
        dict(name="norm_batch_e4m3", op="norm", rows=512, width=6656, res=True, x32=False, r32=False, out="e4m3", group=0),
        # 4-bit weights: one sequence, the output projection at the Llama-7B width
        dict(name="quant_row", op="quant", rows=1, k=4096, n=4096, group=128, zeros=False, x8=-1, out32=False),
        # 4-bit weights: 16 sequences, 8-bit activations with block scales, a gate-and-up projection, zero points
        dict(name="quant_step_e4m3", op="quant", rows=16, k=4096, n=22016, group=64, zeros=True, x8=128, out32=False),
        # 4-bit weights: 200 sequences, a down projection, fp32 out
        dict(name="quant_batch", op="quant", rows=200, k=11008, n=4096, group=128, zeros=False, x8=-1, out32=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "rope", "tables", "append", "append", "prompt", "norm", "norm", "norm", "quant", "quant", "quant", "quant"])
    if op == "rope":
        d = rng.choice([64, 128])
        heads = _log(rng, 1, 64)
        fp32 = rng.random() < 0.25
        most = 32768 * 32 * 128 // (heads * d * (2 if fp32 else 1))
        return dict(op=op, tokens=_log(rng, 1, min(most, 100000)), heads=heads, d=d, rot=rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)]),
                    interleaved=rng.random() < 0.5, fp32=fp32, positions=_log(rng, 64, 32768), fused=rng.random() < 0.5)
    if op == "tables":
        return dict(op=op, positions=_log(rng, 1, 131072), rot=rng.choice([128, 64, 32, 2 * rng.randint(1, 64)]), kind=rng.randint(0, 3),
                    base=rng.choice([10000.0, 500000.0, 1000000.0]), factor=rng.choice([1.0, 2.0, 4.0, 8.0, 32.0]), original=float(rng.choice([2048, 4096, 8192])))
    if op in ("append", "prompt"):
        d = rng.choice([64, 128])
        hkv = _log(rng, 1, 32)
        c = dict(op=op, hq=hkv * rng.choice([g for g in (1, 2, 4, 8) if g * hkv <= 64]), hkv=hkv, d=d, rot=rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)]),
                 interleaved=rng.random() < 0.3, page=rng.choice([0, 64, 128, 256]), fused=rng.random() < 0.5)
        width = (c["hq"] + 2 * hkv) * d
        if op == "append":
            new = rng.choice([1, 1, 1, rng.randint(2, 9)])
            return dict(c, batch=_log(rng, 1, 512 if hkv <= 8 else 64), new=new, lo=0, hi=_log(rng, 1, 2048))
        longest = _log(rng, 1, 4096)
        return dict(c, longest=longest, batch=_log(rng, 1, max(1, min(64, 8 * 4096 * 96 * 128 // (longest * width)))))
    if op == "norm":
        width = rng.choice([rng.choice([1024, 2048, 4096, 5120, 6656, 8192]), _log(rng, 8, 16384), 8 * _log(rng, 1, 2048)])
        out = rng.choice(["bf16", "bf16", "fp32", "e4m3", "e4m3"])
        return dict(op=op, rows=_log(rng, 1, max(1, min(65536, 2 ** 25 // width))), width=width, res=rng.random() < 0.7, x32=rng.random() < 0.2, r32=rng.random() < 0.3,
                    out=out, group=rng.choice([0, 128]) if out == "e4m3" else 0)
    group = rng.choice([32, 64, 128])
    rows = rng.choice([_log(rng, 1, 16), _log(rng, 1, 512)])
    k = group * _log(rng, max(1, 256 // group), 16384 // group)
    n = _log(rng, 16, max(16, min(28672, 2 ** 26 // k, 9 * 10 ** 9 // (rows * k))))
    return dict(op=op, rows=rows, k=k, n=n, group=group, zeros=rng.random() < 0.4, x8=rng.choice([-1, -1, 0, 128]), out32=rng.random() < 0.3)


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _bf16(g, *shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16) * std


def _tables(positions, rot, base=10000.0):
    """cos and sin of position * base^(-2 i / rot), as a user's program holds them."""
    i = torch.arange(rot // 2, device=DEV, dtype=torch.float64)
    ang = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * base ** (-2.0 * i / rot)
    return torch.cos(ang).float(), torch.sin(ang).float()


def _fill(t, g):
    """A cache's earlier rows: a random block, repeated."""
    flat = t.view(-1)
    m = min(flat.numel(), 1 << 20)
    block = torch.randn(m, generator=g, device=DEV, dtype=torch.float32).to(t.dtype)
    full = flat.numel() // m
    flat[:full * m].view(full, m).copy_(block.expand(full, m))
    flat[full * m:].copy_(block[:flat.numel() - full * m])


def _page_table(lens, new, rows):
    """Pages as the library hands them out from a fresh pool: for the cached rows of sequence 0, 1, ..., then for the new ones."""
    held = [-(-n // rows) for n in lens]
    table, at = [], 0
    for n in held:
        table.append(list(range(at, at + n)))
        at += n
    for b, n in enumerate(lens):
        while len(table[b]) * rows < n + new:
            table[b].append(at)
            at += 1
    wide = max(1, max(len(t) for t in table))
    return torch.tensor([t + [0] * (wide - len(t)) for t in table], dtype=torch.int64)


def _prepare_cache(c, seed):
    g = _gen(seed)
    prompt = c["op"] == "prompt"
    batch, hq, hkv, d, page = c["batch"], c["hq"], c["hkv"], c["d"], c["page"]
    cpu = torch.Generator().manual_seed(int(seed))
    if prompt:
        new = c["longest"]
        lens = torch.randint((new + 1) // 2, new + 1, (batch,), generator=cpu)
        lens[0] = new
        first = torch.zeros_like(lens)
        count = lens
        cap = new
    else:
        new = c["new"]
        lens = torch.randint(c["lo"], c["hi"] + 1, (batch,), generator=cpu)
        first = lens
        count = torch.full_like(lens, new)
        cap = c["hi"] + new
    held = lens.tolist()
    s = dict(c, cap=cap, new=new, lens=lens.to(DEV))
    if page:
        s["table"] = _page_table(held, 0 if prompt else new, page).to(DEV)
        s["pages"] = batch * -(-cap // page)  # a pool with room for every sequence at its longest
        shape = (s["pages"], hkv, page, d)
    else:
        shape = (batch, hkv, cap, d)
    if own:  # the cache that a user's program keeps; its slot is the pool
        from paper_2405_10637_b200 import binding as lk
        cfg = lk.make_config(1, 0, hq, hkv, d, batch, cap, page_rows=page, n_pages=s.get("pages", 0))
        s["cache"] = lk.Cache(cfg, device=torch.device(DEV, torch.cuda.current_device()))
        s["cache"].lckv_cache_reset(held)
        s["pool_k"], s["pool_v"] = s["cache"].slot_tensors(0)
    else:
        s["pool_k"], s["pool_v"] = (torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    _fill(s["pool_k"], g)
    _fill(s["pool_v"], g)
    if c["fused"]:
        qkv = _bf16(g, batch, new, hq + 2 * hkv, d)
        s["q"], s["k"], s["v"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
    else:
        s["q"], s["k"], s["v"] = _bf16(g, batch, new, hq, d), _bf16(g, batch, new, hkv, d), _bf16(g, batch, new, hkv, d)
    s["q_out"] = torch.zeros(batch, new, hq, d, dtype=torch.bfloat16, device=DEV)
    s["cos"], s["sin"] = _tables(cap + 1, c["rot"])
    # which (sequence, new token) there is, and its position
    i = torch.arange(new)
    there = i[None, :] < count[:, None]
    b, i = torch.nonzero(there, as_tuple=True)
    s["b"], s["i"] = b.to(DEV), i.to(DEV)
    s["pos"] = (first[b] + i).to(DEV)
    if own:
        s["rope"] = lk.make_rope(s["cos"], s["sin"], interleaved=c["interleaved"])
    return s


def _codes(g, c):
    n, k, group = c["n"], c["k"], c["group"]
    codes = (torch.randn((n, k), generator=g, device=DEV) * 2.5 + 8.0).round_().clamp_(0, 15).to(torch.uint8)
    packed = codes[:, 0::2] | (codes[:, 1::2] << 4)
    scales = ((torch.rand((n, k // group), generator=g, device=DEV) + 0.5) * (0.4 / math.sqrt(k))).to(torch.bfloat16)
    zeros = torch.randint(5, 11, (n, k // group), generator=g, device=DEV, dtype=torch.uint8) if c["zeros"] else None
    return packed, scales, zeros


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    if own:
        from paper_2405_10637_b200 import binding as lk
    if c["op"] == "rope":
        dt = torch.float32 if c["fp32"] else torch.bfloat16
        x = torch.randn((c["tokens"], c["heads"] * (2 if c["fused"] else 1), c["d"]), generator=g, device=DEV, dtype=dt)[:, :c["heads"]]
        pos = torch.randint(0, c["positions"], (c["tokens"],), generator=g, device=DEV, dtype=torch.int32)
        cos, sin = _tables(c["positions"], c["rot"])
        s = dict(c, x=x, pos=pos, cos=cos, sin=sin, y=torch.empty((c["tokens"], c["heads"], c["d"]), dtype=dt, device=DEV))
        if own:
            s["rope"] = lk.make_rope(cos, sin, interleaved=c["interleaved"])
        return s
    if c["op"] == "tables":
        # a scaling as a configuration states it; the amplitude differs from seed to seed
        amp = 1.0 + 0.1 * float(torch.rand((), generator=torch.Generator().manual_seed(int(seed))))
        s = dict(c, low=1.0, high=4.0, amplitude=amp)
        s["cos"], s["sin"] = (torch.empty((c["positions"], c["rot"] // 2), device=DEV) for _ in range(2))
        if own:
            s["scaling"] = lk.make_rope_scaling(c["kind"], c["base"], c["factor"], c["original"], s["low"], s["high"], amp)
        return s
    if c["op"] in ("append", "prompt"):
        return _prepare_cache(c, seed)
    if c["op"] == "norm":
        r, w = c["rows"], c["width"]
        f = {True: torch.float32, False: torch.bfloat16}
        s = dict(c, x=torch.randn((r, w), generator=g, device=DEV, dtype=f[c["x32"]]), weight=_bf16(g, w, std=0.1) + 1.0)
        if c["res"]:
            s["r"] = torch.randn((r, w), generator=g, device=DEV, dtype=f[c["r32"]]) * 3.0
            s["h"] = torch.empty_like(s["r"])
        s["y"] = torch.empty((r, w), device=DEV, dtype={"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}[c["out"]])
        if c["out"] == "e4m3":
            s["scale"] = torch.empty((r, -(-w // c["group"]) if c["group"] else 1), device=DEV)
        return s
    s = dict(c)
    s["codes"], s["scales"], s["zero"] = _codes(g, c)
    x = _randn(g, c["rows"], c["k"])
    if c["x8"] >= 0:  # 8-bit activations with their scales, as the norm leaves them
        blocks = -(-c["k"] // 128) if c["x8"] else 1
        s["x_scale"] = torch.rand((c["rows"], blocks), generator=g, device=DEV) * 0.01 + 0.005
        s["x"] = (x * 100.0).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    else:
        s["x"] = x.to(torch.bfloat16)
    s["y"] = torch.empty((c["rows"], c["n"]), device=DEV, dtype=torch.float32 if c["out32"] else torch.bfloat16)
    if own:  # weights are laid out once
        s["w"] = lk.lckv_quant_pack(s["codes"], s["scales"], s["zero"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------


def _rotate(x, cos, sin, rot, interleaved):
    """x [..., heads, d], cos and sin [..., rot / 2]: the first `rot` dimensions of each head turned, in fp32."""
    x = x.float()
    c, s = cos.unsqueeze(-2), sin.unsqueeze(-2)
    turned, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
    else:
        a, b = turned[..., :rot // 2], turned[..., rot // 2:]
        turned = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    return torch.cat((turned, rest), dim=-1)


def _plain_tables(s):
    rot, f = s["rot"], s["factor"]
    i = torch.arange(rot // 2, device=DEV, dtype=torch.float64)
    base = s["base"]
    if s["kind"] == 2 and rot > 2:
        base = base * f ** (rot / (rot - 2.0))
    theta = base ** (-2.0 * i / rot)
    if s["kind"] == 1:
        theta = theta / f
    if s["kind"] == 3:
        turns = s["original"] * theta / (2.0 * math.pi)
        keep = ((turns - s["low"]) / (s["high"] - s["low"])).clamp(0.0, 1.0)
        theta = theta * (keep + (1.0 - keep) / f)
    ang = torch.arange(s["positions"], device=DEV, dtype=torch.float64)[:, None] * theta
    s["cos"].copy_(torch.cos(ang) * s["amplitude"])
    s["sin"].copy_(torch.sin(ang) * s["amplitude"])
    return s["cos"], s["sin"]


def _plain_append(s):
    b, i, pos = s["b"], s["i"], s["pos"]
    cos, sin = s["cos"][pos], s["sin"][pos]
    s["q_out"][b, i] = _rotate(s["q"][b, i], cos, sin, s["rot"], s["interleaved"]).to(torch.bfloat16)
    k = _rotate(s["k"][b, i], cos, sin, s["rot"], s["interleaved"]).to(torch.bfloat16)
    if s["page"]:
        at, row = s["table"][b, pos // s["page"]], pos % s["page"]
    else:
        at, row = b, pos
    s["pool_k"][at, :, row] = k
    s["pool_v"][at, :, row] = s["v"][b, i]
    return s["q_out"], s["pool_k"], s["pool_v"]


def _plain_norm(s):
    h = s["x"].float()
    outs = []
    if s["res"]:
        h = h + s["r"].float()
        outs.append(h.to(s["r"].dtype))
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6) * s["weight"].float()
    if s["out"] != "e4m3":
        return [y.to(s["y"].dtype)] + outs
    rows, width = y.shape
    group = s["group"] or width
    full = torch.nn.functional.pad(y, (0, -width % group)).view(rows, -1, group)
    scale = full.abs().amax(-1) / E4M3_MAX
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    q = (full * inv.unsqueeze(-1)).clamp(-E4M3_MAX, E4M3_MAX).view(rows, -1)[:, :width]
    return [q.to(torch.float8_e4m3fn), scale] + outs


def _plain_quant(s):
    n, k, group = s["n"], s["k"], s["group"]
    c = s["codes"]
    w = torch.stack((c & 15, c >> 4), dim=-1).view(n, k // group, group).float()
    w = w - (s["zero"].float().unsqueeze(-1) if s["zero"] is not None else 8.0)
    w = (w * s["scales"].float().unsqueeze(-1)).view(n, k)
    x = s["x"].float()
    if s["x8"] >= 0:
        x = x * (s["x_scale"].repeat_interleave(128, dim=1)[:, :k] if s["x8"] else s["x_scale"])
    return (x @ w.t()).to(s["y"].dtype)


def run(s):
    op = s["op"]
    if not own:
        if op == "rope":
            p = s["pos"].long()
            return _rotate(s["x"], s["cos"][p], s["sin"][p], s["rot"], s["interleaved"]).to(s["x"].dtype)
        return {"tables": _plain_tables, "append": _plain_append, "prompt": _plain_append, "norm": _plain_norm, "quant": _plain_quant}[op](s)
    from paper_2405_10637_b200 import binding as lk
    if op == "rope":
        return lk.lckv_rope_apply(s["rope"], s["pos"], s["x"], s["y"])
    if op == "tables":
        return lk.lckv_rope_tables(s["cos"], s["sin"], s["scaling"])
    if op == "append":
        s["cache"].lckv_rope_append_kv(0, s["rope"], s["q"], s["k"], s["v"], s["q_out"])
        return s["q_out"], s["pool_k"], s["pool_v"]
    if op == "prompt":
        s["cache"].lckv_rope_prefill_write_kv(0, s["rope"], s["q"], s["k"], s["v"], s["q_out"])
        return s["q_out"], s["pool_k"], s["pool_v"]
    if op == "norm":
        lk.lckv_rms_norm(s["x"], s["weight"], s["y"], residual=s.get("r"), residual_out=s.get("h"), out_scale=s.get("scale"), scale_group=s["group"], eps=1e-6)
        return [s["y"]] + ([s["scale"]] if s["out"] == "e4m3" else []) + ([s["h"]] if s["res"] else [])
    return lk.lckv_quant_linear(s["w"], s["x"], s["y"], x_scale=s.get("x_scale"))


# ---- what a pass cannot do without ------------------------------------------------------------------------------------


def work(c):
    op = c["op"]
    if op == "rope":
        n = c["tokens"] * c["heads"]
        size = 4 if c["fp32"] else 2
        rows = min(c["tokens"], c["positions"])
        return {"bytes": 2 * n * c["d"] * size + 4 * c["tokens"] + rows * c["rot"] * 4, "flops": 3 * n * c["rot"]}
    if op == "tables":
        return {"bytes": c["positions"] * c["rot"] * 4, "flops": 40 * c["positions"] * c["rot"] // 2}
    if op in ("append", "prompt"):
        # ragged prompts: lengths between half and all of the longest
        tokens = c["batch"] * c["new"] if op == "append" else c["longest"] + (c["batch"] - 1) * (c["longest"] * 3 // 4)
        rows = min(tokens, (c["hi"] + c["new"]) if op == "append" else c["longest"])
        return {"bytes": 4 * tokens * (c["hq"] + 2 * c["hkv"]) * c["d"] + rows * c["rot"] * 4 + 4 * c["batch"],
                "flops": 3 * tokens * (c["hq"] + c["hkv"]) * c["rot"]}
    if op == "norm":
        n = c["rows"] * c["width"]
        per = (4 if c["x32"] else 2) + (2 * (4 if c["r32"] else 2) if c["res"] else 0) + {"bf16": 2, "fp32": 4, "e4m3": 1}[c["out"]]
        scales = (c["rows"] * (-(-c["width"] // c["group"]) if c["group"] else 1) * 4) if c["out"] == "e4m3" else 0
        return {"bytes": n * per + scales + 2 * c["width"], "flops": 6 * n}
    n, k, m = c["n"], c["k"], c["rows"]
    x = m * k * (2 if c["x8"] < 0 else 1) + (4 * m * (-(-k // 128) if c["x8"] else 1) if c["x8"] >= 0 else 0)
    return {"bytes": n * k // 2 + n * (k // c["group"]) * (3 if c["zeros"] else 2) + x + m * n * (4 if c["out32"] else 2), "flops": 2 * m * n * k}


# ---- the same from the definitions, in 64 bits ------------------------------------------------------------------------


def _exact_turn(x, cos, sin, rot, interleaved):
    """Pair j of a head is a complex number; the rotation multiplies it by cos + i sin."""
    half = rot // 2
    j = torch.arange(half, device=DEV)
    re, im = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
    z = torch.complex(x[..., re].double(), x[..., im].double()) * torch.complex(cos.double(), sin.double())[..., None, :]
    y = x.double().clone()
    y[..., re], y[..., im] = z.real, z.imag
    return y


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    op = s["op"]
    if op == "rope":
        p = s["pos"].long()
        return _exact_turn(s["x"], s["cos"][p], s["sin"][p], s["rot"], s["interleaved"])
    if op == "tables":
        rot, f, rows = s["rot"], s["factor"], []
        for i in range(rot // 2):
            th = s["base"] ** (-2.0 * i / rot)
            if s["kind"] == 1:
                th /= f
            elif s["kind"] == 2 and rot > 2:
                th = (s["base"] * f ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
            elif s["kind"] == 3:
                t = s["original"] / (2.0 * math.pi / th)
                g = 0.0 if t < s["low"] else 1.0 if t > s["high"] else (t - s["low"]) / (s["high"] - s["low"])
                th = (1.0 - g) * th / f + g * th
            rows.append(th)
        ang = torch.outer(torch.arange(s["positions"], dtype=torch.float64, device=DEV), torch.tensor(rows, dtype=torch.float64, device=DEV))
        return s["amplitude"] * torch.cos(ang), s["amplitude"] * torch.sin(ang)
    if op in ("append", "prompt"):
        q, k, v = s["q_out"].double(), s["pool_k"].clone(), s["pool_v"].clone()
        cos, sin = s["cos"][s["pos"]], s["sin"][s["pos"]]
        q[s["b"], s["i"]] = _exact_turn(s["q"][s["b"], s["i"]], cos, sin, s["rot"], s["interleaved"])
        kr = _exact_turn(s["k"][s["b"], s["i"]], cos, sin, s["rot"], s["interleaved"])
        k = k.double()
        # one flat row index per (token, head) of the pool
        heads = torch.arange(s["hkv"], device=DEV)
        if s["page"]:
            page = s["table"][s["b"], torch.div(s["pos"], s["page"], rounding_mode="floor")]
            at = (page[:, None] * s["hkv"] + heads) * s["page"] + (s["pos"] % s["page"])[:, None]
        else:
            at = (s["b"][:, None] * s["hkv"] + heads) * s["cap"] + s["pos"][:, None]
        k.view(-1, s["d"])[at] = kr
        v.view(-1, s["d"])[at] = s["v"][s["b"], s["i"]]
        return q, k, v.double()
    if op == "norm":
        h = s["x"].double() + (s["r"].double() if s["res"] else 0.0)
        y = h / torch.sqrt(torch.sum(h * h, 1, keepdim=True) / s["width"] + 1e-6) * s["weight"].double()
        if s["out"] != "e4m3":
            return [y] + ([h] if s["res"] else [])
        # the 8-bit values before their rounding
        step = s["group"] or s["width"]
        top = torch.stack([y[:, a:a + step].abs().max(1).values for a in range(0, s["width"], step)], 1) / E4M3_MAX
        unit = top.repeat_interleave(step, 1)[:, :s["width"]]
        q = torch.where(unit > 0, y / unit, torch.zeros_like(y))
        return [q, top] + ([h] if s["res"] else [])
    n, k = s["n"], s["k"]
    w = torch.empty((n, k), dtype=torch.float64, device=DEV)
    w[:, 0::2], w[:, 1::2] = (s["codes"] % 16).double(), torch.div(s["codes"], 16, rounding_mode="floor").double()
    w -= s["zero"].double().repeat_interleave(s["group"], 1) if s["zero"] is not None else 8.0
    w *= s["scales"].double().repeat_interleave(s["group"], 1)
    x = s["x"].double()
    if s["x8"] > 0:
        x = x * s["x_scale"].double().repeat_interleave(128, 1)[:, :k]
    elif s["x8"] == 0:
        x = x * s["x_scale"].double()
    return torch.matmul(x, w.mT)
