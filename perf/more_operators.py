"""What a network that classifies nodes has besides its layers, as cases to be timed: rows looked up in a table and the table's gradient, dropout whose
mask is never stored, log probabilities of given classes with entropy, alternatives and gradient, and products of matrices held in 8 bits (e4m3 codes that share a
power of two over 128 columns).  Sizes are those of the layers that the package's partitions stand for and generic ones.

`run` computes a case in its plain form, elementary torch operations in 32 bits (64 where a table's gradient sums many rows), or (own = True) by the package's
calls.  `exact` computes the definitions in 64 bits, written apart from the plain form.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
RANDOM_TAG = 0x44524F50                 # last counter word of dropout's numbers
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(kind, name=None, **sizes):
    case = dict(kind=kind, **sizes)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # The smallest partition in use, a narrow hidden layer: a few microseconds, what counts is the call.
        _case("dropout", "dropout tiny", rows=2_000, dim=128, type="f32", add=False, p=0.5),
        # A hidden layer of one of eight parts of a graph, in 16 bits, added to the layer's input (a residual connection).
        _case("dropout", "dropout residual", rows=376_000, dim=256, type="bf16", add=True, p=0.1),
        # A few hundred rows asked for while serving: latency.
        _case("lookup", "lookup few", ids=512, entries=32_000, dim=1_024, type="bf16"),
        # A training step over a batch of sampled nodes, rows of an odd width: lookup, then the whole table's gradient.
        _case("embedding step", "embedding step ragged", ids=9_001, entries=20_000, dim=301, type="bf16"),
        # A training step over many positions of a vocabulary, frequencies falling as a power law.
        _case("embedding step", "embedding step large", ids=131_072, entries=50_000, dim=1_024, type="f32"),
        # The answer of a node classifier of 41 classes and its gradients; most nodes have no label.  Rows are a quarter of a wave.
        _case("loss step", "loss step 41", rows=58_000, classes=41, type="f32", entropy=True),
        # Many classes in 16 bits, rows of odd length: bound by reading the logits twice and writing their gradient.
        _case("loss step", "loss step wide", rows=4_096, classes=32_001, type="bf16", entropy=False),
        # A few rows while serving, with the twenty most likely answers.
        _case("alternatives", "alternatives few", rows=3, classes=128_000, type="bf16", top=20),
        # A layer's product in a forward pass: the features are quantised and multiplied with weights kept in 8 bits.
        _case("linear forward", "linear forward 300", rows=179_000, k=300, n=256, type="bf16"),
        # Its gradients in a backward pass: the output's gradient is quantised by rows and by columns and gives the input's and the weight's.
        _case("linear backward", "linear backward 602", rows=58_000, k=602, n=256, type="f32"),
        # A few rows at a time, wide layer, both operands kept in 8 bits: latency and the reading of the weights.
        _case("product", "product few rows", rows=5, k=4_096, n=8_192, type="bf16"),
        # The same layer over many rows: bound by the matrix cores.
        _case("product", "product large", rows=8_192, k=4_096, n=8_192, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["dropout", "lookup", "embedding step", "loss step", "alternatives", "linear forward", "linear backward", "product"])
    kind_of_type = rng.choice(["f32", "bf16"])
    width = _log(rng, 16, 2_048)
    if rng.random() < 0.5:
        width = max(8, width // 8 * 8)
    if kind == "dropout":
        return _case(kind, rows=min(_log(rng, 1, 376_000), 376_000 * 256 // width), dim=width, type=kind_of_type, add=rng.random() < 0.5,
                     p=round(rng.uniform(0.0, 0.9), 3))
    if kind in ("lookup", "embedding step"):
        most = 131_072 * 1_024 // width
        return _case(kind, ids=min(_log(rng, 1, 306_000), most), entries=min(_log(rng, 2, 456_000), most // 2), dim=width, type=kind_of_type)
    if kind in ("loss step", "alternatives"):
        classes = _log(rng, 2, 131_000)
        most = 4_096 * 32_001 // classes
        if kind == "loss step":
            return _case(kind, rows=min(_log(rng, 1, 179_000), most), classes=classes, type=kind_of_type, entropy=rng.random() < 0.5)
        return _case(kind, rows=min(_log(rng, 1, 256), most), classes=classes, type=kind_of_type, top=rng.randint(1, min(32, classes)))
    n = _log(rng, 16, 2_048)
    rows = _log(rng, 16, 306_000) if kind != "product" else _log(rng, 1, 306_000)
    rows = max(1, min(rows, 306_000 * 256 // max(width, n), 8_192 * 4_096 * 8_192 // (width * n)))
    return _case(kind, rows=rows, k=width, n=n, type=kind_of_type)


# ---- inputs ------------------------------------------------------------------------------------------------------------------------

def _rows(rows, dim, dtype):
    """An uninitialised matrix whose rows cover whole 128-byte lines."""
    line = 128 // dtype.itemsize
    return torch.empty(rows, -(-dim // line) * line, dtype=dtype, device=DEV)[:, :dim]


def _normal(gen, rows, dim, dtype, scale=1.0):
    x = _rows(rows, dim, dtype)
    x.copy_(torch.randn(rows, dim, generator=gen, device=DEV).mul_(scale))
    return x


def _gradient(gen, rows, dim, dtype):
    """Gradients of nodes: of a few the loss knows nothing."""
    g = torch.randn(rows, dim, generator=gen, device=DEV) * 1e-3
    g *= torch.rand(rows, 1, generator=gen, device=DEV) > 0.05
    return g.to(dtype)


def _popular(gen, n, entries):
    """Ids whose frequencies fall about as 1 / rank, the ranks scattered over the table; one in fifty is -1, a place that is filled up."""
    rank = torch.exp(torch.rand(n, generator=gen, device=DEV, dtype=torch.float64) * math.log(entries + 1)).long().clamp_(1, entries) - 1
    ids = torch.randperm(entries, generator=gen, device=DEV)[rank]
    ids[torch.rand(n, generator=gen, device=DEV) < 0.02] = -1
    return ids.int()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dtype, kind = TYPES[case["type"]], case["kind"]
    state = dict(case=dict(case), dtype=dtype, kept={})
    if kind == "dropout":
        state["x"] = _normal(gen, case["rows"], case["dim"], dtype)
        state["add"] = _normal(gen, case["rows"], case["dim"], dtype) if case["add"] else None
        state["seed"] = seed * 2_654_435_761 + 97
    elif kind in ("lookup", "embedding step"):
        state["table"] = _normal(gen, case["entries"], case["dim"], dtype)
        state["ids"] = _popular(gen, case["ids"], case["entries"])
        state["scale"] = math.sqrt(case["dim"])
        if kind == "embedding step":
            state["dy"] = _gradient(gen, case["ids"], case["dim"], dtype)
    elif kind in ("loss step", "alternatives"):
        rows, classes = case["rows"], case["classes"]
        state["logits"] = (torch.randn(rows, classes, generator=gen, device=DEV) * 2.5).to(dtype)
        state["targets"] = torch.randint(classes, (rows,), generator=gen, device=DEV, dtype=torch.int32)
        if kind == "loss step":
            labelled = torch.rand(rows, generator=gen, device=DEV) < (0.3 if case["entropy"] else 0.98)
            state["targets"][~labelled] = -1
            state["scale"] = -1.0 / rows
            state["dentropy"] = torch.full((rows,), 0.01, device=DEV) if case["entropy"] else None
    elif kind == "linear forward":
        state["x"] = torch.randn(case["rows"], case["k"], generator=gen, device=DEV).to(dtype)
        state["w"] = _quantize(torch.randn(case["n"], case["k"], generator=gen, device=DEV) / math.sqrt(case["k"]), tiles=True)
    elif kind == "linear backward":
        state["dz"] = _gradient(gen, case["rows"], case["n"], dtype)
        state["wt"] = _quantize((torch.randn(case["n"], case["k"], generator=gen, device=DEV) / math.sqrt(case["k"])).t(), tiles=True)
        state["xt"] = _quantize(torch.randn(case["rows"], case["k"], generator=gen, device=DEV).relu_().t())
    else:
        state["a"] = _quantize(torch.randn(case["rows"], case["k"], generator=gen, device=DEV))
        state["b"] = _quantize(torch.randn(case["n"], case["k"], generator=gen, device=DEV) / math.sqrt(case["k"]), tiles=True)
    return state


# ---- the plain forms -----------------------------------------------------------------------------------------------------------------
# A matrix in 8 bits of r rows and c columns: codes [r, 128 ceil(c / 128)] in e4m3, what lies beyond column c code 0; scales [ceil(c / 128), 16 ceil(r / 16)],
# of a row and 128 columns the exponent of a power of two plus 127, what lies beyond row r 0.

def _random16(rows, columns, seed):
    """[rows, columns] integers below 2^16 (columns a multiple of 8): Philox4x32-10, counter (column / 8, row low, row high, tag), key = seed."""
    low = 0xFFFFFFFF
    c0 = torch.arange(columns // 8, device=DEV).expand(rows, -1)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(-1, columns // 8)
    c2, c3 = torch.zeros_like(c0), torch.full_like(c0, RANDOM_TAG)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, columns)


def _quantize(x, tiles=False):
    """(codes, scales) of a matrix, a scale for 128 columns of a row or (tiles) of 128 rows."""
    rows, cols = x.shape
    padded = torch.nn.functional.pad(x.float(), (0, -cols % 128)).contiguous()
    most = padded.reshape(rows, -1, 128).abs().amax(2)
    if tiles:
        most = torch.nn.functional.pad(most, (0, 0, 0, -rows % 128)).reshape(-1, 128, most.shape[1]).amax(1).repeat_interleave(128, 0)[:rows]
    bits = most.contiguous().view(torch.int32)
    byte = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp_(min=0)
    y = padded.reshape(rows, -1, 128) * ((254 - byte) << 23).view(torch.float32)[:, :, None]
    codes = y.reshape(rows, -1).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, torch.nn.functional.pad(byte.to(torch.uint8).t(), (0, -rows % 16)).contiguous()


def _dequantize(packed, cols):
    codes, scales = packed
    rows = codes.shape[0]
    byte = scales[:, :rows].t().int()
    scale = torch.where(byte == 0, 0x400000, byte << 23).view(torch.float32)
    return (codes.view(torch.float8_e4m3fn).float().reshape(rows, -1, 128) * scale[:, :, None]).reshape(rows, -1)[:, :cols]


def _looked_up(state):
    ids = state["ids"].long()
    out = state["table"][ids.clamp(min=0)].float() * state["scale"]
    return torch.where((ids >= 0)[:, None], out, 0.0).to(state["dtype"])


def _log_probabilities(state):
    """(logits less their largest, log of the sum of their exponentials) of each row."""
    x = state["logits"].float()
    x = x - x.amax(1, keepdim=True)
    return x, x.exp().sum(1, keepdim=True).log()


def _plain(state):
    case, dtype, kind = state["case"], state["dtype"], state["case"]["kind"]
    if kind == "dropout":
        dim, t = case["dim"], int(case["p"] * 65536 + 0.5)
        kept = _random16(case["rows"], -(-dim // 8) * 8, state["seed"])[:, :dim] >= t
        y = torch.where(kept, state["x"].float() * (65536 / (65536 - t)), 0.0)
        return (y if state["add"] is None else state["add"].float() + y).to(dtype)
    if kind == "lookup":
        return _looked_up(state)
    if kind == "embedding step":
        entries = case["entries"]
        ids = state["ids"].long()
        sums = torch.zeros(entries + 1, case["dim"], dtype=torch.float64, device=DEV)
        sums.index_add_(0, torch.where(ids < 0, entries, ids), state["dy"].double())
        return dict(out=_looked_up(state), dtable=(sums[:entries] * state["scale"]).float())
    if kind == "loss step":
        x, l = _log_probabilities(state)
        logp = x - l
        p = logp.exp()
        targets = state["targets"].long()
        there, at = targets >= 0, targets.clamp(min=0)
        entropy = -(p * logp).sum(1)
        dx = -p * there[:, None]
        dx.scatter_add_(1, at[:, None], there[:, None].float())
        if state["dentropy"] is not None:
            dx -= state["dentropy"][:, None] * p * (logp + entropy[:, None])
        dx *= state["scale"]
        return dict(logp=torch.where(there, logp.gather(1, at[:, None])[:, 0], 0.0), entropy=entropy, dlogits=dx.to(dtype))
    if kind == "alternatives":
        x, l = _log_probabilities(state)
        logp = x - l
        order = x.sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]
        return dict(logp=logp.gather(1, state["targets"].long()[:, None])[:, 0], entropy=-(logp.exp() * logp).sum(1),
                    top_logp=logp.gather(1, order), top_index=order.int())
    if kind == "linear forward":
        return (_dequantize(_quantize(state["x"]), case["k"]) @ _dequantize(state["w"], case["k"]).t()).to(dtype)
    if kind == "linear backward":
        dz = state["dz"]
        rows, columns = _dequantize(_quantize(dz), case["n"]), _dequantize(_quantize(dz.t()), case["rows"])
        return dict(dx=(rows @ _dequantize(state["wt"], case["n"]).t()).to(dtype), dw=columns @ _dequantize(state["xt"], case["rows"]).t())
    return (_dequantize(state["a"], case["k"]) @ _dequantize(state["b"], case["k"]).t()).to(dtype)


# ---- the package's calls -------------------------------------------------------------------------------------------------------------

def _buffers(state, make):
    """Outputs, workspaces and intermediate matrices, which a program keeps from step to step."""
    if not state["kept"]:
        state["kept"].update(make())
    return state["kept"]


def _bytes(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)


def _own(state):
    from paper_2306_01381_amd import binding as B
    case, dtype, kind = state["case"], state["dtype"], state["case"]["kind"]
    if kind == "dropout":
        rows, dim = case["rows"], case["dim"]
        kept = _buffers(state, lambda: dict(y=_rows(rows, dim, dtype)))
        B.adaqp_dropout(state["x"], dim, case["p"], state["seed"], kept["y"], add=state["add"])
        return kept["y"]
    if kind == "lookup":
        kept = _buffers(state, lambda: dict(out=_rows(case["ids"], case["dim"], dtype)))
        B.adaqp_embedding_forward(state["table"], case["dim"], state["ids"], state["scale"], kept["out"])
        return kept["out"]
    if kind == "embedding step":
        n, entries, dim = case["ids"], case["entries"], case["dim"]
        need = lambda: max(B.adaqp_embedding_sort_workspace_bytes(n, entries), B.adaqp_embedding_backward_workspace_bytes(n, dim))  # noqa: E731
        kept = _buffers(state, lambda: dict(out=_rows(n, dim, dtype), dtable=_rows(entries, dim, torch.float32), work=_bytes(need()),
                                            sorted_ids=torch.empty(n, dtype=torch.int32, device=DEV), order=torch.empty(n, dtype=torch.int32, device=DEV)))
        B.adaqp_embedding_forward(state["table"], dim, state["ids"], state["scale"], kept["out"])
        B.adaqp_embedding_sort(state["ids"], entries, kept["sorted_ids"], kept["order"], kept["work"])
        B.adaqp_embedding_backward(state["dy"], dim, kept["sorted_ids"], kept["order"], state["scale"], False, kept["dtable"], kept["work"])
        return dict(out=kept["out"], dtable=kept["dtable"])
    if kind == "loss step":
        rows, classes = case["rows"], case["classes"]
        kept = _buffers(state, lambda: dict(logp=torch.empty(rows, device=DEV), entropy=torch.empty(rows, device=DEV), stats=torch.empty(rows, 2, device=DEV),
                                            dlogits=torch.empty_like(state["logits"]), work=_bytes(B.adaqp_logprob_workspace_bytes(rows, classes, 0))))
        B.adaqp_logprob_forward(state["logits"], classes, state["targets"], kept["logp"], kept["entropy"], kept["stats"], None, None, kept["work"])
        B.adaqp_logprob_backward(state["logits"], classes, state["targets"], kept["stats"], kept["entropy"], None, state["dentropy"], state["scale"], kept["dlogits"])
        return dict(logp=kept["logp"], entropy=kept["entropy"], dlogits=kept["dlogits"])
    if kind == "alternatives":
        rows, classes, top = case["rows"], case["classes"], case["top"]
        kept = _buffers(state, lambda: dict(logp=torch.empty(rows, device=DEV), entropy=torch.empty(rows, device=DEV), top_logp=torch.empty(rows, top, device=DEV),
                                            top_index=torch.empty(rows, top, dtype=torch.int32, device=DEV),
                                            work=_bytes(B.adaqp_logprob_workspace_bytes(rows, classes, top))))
        B.adaqp_logprob_forward(state["logits"], classes, state["targets"], kept["logp"], kept["entropy"], None, kept["top_logp"], kept["top_index"], kept["work"])
        return dict(logp=kept["logp"], entropy=kept["entropy"], top_logp=kept["top_logp"], top_index=kept["top_index"])
    rows, k, n = case["rows"], case["k"], case["n"]
    if kind == "linear forward":
        kept = _buffers(state, lambda: dict(x=B.f8_empty(rows, k, DEV), z=torch.empty(rows, n, dtype=dtype, device=DEV),
                                            work=_bytes(B.adaqp_f8_matmul_workspace_bytes(rows, n, k))))
        B.adaqp_f8_quantize(state["x"], k, B.F8_ROWS, kept["x"], None)
        B.adaqp_f8_matmul(kept["x"], state["w"], k, kept["z"], kept["work"])
        return kept["z"]
    if kind == "linear backward":
        need = lambda: max(B.adaqp_f8_matmul_workspace_bytes(rows, k, n), B.adaqp_f8_matmul_workspace_bytes(n, k, rows))  # noqa: E731
        kept = _buffers(state, lambda: dict(rows=B.f8_empty(rows, n, DEV), columns=B.f8_empty(n, rows, DEV), dx=torch.empty(rows, k, dtype=dtype, device=DEV),
                                            dw=torch.empty(n, k, device=DEV), work=_bytes(need())))
        B.adaqp_f8_quantize(state["dz"], n, B.F8_ROWS, kept["rows"], kept["columns"])
        B.adaqp_f8_matmul(kept["rows"], state["wt"], n, kept["dx"], kept["work"])
        B.adaqp_f8_matmul(kept["columns"], state["xt"], rows, kept["dw"], kept["work"])
        return dict(dx=kept["dx"], dw=kept["dw"])
    kept = _buffers(state, lambda: dict(out=torch.empty(rows, n, dtype=dtype, device=DEV), work=_bytes(B.adaqp_f8_matmul_workspace_bytes(rows, n, k))))
    B.adaqp_f8_matmul(state["a"], state["b"], k, kept["out"], kept["work"])
    return kept["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------------------

def work(case):
    kind, size = case["kind"], TYPES[case["type"]].itemsize
    packed = lambda rows, cols: rows * cols * (1 + 1 / 128)  # noqa: E731
    if kind == "dropout":
        cells = case["rows"] * case["dim"]
        return dict(bytes=size * cells * (3 if case["add"] else 2), flops=3 * cells)
    if kind in ("lookup", "embedding step"):
        cells = case["ids"] * case["dim"]
        # a row that is looked up several times is read once: at most as many as the table has
        read = min(case["ids"], case["entries"]) * case["dim"] * size
        if kind == "lookup":
            return dict(bytes=read + size * cells + 4 * case["ids"], flops=cells)
        return dict(bytes=read + 2 * size * cells + 4 * case["ids"] + 4 * case["entries"] * case["dim"], flops=3 * cells)
    if kind in ("loss step", "alternatives"):
        rows, cells = case["rows"], case["rows"] * case["classes"]
        if kind == "loss step":
            return dict(bytes=2 * size * cells + 12 * rows, flops=12 * cells)
        return dict(bytes=size * cells + 12 * rows + 8 * rows * case["top"], flops=6 * cells)
    rows, k, n = case["rows"], case["k"], case["n"]
    if kind == "linear forward":
        return dict(bytes=size * rows * (k + n) + packed(n, k), flops=2 * rows * k * n)
    if kind == "linear backward":
        return dict(bytes=size * rows * (n + k) + packed(k, n) + packed(k, rows) + 4 * n * k, flops=4 * rows * k * n)
    return dict(bytes=packed(rows, k) + packed(n, k) + size * rows * n, flops=2 * rows * k * n)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------------------

def _philox(rows, columns, seed):
    """The numbers that _random16 gives, from the generator's definition on 64-bit words of the host."""
    word, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    x = [np.broadcast_to(np.arange(columns // 8, dtype=np.uint64), (rows, columns // 8)).copy(),
         np.broadcast_to(np.arange(rows, dtype=np.uint64)[:, None], (rows, columns // 8)).copy(),
         np.zeros((rows, columns // 8), np.uint64), np.full((rows, columns // 8), RANDOM_TAG, np.uint64)]
    key = [seed % (1 << 32), (seed >> 32) % (1 << 32)]
    for _ in range(10):
        first, second = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(second >> shift) ^ x[1] ^ np.uint64(key[0]), second & word, (first >> shift) ^ x[3] ^ np.uint64(key[1]), first & word]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    out = np.empty((rows, columns // 8, 8), np.int32)
    for j in range(8):
        out[:, :, j] = (x[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)
    return torch.from_numpy(out.reshape(rows, columns)).to(DEV)


def _exact_f8(x, tiles=False):
    """The values that a matrix's 8-bit form stands for: in units of 2^e, the smallest in which the block's largest magnitude is at most 448, each to the nearest
    multiple of an eighth of its power of two, at least 2^-9."""
    rows, cols = x.shape
    full = torch.zeros(-(-rows // 128) * 128 if tiles else rows, -(-cols // 128) * 128, dtype=torch.float64, device=DEV)
    full[:rows, :cols] = x
    block = full.reshape(-1, 128 if tiles else 1, full.shape[1] // 128, 128)
    most = block.abs().amax((1, 3), keepdim=True)
    fraction, exponent = torch.frexp(most / 448)                 # most / 448 = fraction 2^exponent, fraction in [1/2, 1)
    e = torch.where(most == 0, -127.0, (exponent.double() - (fraction == 0.5).double()).clamp(min=-127))
    y = block / torch.exp2(e)
    _, power = torch.frexp(y)
    step = torch.exp2((power.double() - 4).clamp(min=-9))
    return (torch.round(y / step) * step * torch.exp2(e)).reshape(full.shape)[:rows, :cols]


def _exact_kept(packed, cols):
    codes, scales = (t.cpu().numpy() for t in packed)
    all_codes = np.arange(256)
    field, last = all_codes // 8 % 16, all_codes % 8
    values = np.where(field == 0, last / 8 * 2.0 ** -6, (1 + last / 8) * 2.0 ** (field - 7.0)) * np.where(all_codes >= 128, -1, 1)
    rows = codes.shape[0]
    e = scales[:, :rows].T.astype(np.float64) - 127
    return torch.from_numpy((values[codes].reshape(rows, -1, 128) * np.exp2(e)[:, :, None]).reshape(rows, -1)[:, :cols].copy()).to(DEV)


def _exact_rows(state):
    """Of each row of the table that is asked for, scale times it."""
    ids = state["ids"].long()
    out = torch.zeros(ids.numel(), state["table"].shape[1], dtype=torch.float64, device=DEV)
    out[ids >= 0] = state["table"].double()[ids[ids >= 0]] * state["scale"]
    return out


def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    if kind == "dropout":
        dim, t = case["dim"], int(case["p"] * 65536 + 0.5)
        y = state["x"].double() / (1 - t / 65536)
        y[_philox(case["rows"], -(-dim // 8) * 8, state["seed"])[:, :dim] < t] = 0.0
        return y if state["add"] is None else state["add"].double() + y
    if kind == "lookup":
        return _exact_rows(state)
    if kind == "embedding step":
        # sums of neighbours in sorted order, as differences of the running sums of each column in blocks of columns
        ids, entries, dim = state["ids"].long(), case["entries"], case["dim"]
        ids, order = ids.sort()
        begin = torch.searchsorted(ids, torch.arange(entries + 1, device=DEV))
        dtable = torch.empty(entries, dim, dtype=torch.float64, device=DEV)
        for at in range(0, dim, 128):
            running = torch.zeros(ids.numel() + 1, min(128, dim - at), dtype=torch.float64, device=DEV)
            torch.cumsum(state["dy"][:, at:at + 128].double()[order], 0, out=running[1:])
            dtable[:, at:at + 128] = (running[begin[1:]] - running[begin[:-1]]) * state["scale"]
        return dict(out=_exact_rows(state), dtable=dtable)
    if kind in ("loss step", "alternatives"):
        x = state["logits"].double()
        rows = torch.arange(case["rows"], device=DEV)
        lse = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[:, None])
        entropy = lse - (p * x).sum(1)
        targets = state["targets"].long()
        if kind == "alternatives":
            # ties to the lowest index: negated values in ascending stable order
            index = torch.argsort(-x, dim=1, stable=True)[:, :case["top"]]
            return dict(logp=x[rows, targets] - lse, entropy=entropy, top_logp=x[rows[:, None], index] - lse[:, None], top_index=index.int())
        labelled = targets >= 0
        logp = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
        logp[labelled] = x[rows[labelled], targets[labelled]] - lse[labelled]
        dx = torch.zeros_like(x)
        dx[labelled] = -p[labelled]
        dx[rows[labelled], targets[labelled]] += 1.0
        if state["dentropy"] is not None:
            # H = lse - sum p x:  dH / dx_j = -p_j (x_j - sum p x)
            dx += state["dentropy"].double()[:, None] * p * ((p * x).sum(1, keepdim=True) - x)
        return dict(logp=logp, entropy=entropy, dlogits=dx * state["scale"])
    if kind == "linear forward":
        return _exact_f8(state["x"]) @ _exact_kept(state["w"], case["k"]).t()
    if kind == "linear backward":
        rows, columns = _exact_f8(state["dz"]), _exact_f8(state["dz"].t())
        return dict(dx=rows @ _exact_kept(state["wt"], case["n"]).t(), dw=columns @ _exact_kept(state["xt"], case["rows"]).t())
    return _exact_kept(state["a"], case["k"]) @ _exact_kept(state["b"], case["k"]).t()
