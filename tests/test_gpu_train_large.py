"""What adaqp_train.h declares at sizes whose places pass 32 bits or whose pieces pass 2^31.  Parts of the results are compared with calls of few rows, which the other tests compare with the
definitions.  Each test says how much device memory it needs and is skipped where there is less."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2306_01381_amd import binding as B                      # noqa: E402

DEV = "cuda:0"
GIB = 1 << 30


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.empty_cache()


def _say(*what):
    print(*what, flush=True)
    sys.stdout.flush()


def _need(gib):
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < (gib + 4) * GIB:
        pytest.skip(f"{free // GIB} GiB of device memory are free, {gib + 4} are needed")


def _random(rows, cols, seed, dtype=torch.bfloat16):
    """Normal numbers, made in pieces of at most 2^28."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.empty(rows, cols, dtype=dtype, device=DEV)
    step = max(1, (1 << 28) // cols)
    for at in range(0, rows, step):
        t[at:at + step].normal_(generator=gen)
    return t


def _ends(n, k=1000):
    """The first and last rows, and some around the middle."""
    return [(0, k), (n // 2 - k, n // 2 + k), (n - k, n)]


@pytest.mark.parametrize("rows,dim", [((1 << 24) + 3, 136), ((1 << 31) + 10, 1)])
def test_dropout(rows, dim):
    _need(10)
    _say("dropout", rows, dim)
    x = _random(rows, dim, 1)
    y = torch.empty_like(x)
    B.adaqp_dropout(x, dim, 0.4, 7, y)
    for a, b in _ends(rows):
        want = torch.empty_like(x[a:b])
        B.adaqp_dropout(x[a:b], dim, 0.4, 7, want, first_row=a)
        assert torch.equal(y[a:b], want)


@pytest.mark.parametrize("entries,n,dim", [((1 << 21) + 5, (1 << 21) + 70, 1100), (50, (1 << 30) + 8, 9)])
def test_embedding_forward(entries, n, dim):
    _need(26)
    _say("embedding forward", entries, n, dim)
    table = _random(entries, dim, 2)
    ids = torch.randint(-1, entries, (n,), device=DEV, dtype=torch.int32, generator=torch.Generator(device=DEV).manual_seed(1))
    ids[-1], ids[n // 2], ids[0] = entries - 1, entries - 2, entries - 1
    out = torch.empty(n, dim, dtype=torch.bfloat16, device=DEV)
    B.adaqp_embedding_forward(table, dim, ids, 1.0, out)
    for a, b in _ends(n):
        at = ids[a:b].long()
        assert torch.equal(out[a:b], torch.where((at >= 0)[:, None], table[at.clamp(min=0)], 0))


def test_embedding_backward():
    """Rows of both matrices past 2^31 elements; ids in descending order, two of each, so that a row is the sum of two neighbours."""
    entries, dim = (1 << 21) + 5, 1100
    n = 2 * entries
    _need(36)
    _say("embedding backward", entries, n, dim)
    dy = _random(n, dim, 3)
    ids = torch.arange(entries - 1, -1, -1, device=DEV, dtype=torch.int32).repeat_interleave(2)
    by_id, order = torch.empty_like(ids), torch.empty_like(ids)
    work = torch.empty(max(B.adaqp_embedding_sort_workspace_bytes(n, entries), B.adaqp_embedding_backward_workspace_bytes(n, dim)), dtype=torch.uint8, device=DEV)
    B.adaqp_embedding_sort(ids, entries, by_id, order, work)
    assert torch.equal(by_id.long(), torch.arange(n, device=DEV) // 2)
    assert torch.equal(order[0::2].long(), torch.arange(n - 2, -1, -2, device=DEV)) and torch.equal(order[1::2], order[0::2] + 1)
    dtable = torch.empty(entries, dim, device=DEV)
    B.adaqp_embedding_backward(dy, dim, by_id, order, 1.0, False, dtable, work)
    for a, b in _ends(entries):
        want = dy[n - 2 * b:n - 2 * a].float().view(b - a, 2, dim).sum(1).flip(0)
        assert torch.equal(dtable[a:b], want)


@pytest.mark.parametrize("rows,classes", [(20_000, 128_001), ((1 << 30) + 8, 9)])
def test_log_probabilities(rows, classes):
    _need(62)
    _say("logprob", rows, classes)
    x = _random(rows, classes, 4)
    targets = torch.randint(-1, classes, (rows,), device=DEV, dtype=torch.int32, generator=torch.Generator(device=DEV).manual_seed(2))
    logp, stats, d = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV), torch.empty_like(x)
    top, top_class = torch.empty(rows, 2, device=DEV), torch.empty(rows, 2, dtype=torch.int32, device=DEV)
    B.adaqp_logprob_forward(x, classes, targets, logp, None, stats, top, top_class, None)
    B.adaqp_logprob_backward(x, classes, targets, stats, None, None, None, 1.0, d)
    for a, b in _ends(rows, 600):
        lp, st, dd, tp, tc = (torch.empty_like(t[a:b]) for t in (logp, stats, d, top, top_class))
        B.adaqp_logprob_forward(x[a:b], classes, targets[a:b], lp, None, st, tp, tc, None)
        B.adaqp_logprob_backward(x[a:b], classes, targets[a:b], st, None, None, None, 1.0, dd)
        for got, want in ((logp, lp), (stats, st), (d, dd), (top, tp), (top_class, tc)):
            assert torch.equal(got[a:b], want)


def test_8_bit_matrices():
    """Rows of codes past 2^32 bytes, quantised both ways, read back and multiplied."""
    rows, cols, n = (1 << 24) + 133, 300, 40
    _need(45)
    _say("f8", rows, cols, n)
    x = _random(rows, cols, 5)
    p, t = B.f8_empty(rows, cols, DEV), B.f8_empty(cols, rows, DEV)
    w = B.f8_empty(n, cols, DEV)
    B.adaqp_f8_quantize(x, cols, B.F8_ROWS, p, t)
    B.adaqp_f8_quantize(_random(n, cols, 6), cols, B.F8_TILES, w, None)
    back, out = torch.empty_like(x), torch.empty(rows, n, device=DEV)
    B.adaqp_f8_dequantize(p, cols, back)
    B.adaqp_f8_matmul(p, w, cols, out, torch.empty(max(1, B.adaqp_f8_matmul_workspace_bytes(rows, n, cols)), dtype=torch.uint8, device=DEV))
    values = torch.empty(n, cols, device=DEV)
    B.adaqp_f8_dequantize(w, cols, values)
    for a, b in ((0, 1024), (rows // 2 // 128 * 128, rows // 2 // 128 * 128 + 1024), (rows - 1024 - 133 % 128, rows)):
        k = b - a
        q, qt = B.f8_empty(k, cols, DEV), B.f8_empty(cols, k, DEV)
        B.adaqp_f8_quantize(x[a:b], cols, B.F8_ROWS, q, qt)
        assert torch.equal(p[0][a:b], q[0]) and torch.equal(p[1][:, a:b], q[1][:, :k])
        assert a % 128 == 0 and torch.equal(t[0][:, a:a + qt[0].shape[1]], qt[0]) and torch.equal(t[1][a // 128:a // 128 + qt[1].shape[0]], qt[1])
        want = torch.empty_like(x[a:b])
        B.adaqp_f8_dequantize(q, cols, want)
        assert torch.equal(back[a:b], want)
        product = want.double() @ values.double().t()
        assert torch.all((out[a:b].double() - product).abs() <= 2 * 2.0 ** -24 * (cols / 64 + 16) * (want.double().abs() @ values.double().abs().t()))
