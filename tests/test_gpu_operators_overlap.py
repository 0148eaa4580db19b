"""Results of operators as payloads of calls that overlap (GLEAM_OVERLAP_CALLS), which read
their payload before they wait for the work before them: one buffer, written again and again
and uploaded after each time, must give what a cache without the flag gives."""
import pytest
import torch

from paper_2607_23115_gb300 import binding as B
from paper_2607_23115_gb300 import experts, fp8
from paper_2607_23115_gb300.cache import Cache, DedupOutputs

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TURNS = 24


def _uploads(write, like, chunk, flags, between=None):
    """Every call's result, mask and packed misses, and the cache's keys at the end."""
    n = like.numel() * like.element_size()
    buf = torch.zeros_like(like)
    outs = [DedupOutputs.alloc(n, chunk, DEV) for _ in range(TURNS)]
    res = torch.zeros(TURNS, B.RESULT_WORDS, dtype=torch.int64, device=DEV)
    with Cache(8 * n + 64 * chunk, chunk, flags) as cache:
        cache.reserve(-(-n // chunk))
        torch.cuda.synchronize()
        for i in range(TURNS):
            write(i, buf)
            if between is not None:
                between()
            cache.dedup_async(buf, outs[i], res[i])
        torch.cuda.synchronize()
        keys, lens, used = cache.export()
    got = []
    for r, o in zip(res.cpu().tolist(), outs):
        got.append((r, o.hit_mask.cpu(), o.miss_idx[:r[1]].cpu(), o.miss_bytes[:r[5]].cpu()))
    return got, sorted(keys.tolist()), used


def _same(write, like, chunk, between=None):
    a = _uploads(write, like, chunk, B.GLEAM_OVERLAP_CALLS, between)
    b = _uploads(write, like, chunk, 0, between)
    assert a[1:] == b[1:]
    for i, (x, y) in enumerate(zip(a[0], b[0])):
        assert x[0] == y[0] and x[0][0] == 0, (i, x[0], y[0])
        assert all(torch.equal(p, q) for p, q in zip(x[1:], y[1:])), i
    return b[0]


def _ok(rc):
    assert rc == 0, rc


def _variants(n, k, count=6):
    """Weights of which each changes a block of the one before."""
    torch.manual_seed(n + k)
    w = (0.02 * torch.randn(n, k, device=DEV)).to(torch.bfloat16)
    ws = [w]
    for i in range(1, count):
        w = w.clone()
        w[:128, 128 * i:128 * i + 128] *= 1.5
        ws.append(w)
    return ws


def _turn(i, count):
    return i % count if i < count else (7 * i) % count


@pytest.mark.parametrize("linear", [False, True])
@pytest.mark.parametrize("chunk", [16384, 65536])
@pytest.mark.parametrize("n,k", [(512, 896), (4096, 2048), (8192, 4096)])
def test_quantised_weights(n, k, chunk, linear):
    ws = _variants(n, k)
    like = fp8.quantize_weight(ws[0])
    stream, lib = torch.cuda.current_stream().cuda_stream, B.lib()

    def write(i, buf):
        w = ws[_turn(i, len(ws))]
        _ok(lib.gleam_fp8_quantize(fp8._matrix(w), B.GLEAM_FP8_BLOCKS, None, 0, n, buf.data_ptr(),
                                   like.s.data_ptr(), None, None, stream))

    x = torch.randn(200, k, device=DEV).to(torch.bfloat16)
    calls = _same(write, like.q, chunk, (lambda: fp8.linear(x, like)) if linear else None)
    assert [r[0][1] for r in calls[:3]] == [like.q.numel() // chunk, 1, 1]


# rows of x: one kernel; w's rows as the lanes; x's, by one block and by two
@pytest.mark.parametrize("m,n,k", [(3, 4096, 512), (40, 4096, 512), (300, 4096, 512), (4096, 4096, 512)])
def test_products(m, n, k):
    xs = [torch.randn(m, k, device=DEV).to(torch.bfloat16) for _ in range(5)]
    w = fp8.quantize_weight(0.02 * torch.randn(n, k, device=DEV))
    size = B.gleam_fp8_linear_work(m, k)
    work = torch.empty(size + 16, dtype=torch.uint8, device=DEV)

    def write(i, buf):
        x = xs[_turn(i, 5)]
        _ok(B.gleam_fp8_linear(B.gleam_fp8_linear_t(
            x.data_ptr(), B.GLEAM_BF16, 1, m, k, k, 0, n, w.q.data_ptr(), w.s.data_ptr(), buf.data_ptr(), n, m, None,
            0, 0, 0, 0, None, None, work.data_ptr(), size), torch.cuda.current_stream().cuda_stream))

    _same(write, torch.empty(m, n, dtype=torch.bfloat16, device=DEV), 16384)


@pytest.mark.parametrize("what", ["gather", "combine", "combine_grad", "sort"])
def test_rows_by_expert(what):
    t, per, cols, n = 3000, 2, 1024, 8
    rng = torch.Generator(device=DEV).manual_seed(1)
    ids = [torch.randint(0, n, (t, per), generator=rng, device=DEV, dtype=torch.int32) for _ in range(5)]
    plan = experts.sort(ids[0], n)
    x = [torch.randn(t, cols, generator=rng, device=DEV) for _ in range(5)]
    rows = [torch.randn(plan.rows, cols, generator=rng, device=DEV) for _ in range(5)]
    g = torch.rand(t, per, generator=rng, device=DEV)
    dg = torch.empty_like(g)
    other = experts.sort(ids[0], n)
    lib, stream = B.lib(), torch.cuda.current_stream().cuda_stream

    def write(i, buf):
        j = _turn(i, 5)
        if what == "gather":
            rc = lib.gleam_expert_gather(fp8._matrix(x[j]), plan.at_src_of, per, plan.rows, buf.data_ptr(), stream)
        elif what == "combine":
            rc = lib.gleam_expert_combine(fp8._matrix(rows[j]), plan.at_row_of, g.data_ptr(), t, per, buf.data_ptr(),
                                          stream)
        elif what == "combine_grad":
            rc = lib.gleam_expert_combine_grad(fp8._matrix(x[j]), fp8._matrix(rows[j]), plan.at_row_of, plan.at_src_of,
                                               g.data_ptr(), per, buf.data_ptr(), dg.data_ptr(), stream)
        else:
            rc = lib.gleam_expert_sort(ids[j].data_ptr(), 4, t, per, n, 128, other.at_offsets, other.at_counts,
                                       other.at_row_of, buf.data_ptr(), stream)
        _ok(rc)

    like = {"gather": rows[0], "combine_grad": rows[0], "combine": x[0], "sort": plan.src_of.clone()}[what]
    _same(write, like, 4096)
