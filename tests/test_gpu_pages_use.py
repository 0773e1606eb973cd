"""The paged cache as a program uses it: all its calls in a row beside the dense ones, in captured graphs whose lengths
change between replays, on other streams, with pools beyond 32-bit offsets and many sequences; and no result may depend on
the order in which workgroups run."""
import os
import random
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2505_19602_amd as skv
import pages_util as P
from parity_util import check_indices

pytestmark = pytest.mark.gpu
DEV, BF16, F32, E4M3 = "cuda", torch.bfloat16, torch.float32, P.E4M3
HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
REVERSED = os.path.join(ROOT, "paper_2505_19602_amd", "libscalekv_reversed_order.so")


def _workspace(shape, pages, new, **mask):
    return torch.full((skv.pages_workspace_bytes(shape, pages, new, **mask),), 255, dtype=torch.uint8, device=DEV)


def _check(cache, s, q, out, causal=False, window=0, sinks=0):
    want, tol = P.attend(cache, s, q, causal, window, sinks, cache.d ** -0.5)
    err = (out.cpu().double() - want).abs()
    assert torch.all(err <= tol), f"sequence {s}: {float((err / tol).max()):.3f} of the bound"


@pytest.mark.parametrize("cache_dtype", [BF16, E4M3])
@pytest.mark.parametrize("d", [64, 128])
def test_maps_of_growing_scales_through_a_quantised_cache(cache_dtype, d):
    """Two layers of one pool: each map is written and attends over the pages; then the layer's rows are read back, ranked by
    the map's last queries and pruned to the budget, and what is kept goes back into the layer's pages."""
    S, H, page, dtype = 2, 4, 16, BF16
    shape, gen = skv.Shape(S, H, d, dtype), torch.Generator().manual_seed(d)
    budgets, sides, width = (40, 12), (2, 4, 7, 9), 16
    n_page = 2 * S * width
    pool = [torch.zeros(n_page, H, page, d, device=DEV).to(cache_dtype) for _ in range(2)]
    scales = [None, None] if cache_dtype == BF16 else [torch.full((n_page, H, page), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
    order = torch.randperm(n_page, generator=gen).int().reshape(2, S, width)
    lens = [torch.zeros(S, dtype=torch.int32, device=DEV) for _ in range(2)]
    layers = [skv.Pages(pool[0], pool[1], order[x].to(DEV), lens[x], *scales) for x in range(2)]
    held = [[torch.zeros(S, H, 0, d).double() for _ in range(2)] for _ in range(2)]      # what each layer's pages stand for
    dense = torch.zeros(2, S, H, width * page, d, dtype=dtype, device=DEV)
    kept_rows = torch.zeros_like(dense)
    cached = [0, 0]
    for side in sides:
        n = side * side
        for layer, pages in enumerate(layers):
            q, k, v = ((torch.randn(S, H, n, d, generator=gen) * 1.5).to(dtype) for _ in range(3))
            total = cached[layer] + n
            pages.lens.fill_(total)
            skv.pages_write(shape, pages, k.to(DEV), v.to(DEV))
            out = torch.full((S, H, n, d), 7.0, dtype=dtype, device=DEV)
            skv.pages_attend(shape, pages, q.to(DEV), out, _workspace(shape, pages, n))
            skv.pages_read(shape, pages, None, total, dense[0], dense[1])
            win = min(16, n)
            ws = torch.zeros(skv.workspace_bytes(shape, total, n), dtype=torch.uint8, device=DEV)
            scores = torch.zeros(S, H, total, device=DEV)
            skv.score(shape, q[:, :, n - win:].contiguous().to(DEV), dense[0], total, scores, ws)
            keep = min(budgets[layer], total)
            idx = torch.full((S, H, keep), -1, dtype=torch.int32, device=DEV)
            skv.select(shape, scores, total, keep, idx)
            skv.pages_read(shape, pages, idx, keep, kept_rows[0], kept_rows[1])
            pages.lens.fill_(keep)
            skv.pages_write(shape, pages, kept_rows[0, :, :, :keep], kept_rows[1, :, :, :keep])
            torch.cuda.synchronize()
            # the same in 64 bits: the pages hold what was kept before and the rounded new rows
            view = P.Cache(0, [total] * S, H, d, page, dtype, dtype)
            for i, x in enumerate((k, v)):
                if cache_dtype == E4M3:
                    codes, scale = P.quantised_tensor(x)
                    x = codes.float().double() * torch.ldexp(torch.ones(()).double(), scale.int() - 127).unsqueeze(-1)
                held[layer][i] = torch.cat([held[layer][i], x.double()], 2)
                assert torch.equal(dense[i, :, :, :total].cpu().double(), held[layer][i])
            view.rows = lambda name, s: held[layer]["kv".index(name)][s]
            for s in range(S):
                _check(view, s, q[s], out[s])
            units = lambda t: t.reshape(S * H, *t.shape[2:])
            logits = units(q[:, :, n - win:].double()) @ units(held[layer][0]).transpose(1, 2) * d ** -0.5
            log_scores = torch.logsumexp(torch.log_softmax(logits, -1), 1).numpy()
            picked = units(idx).cpu().numpy()
            for u in range(S * H):
                check_indices(picked[u], log_scores[u], keep, np.sort(np.argsort(-log_scores[u], kind="stable")[:keep]))
            # what is kept is exact already: writing it again changes nothing
            at = idx.long().cpu().unsqueeze(-1).expand(-1, -1, -1, d)
            held[layer] = [x.gather(2, at) for x in held[layer]]
            cached[layer] = keep
    for layer, pages in enumerate(layers):
        skv.pages_read(shape, pages, None, cached[layer], dense[0], dense[1])
        for i in range(2):
            assert torch.equal(dense[i, :, :, :cached[layer]].cpu().double(), held[layer][i])


@pytest.mark.parametrize("cache_dtype", [BF16, E4M3])
def test_tokens_in_a_graph_whose_lengths_change_between_replays(cache_dtype):
    """A decoding step (write, attend) captured once: lengths, tables and tokens change in device memory, and two graphs run
    in turn with eager work between them; every replay is what the eager calls give, bit for bit."""
    S, H, kv, d, page, dtype, width = 5, 8, 2, 128, 32, BF16, 40
    shape = skv.Shape(S, H, d, dtype)
    cache = P.Cache(3, [width * page] * S, kv, d, page, cache_dtype, dtype)
    pages, gen = cache.on(DEV), torch.Generator(device=DEV).manual_seed(1)
    q, k, v = (torch.zeros(S, h, 1, d, dtype=dtype, device=DEV) for h in (H, kv, kv))
    graphs = []
    side = torch.cuda.Stream()
    for mask in (dict(causal=True), dict(causal=True, window=100, n_sink=4)):
        out, ws = torch.zeros_like(q), _workspace(shape, pages, 1, **mask)
        pages.lens.fill_(50)
        with torch.cuda.stream(side):
            skv.pages_write(shape, pages, k, v)
            skv.pages_attend(shape, pages, q, out, ws, **mask)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            skv.pages_write(shape, pages, k, v)
            skv.pages_attend(shape, pages, q, out, ws, **mask)
        graphs.append((graph, out, mask))
    rng = random.Random(4)
    for step in range(6):
        lens = [rng.choice((1, 33, 640, 1279, rng.randint(1, width * page))) for _ in range(S)]
        for i in range(S):
            pages.lens[i] = lens[i]
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device=DEV, generator=gen))
        got = []
        for graph, out, mask in graphs:
            graph.replay()
            torch.cuda.synchronize()
            got.append(out.clone())
            eager = torch.zeros_like(q)
            skv.pages_attend(shape, pages, q, eager, _workspace(shape, pages, 1, **mask), **mask)
            assert torch.equal(eager, got[-1]), (step, mask)
        for name in ("k", "v"):
            cache.pool[name] = getattr(pages, name).cpu()
            if cache_dtype == E4M3:
                cache.scales[name] = getattr(pages, name + "_scale").cpu()
        cache.lens = lens
        for s in range(S):
            _check(cache, s, q[s].cpu(), got[0][s], causal=True)
            _check(cache, s, q[s].cpu(), got[1][s], causal=True, window=100, sinks=4)


@pytest.mark.parametrize("new,d", [(1, 64), (1, 128), (20, 128), (70, 64)])
def test_many_sequences_of_any_length(new, d):
    """More sequences than a wave has lanes, some of them empty, some without new tokens, one far longer than the rest."""
    rng, dtype, page, heads, kv = random.Random(new), BF16, 16, 3, 3
    S = 150
    counts = [rng.choice((0, 1, new, rng.randint(0, new))) for _ in range(S)]
    lens = [n + rng.choice((0, 0, 5, rng.randint(0, 200))) for n in counts]
    lens[77] = counts[77] + 4000
    cache = P.Cache(1, lens, kv, d, page, E4M3, dtype)
    shape, pages = skv.Shape(S, heads, d, dtype), cache.on(DEV)
    total = sum(counts)
    first = [sum(counts[:s]) for s in range(S)]
    q = torch.randn(total + 3, heads, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 7.0, device=DEV)
    skv.pages_attend(shape, pages, q.to(DEV), out, _workspace(shape, pages, new, causal=True), causal=True, first=ints(first),
                     count=ints(counts), max_new=new)
    torch.cuda.synchronize()
    for s in range(S):
        at = slice(first[s], first[s] + counts[s])
        _check(cache, s, q[at].transpose(0, 1), out[at].transpose(0, 1), causal=True)
    assert torch.all(out[total:] == 7.0)


def test_pools_beyond_32_bit_offsets():
    """Pages behind 2^31 elements of a pool in 8 bits (2.2 GB), reached by writing, reading and attending."""
    d, heads, page, dtype = 128, 4, 64, BF16
    n_page = (1 << 31) // (heads * page * d) + 40
    pool = [torch.zeros(n_page, heads, page, d, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)]
    scales = [torch.full((n_page, heads, page), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
    ids = [n_page - 1, 3, n_page - 7]
    pages = skv.Pages(*pool, torch.tensor([ids], dtype=torch.int32, device=DEV), torch.tensor([150], dtype=torch.int32, device=DEV),
                      *scales)
    shape = skv.Shape(1, heads, d, dtype)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(1, heads, 150, d, generator=g).to(dtype) for _ in range(3))
    skv.pages_write(shape, pages, k.to(DEV), v.to(DEV))
    out = torch.zeros(1, heads, 150, d, dtype=dtype, device=DEV)
    skv.pages_attend(shape, pages, q.to(DEV), out, _workspace(shape, pages, 150, causal=True), causal=True)
    one = torch.zeros(1, heads, 1, d, dtype=dtype, device=DEV)
    skv.pages_attend(shape, pages, q[:, :, -1:].to(DEV), one, _workspace(shape, pages, 1, causal=True), causal=True)
    back = torch.zeros(2, 1, heads, 150, d, dtype=dtype, device=DEV)
    skv.pages_read(shape, pages, None, 150, back[0], back[1])
    torch.cuda.synchronize()
    cache = P.Cache(0, [150], heads, d, page, dtype, dtype)
    rows = []
    for x, b in ((k, back[0]), (v, back[1])):
        codes, scale = P.quantised_tensor(x)
        rows.append((codes.float().double() * torch.ldexp(torch.ones(()).double(), scale.int() - 127).unsqueeze(-1))[0])
        assert torch.equal(b[0].cpu().double(), rows[-1])
    cache.rows = lambda name, s: rows["kv".index(name)]
    _check(cache, 0, q[0], out[0], causal=True)
    _check(cache, 0, q[0, :, -1:], one[0], causal=True)
    used = torch.zeros(n_page, dtype=torch.bool, device=DEV)
    used[ids] = True
    for t in scales:
        assert torch.all(t[~used] == 127)


def test_two_streams_at_once_and_twice_the_same():
    """Calls on two streams with a workspace each; results do not change from run to run."""
    S, H, d, page, dtype = 3, 4, 128, 64, BF16
    shape = skv.Shape(S, H, d, dtype)
    cache = P.Cache(5, [7000, 300, 2000], H, d, page, BF16, dtype)
    pages = cache.on(DEV)
    q = torch.randn(S, H, 1, d, generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    spaces = [_workspace(shape, pages, 1, causal=True) for _ in range(2)]
    assert spaces[0].numel() > 0
    torch.cuda.synchronize()
    for turn in range(4):
        for stream, ws in zip(streams, spaces):
            with torch.cuda.stream(stream):
                out = torch.zeros_like(q)
                skv.pages_attend(shape, pages, q, out, ws, causal=True)
                outs.append(out)
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])
    for s in range(S):
        _check(cache, s, q[s].cpu(), outs[0][s], causal=True)


def test_the_binding_refuses_what_does_not_fit_and_says_so():
    """The calls that native code does not take come to checks that name the argument."""
    S, H, d, page, dtype = 2, 4, 64, 16, BF16
    shape, pages = skv.Shape(S, H, d, dtype), P.Cache(1, [20, 30], 2, d, page, E4M3, dtype).on(DEV)
    q, k = (torch.zeros(S, h, 3, d, dtype=dtype, device=DEV) for h in (H, 2))
    ws, ints = _workspace(shape, pages, 3), lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    dst = torch.zeros(S, H, 8, d, dtype=dtype, device=DEV)
    packed = q[0].transpose(0, 1).contiguous()
    for call, word in (
            (lambda: skv.pages_write(shape, pages, q, q), "k_new has shape"), (lambda: skv.pages_write(shape, pages, k.float(), k), "dtype"),
            (lambda: skv.pages_write(shape, pages, k.cpu(), k), "current device"),
            (lambda: skv.pages_write(shape, pages, k[..., ::2], k), "k_new has shape"),
            (lambda: skv.pages_write(shape, pages, k, k, count=ints(1)), "count"),
            (lambda: skv.pages_write(shape, pages, k, k, count=ints(1, 2).long()), "count"),
            (lambda: skv.pages_write(shape, pages, k, k, max_new=4), "n_row"),
            (lambda: skv.pages_write(skv.Shape(3, H, d, dtype), pages, k, k), "pages for"),
            (lambda: skv.pages_read(shape, pages, ints(1), 1, dst, dst.clone()), "idx"),
            (lambda: skv.pages_read(shape, pages, None, 9, dst, dst.clone()), "capacity"),
            (lambda: skv.pages_attend(shape, pages, packed, packed.clone(), ws), "max_new is needed"),
            (lambda: skv.pages_attend(shape, pages, packed, packed.clone(), ws, max_new=3), "first is needed"),
            (lambda: skv.pages_attend(shape, pages, q, packed, ws), "packed or not"),
            (lambda: skv.pages_attend(shape, pages, q, q.transpose(2, 3).contiguous().transpose(2, 3), ws), "rows must be contiguous"),
            (lambda: skv.pages_attend(shape, pages, q, q[:, :1].expand(-1, H, -1, -1), ws), "coincide"),
            (lambda: skv.Pages(pages.k, pages.v, pages.table, pages.lens), "k_scale"),
            (lambda: skv.Pages(pages.k, pages.v.transpose(0, 1).contiguous().transpose(0, 1), pages.table, pages.lens,
                               pages.k_scale, pages.v_scale), "strides"),
            (lambda: skv.Pages(pages.k, pages.v, pages.table.long(), pages.lens, pages.k_scale, pages.v_scale), "table")):
        with pytest.raises(skv.ScaleKVError, match=word):
            call()
    with pytest.raises(AttributeError):
        pages.lens = ints(1, 2)
    skv.pages_check(shape, pages, pages.table.tolist(), [20, 30], max_new=3, n_row=3)
    with pytest.raises(skv.ScaleKVError, match="len"):
        skv.pages_check(shape, pages, pages.table.tolist(), [20, 33], max_new=3, n_row=3)
    # nothing new at all, and a page table of one sequence
    none = torch.zeros(0, H, d, dtype=dtype, device=DEV)
    skv.pages_attend(shape, pages, none, none.clone(), ws, first=ints(0, 0), count=ints(0, 0), max_new=3)
    torch.cuda.synchronize()


def _run_all():
    """Every kind of call on fixed inputs: {name: bytes}."""
    got = {"library": os.path.basename(skv.lib_path())}
    keep = lambda name, t: got.__setitem__(name, t.contiguous().view(torch.uint8).cpu().numpy().copy())
    for n, (S, H, kv, d, dtype, cache_dtype, page, most, new, mask) in enumerate((
            (4, 8, 2, 128, BF16, BF16, 16, 5000, 1, dict(causal=True)),
            (4, 8, 2, 64, BF16, E4M3, 32, 5000, 1, dict(causal=True)),
            (3, 10, 10, 128, BF16, E4M3, 64, 900, 6, dict(causal=True, window=300, n_sink=5)),
            (2, 4, 1, 128, BF16, BF16, 128, 6000, 40, dict(causal=True)),
            (2, 3, 3, 64, BF16, E4M3, 16, 700, 300, dict()),
            (2, 16, 16, 128, BF16, BF16, 64, 4000, 130, dict(causal=True)),
            (2, 2, 2, 128, F32, F32, 16, 3000, 3, dict(causal=True)),
            (2, 2, 2, 64, F32, E4M3, 16, 300, 70, dict(causal=True, window=64)),
            (130, 2, 2, 64, BF16, E4M3, 16, 1300, 70, dict(causal=True)),
            (130, 2, 2, 128, BF16, BF16, 64, 1300, 150, dict()),
            (130, 2, 2, 64, F32, F32, 16, 1300, 80, dict(causal=True)))):
        print(f"workgroup order: pages {S}x{H}/{kv} d {d} {dtype} {cache_dtype} rows {most} new {new} {mask}", flush=True)
        lens, counts = P.lengths(random.Random(n), S, most, new, True)
        pages = P.Cache(n, lens, kv, d, page, cache_dtype, dtype).on(DEV)
        shape, g = skv.Shape(S, H, d, dtype), torch.Generator().manual_seed(n)
        count = torch.tensor(counts, dtype=torch.int32, device=DEV)
        q, k, v = (torch.randn(S, h, new, d, generator=g).to(dtype).to(DEV) for h in (H, kv, kv))
        skv.pages_write(shape, pages, k, v, count=count)
        out = torch.zeros_like(q)
        skv.pages_attend(shape, pages, q, out, _workspace(shape, pages, new, **mask), count=count, **mask)
        back = torch.zeros(2, S, H, 60, d, dtype=dtype, device=DEV)
        idx = torch.randint(0, most, (S, H, 60), generator=g, dtype=torch.int32).to(DEV)
        skv.pages_read(shape, pages, idx, 60, back[0], back[1])
        skv.pages_read(shape, pages, None, 50, back[0], back[1])
        torch.cuda.synchronize()
        for name, t in (("k", pages.k), ("v", pages.v), ("out", out), ("back", back)):
            keep(f"{n}_{name}", t)
    return got


@pytest.mark.skipif(not os.path.exists(REVERSED),
                    reason="build it with: python -m paper_2505_19602_amd.build --variant reversed_order")
def test_results_do_not_depend_on_the_order_of_workgroups(tmp_path):
    plain, path = _run_all(), str(tmp_path / "reversed.npz")
    env = dict(os.environ, SCALEKV_LIBRARY=REVERSED, PYTHONPATH=os.pathsep.join([ROOT, HERE, os.environ.get("PYTHONPATH", "")]))
    res = subprocess.run([sys.executable, "-u", os.path.abspath(__file__), path], env=env, cwd=ROOT, capture_output=True,
                         text=True, timeout=300)
    assert res.returncode == 0, f"worker failed:\n{res.stdout[-2000:]}\n{res.stderr[-4000:]}"
    rev = np.load(path)
    assert sorted(rev.files) == sorted(plain)
    assert plain.pop("library") == "libscalekv.so" and str(rev["library"]) == os.path.basename(REVERSED)
    for name in sorted(plain):
        assert np.array_equal(plain[name], rev[name]), f"{name} differs between the plain and the reversed build"


if __name__ == "__main__":
    np.savez(sys.argv[1], **_run_all())
