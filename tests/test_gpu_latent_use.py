"""Latent caches as they are used: several calls together, captured and replayed, on other streams, with rows that lie apart, many
sequences, pages far into the pool, and prompts of many lengths."""
import numpy as np
import pytest
import torch

import oracle.latent as ol
import paper_2403_11805_amd as kvs

from latent import Latent, attend, check_attend, put, rows

pytestmark = pytest.mark.gpu

MIXED = (16, 8, 4, 2)


def space(p, max_rows=1, n_tokens=None):
    n = len(p.len)
    need = kvs.kv_latent_prompts_workspace_bytes(p.ks, n, n_tokens) if n_tokens else kvs.kv_latent_attend_workspace_bytes(p.ks, n, max_rows)
    return torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_a_prompt_and_steps_behind_it():
    """A prompt is appended and attends in the expanded form, a token follows and attends in the absorbed form, a page is brought to
    another width through read and append: what the cache holds and what comes out are the oracle's all along."""
    p = Latent((2, 3, 512, 64, 128, 64, 128, 16, 64), [70, 33], MIXED, 31)
    w = p.weights()
    counts = [50, 33]
    start, n = rows(counts)
    pages, pool = p.device()
    for layer in range(2):
        c, r = p.halves(n, 512), p.halves(n, 64)
        kvs.kv_latent_append_tokens(pages, layer, put(c), put(r), put(start))
        ol.append(p.os, p.pool, *p.table(), layer, c, r, start)
    assert np.array_equal(pool.cpu().numpy(), p.pool)
    check_attend(p, 1, p.queries(n), w, start, expanded=True)
    p.len += 1
    pages.length.add_(1)
    for layer in range(2):
        c, r = p.halves(2, 512), p.halves(2, 64)
        kvs.kv_latent_append_tokens(pages, layer, put(c), put(r))
        ol.append(p.os, p.pool, *p.table(), layer, c, r, None)
    assert np.array_equal(pool.cpu().numpy(), p.pool)
    q = p.queries(2)
    one, many = check_attend(p, 1, q, w), check_attend(p, 1, q, w, expanded=True)
    assert np.abs(one.astype(float) - many).max() < 0.05
    # the second page of the first sequence goes to a fresh record of 8 bits at the pool's end
    room = ol.record_bytes(p.os, 8)
    grown = np.concatenate([p.pool, np.full(-p.pool.size % 16 + room, 0xff, dtype=np.uint8)])
    at = grown.size - room
    big = put(grown)
    one_page = (np.array([[p.off[0, 1]], [at]]), np.array([[p.bits[0, 1]], [8]], dtype=np.uint8))
    shape = p.ks._replace(n_tokens=16)
    old = kvs.LatentPages(shape, big, put(one_page[0][:1]), put(one_page[1][:1]), put(np.array([16], dtype=np.int32)))
    new = kvs.LatentPages(shape, big, put(one_page[0][1:]), put(one_page[1][1:]), put(np.array([16], dtype=np.int32)))
    moved, _ = rows([16])
    for layer in range(2):
        c, r = torch.empty((16, 512), dtype=torch.float16, device="cuda"), torch.empty((16, 64), dtype=torch.float16, device="cuda")
        kvs.kv_latent_read_tokens(old, layer, c, r, put(moved))
        kvs.kv_latent_append_tokens(new, layer, c, r, put(moved))
    torch.cuda.synchronize()
    p.pool = big.cpu().numpy()
    p.off[0, 1], p.bits[0, 1] = at, 8
    check_attend(p, 1, q, w)
    check_attend(p, 0, q, w, expanded=True)


@pytest.mark.parametrize("expanded", [False, True])
def test_steps_captured_and_replayed(expanded):
    """Append, read and attention as one graph on a stream of its own, replayed with other lengths, rows and weights, eager work
    between the replays: every replay equals the same calls made eagerly."""
    p = Latent((2, 4, 512, 64, 128, 128, 160, 32, 64), [100, 41, 160], MIXED, 21)
    pages, pool = p.device()
    c, r, q, w = (put(a) for a in (p.halves(3, 512), p.halves(3, 64), p.queries(3), p.weights()))
    back = torch.zeros((2, 3, 512), dtype=torch.float16, device="cuda"), torch.zeros((2, 3, 64), dtype=torch.float16, device="cuda")
    out = torch.zeros((2, 3, 4, 128), dtype=torch.float16, device="cuda")
    ws = space(p, n_tokens=400 if expanded else None)

    def step():
        for layer in range(2):
            kvs.kv_latent_append_tokens(pages, layer, c, r)
            kvs.kv_latent_read_tokens(pages, layer, back[0][layer], back[1][layer])
            if expanded:
                kvs.kv_latent_attend_prompts(pages, layer, q, w, ws, out[layer], 400)
            else:
                kvs.kv_latent_attend_tokens(pages, layer, q, w, ws, out[layer])

    state = [pool, *back, out]
    before = [t.clone() for t in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([100, 41, 160], [101, 1, 33], [128, 0, 159], [100, 41, 160]):
        pages.length.copy_(torch.tensor(lens, dtype=torch.int32))
        for t in (c, r, q):
            t.normal_()
        for t, b in zip(state, before):
            t.copy_(b)
        step()
        torch.cuda.synchronize()
        eager = [t.clone() for t in state]
        for t, b in zip(state, before):
            t.copy_(b)
        ws.fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip(state, eager):
            assert same(t, e)


def test_graphs_share_a_workspace():
    """Captured calls over two layers, absorbed and expanded, with one workspace, replayed in turn."""
    p = Latent((2, 8, 256, 32, 64, 64, 512, 16, 64), [512, 300], MIXED, 23)
    pages, _ = p.device()
    q, w = put(p.queries(2)), put(p.weights())
    ws = torch.empty(max(kvs.kv_latent_attend_workspace_bytes(p.ks, 2), kvs.kv_latent_prompts_workspace_bytes(p.ks, 2, 900)), dtype=torch.uint8,
                     device="cuda")
    out = torch.zeros((4, 2, 8, 64), dtype=torch.float16, device="cuda")

    def call(i):
        if i < 2:
            kvs.kv_latent_attend_tokens(pages, i, q, w, ws, out[i])
        else:
            kvs.kv_latent_attend_prompts(pages, i - 2, q, w, ws, out[i], 900)

    want = []
    for i in range(4):
        call(i)
        want.append(out[i].clone())
    graphs = [torch.cuda.CUDAGraph() for _ in range(4)]
    for i, graph in enumerate(graphs):
        with torch.cuda.graph(graph):
            call(i)
    for turn in range(3):
        for i, graph in enumerate(graphs):
            ws.fill_(0xff if turn % 2 else 0x3c)
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[i], want[i])


@pytest.mark.parametrize("expanded", [False, True])
def test_two_calls_at_once_on_streams_of_their_own(expanded):
    p = Latent((2, 8, 512, 64, 128, 128, 1024, 16, 64), [1000, 777, 64], MIXED, 25)
    pages, _ = p.device()
    q, w = put(p.queries(3)), put(p.weights())
    out = torch.zeros((2, 3, 8, 128), dtype=torch.float16, device="cuda")
    spaces = [space(p, n_tokens=2000 if expanded else None) for _ in range(2)]

    def call(layer, stream=None):
        if expanded:
            kvs.kv_latent_attend_prompts(pages, layer, q, w, spaces[layer], out[layer], 2000, stream=stream)
        else:
            kvs.kv_latent_attend_tokens(pages, layer, q, w, spaces[layer], out[layer], stream=stream)

    for layer in range(2):
        call(layer)
    torch.cuda.synchronize()
    want = out.clone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        for layer, s in enumerate(streams):
            call(layer, s)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_rows_that_lie_apart():
    """Latents, position parts and queries as slices of wider tensors, as a projection leaves them."""
    p = Latent((1, 4, 256, 64, 64, 128, 64, 16, 64), [40, 64], MIXED, 27)
    start, n = rows([3, 2])
    both, wide = p.halves(n, 256 + 64 + 32), p.halves(n, 1024)
    c, r = both[:, :256], both[:, 256:320]
    q = wide[:, 64:64 + 4 * 128].reshape(n, 4, 128)
    d_both, d_wide = put(both), put(wide)
    pages, pool = p.device()
    kvs.kv_latent_append_tokens(pages, 0, d_both[:, :256], d_both[:, 256:320], put(start))
    ol.append(p.os, p.pool, *p.table(), 0, c, r, start)
    assert np.array_equal(pool.cpu().numpy(), p.pool)
    back = torch.full((n, 512), 7.0, dtype=torch.float16, device="cuda")
    kvs.kv_latent_read_tokens(pages, 0, back[:, 8:264], back[:, 304:368], put(start))
    c_want, r_want = np.full_like(c, 7.0), np.full_like(r, 7.0)
    ol.read(p.os, p.pool, *p.table(), 0, c_want, r_want, start)
    got = back.cpu().numpy()
    assert np.array_equal(got[:, 8:264], c_want) and np.array_equal(got[:, 304:368], r_want)
    assert np.all(got[:, :8] == 7) and np.all(got[:, 264:304] == 7) and np.all(got[:, 368:] == 7)
    w = put(p.weights())
    outs = []
    for queries in (put(q), d_wide[:, 64:64 + 512].unflatten(1, (4, 128))):
        for expanded in (False, True):
            out = torch.zeros((n, 4, 128), dtype=torch.float16, device="cuda")
            if expanded:
                kvs.kv_latent_attend_prompts(pages, 0, queries, w, space(p, n_tokens=200), out, 200, row_start=put(start))
            else:
                kvs.kv_latent_attend_tokens(pages, 0, queries, w, space(p, 3), out, row_start=put(start), max_rows=3)
            outs.append(out)
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


@pytest.mark.parametrize("expanded", [False, True])
@pytest.mark.parametrize("n_seqs", [63, 64, 65, 300, 4500])
def test_many_sequences(n_seqs, expanded):
    """Lists longer than a wavefront is wide, and than 64 of its widths; some sequences without tokens, some without new rows."""
    rng = np.random.RandomState(n_seqs)
    lens = rng.randint(0, 33, n_seqs)
    p = Latent((1, 2, 256, 32, 64, 64, 32, 16, 256), lens, MIXED + (0,), 33)
    start, n = rows(rng.randint(0, 3, n_seqs), lead=1)
    check_attend(p, 0, p.queries(n + 2), p.weights(), start, 2, expanded)
    c, r = p.halves(n + 2, 256), p.halves(n + 2, 32)
    pages, pool = p.device()
    kvs.kv_latent_append_tokens(pages, 0, put(c), put(r), put(start))
    ol.append(p.os, p.pool, *p.table(), 0, c, r, start)
    assert np.array_equal(pool.cpu().numpy(), p.pool)


def test_more_new_rows_than_max_rows_are_left():
    """Rows past a sequence's first max_rows keep what the output holds, and the others are as if max_rows had been larger."""
    p = Latent((1, 3, 256, 32, 64, 64, 64, 16, 64), [50, 64, 20], MIXED, 35)
    start, n = rows([5, 2, 9])
    q, w = p.queries(n), p.weights()
    whole, some = attend(p, 0, q, w, start, 9), attend(p, 0, q, w, start, 4)
    _, *_ = want = ol.attend(p.os, p.pool, *p.table(), 0, q, w, start, 4)
    left = np.isnan(want[0])
    assert left.any() and np.all(some[left] == 7)
    check_attend(p, 0, q, w, start, 4)
    assert np.abs(whole.astype(float) - some)[~left].max() < 0.02


@pytest.mark.parametrize("expanded", [False, True])
@pytest.mark.parametrize("n", [1, 15, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 191, 193, 255, 257])
def test_lengths_around_the_tiles(n, expanded):
    """A prompt of n tokens in the expanded form, the last of n tokens in the absorbed one, beside a neighbour whose rows follow."""
    p = Latent((1, 3, 512, 32, 128, 64, 272, 16, 128), [n, 40], (16, 4), 37)
    start, rows_n = rows([n if expanded else 1, 1])
    check_attend(p, 0, p.queries(rows_n), p.weights(), start, 1, expanded)


@pytest.mark.parametrize("heads,dims", [(1, (64, 64)), (1, (128, 64)), (3, (64, 64)), (5, (128, 128)), (8, (64, 128)), (16, (64, 64)), (24, (128, 64)),
                                        (40, (64, 128))])
def test_prompts_of_any_number_of_heads(heads, dims):
    """Products of 128 to 7680 columns, whole tiles of 256 of them or not, and heads that are dealt out by eights or not."""
    p = Latent((1, heads, 256, 32, *dims, 208, 16, 64), [200, 70], MIXED, 39)
    start, n = rows([5, 70])
    check_attend(p, 0, p.queries(n), p.weights(), start, expanded=True)


@pytest.mark.parametrize("heads", [15, 16, 17, 31, 33, 63, 65, 127, 129, 160, 191, 193, 257, 321])
def test_tiles_of_query_rows(heads):
    """Numbers of query rows around every size of a tile, one row a head, and as many again for a second sequence's two rows."""
    p = Latent((1, heads, 256, 32, 64, 64, 96, 16, 64), [90, 75], (16, 4), 49)
    check_attend(p, 0, p.queries(2), p.weights())
    start, n = rows([1, 2])
    check_attend(p, 0, p.queries(n), p.weights(), start, 2)


@pytest.mark.parametrize("expanded", [False, True])
def test_the_most_heads_and_rows(expanded):
    """1024 heads and 16 new rows of one sequence: 16384 query rows on one latent a token."""
    p = Latent((1, 1024, 256, 32, 64, 64, 48, 16, 64), [37, 20], (16, 8), 45)
    start, n = rows([16, 1])
    check_attend(p, 0, p.queries(n), p.weights(), start, 16, expanded)


@pytest.mark.parametrize("expanded", [False, True])
def test_lists_of_rows_that_do_not_ascend_reach_no_other_memory(expanded):
    """A list out of order, below zero and past n_rows: what comes out is not said, but pool and the room around the output stay as they are."""
    p = Latent((1, 4, 256, 32, 64, 64, 64, 16, 64), [50, 64, 20, 33], MIXED, 47)
    n = 6
    q, w = put(p.queries(n)), put(p.weights())
    for wild in ([6, 4, 5, 0, 6], [0, 1 << 30, -5, 3, 2], [-(1 << 31), (1 << 31) - 1, 0, (1 << 31) - 1, 0], [5, 5, 5, 5, 5]):
        start = put(np.array(wild, dtype=np.int32))
        pages, pool = p.device()
        room = torch.full((n + 64, 4, 64), 7.0, dtype=torch.float16, device="cuda")
        out = room[32:32 + n]
        if expanded:
            kvs.kv_latent_attend_prompts(pages, 0, q, w, space(p, n_tokens=300), out, 300, row_start=start)
        else:
            kvs.kv_latent_attend_tokens(pages, 0, q, w, space(p, 4), out, row_start=start, max_rows=4)
        c, r = torch.full((n, 256), 3.0, dtype=torch.float16, device="cuda"), torch.full((n, 32), 3.0, dtype=torch.float16, device="cuda")
        kvs.kv_latent_read_tokens(pages, 0, c, r, start)
        torch.cuda.synchronize()
        assert np.array_equal(pool.cpu().numpy(), p.pool)
        assert torch.all(room[:32] == 7) and torch.all(room[32 + n:] == 7)


@pytest.mark.parametrize("room", [70, 129, 500, 5000])
def test_room_for_more_tokens_than_there_are(room):
    """What is made of the tokens does not depend on the room for others."""
    p = Latent((1, 4, 512, 64, 128, 128, 64, 16, 64), [30, 33], MIXED, 41)
    start, n = rows([30, 4])
    q, w = p.queries(n), p.weights()
    few = attend(p, 0, q, w, start, expanded=True, n_tokens=63)
    assert np.abs(few.astype(float) - attend(p, 0, q, w, start, expanded=True, n_tokens=room)).max() < 0.02
    check_attend(p, 0, q, w, start, expanded=True)


@pytest.mark.parametrize("width", [16, 8])
def test_pages_past_four_gigabytes(width):
    """Records on either side of the 32-bit line of a pool of 4.5 GiB."""
    p = Latent((2, 2, 512, 64, 64, 64, 128, 64, 64), [128, 100], (width,), 43)
    size = ol.record_bytes(p.os, width)
    far = (1 << 32) - size // 2 // 16 * 16
    places = [far - size, far, far + size, (9 << 29) - size]                 # the second one across the line
    pool = torch.zeros(9 << 29, dtype=torch.uint8, device="cuda")
    off = np.array(places, dtype=np.int64).reshape(2, 2)
    for i in range(2):
        for j in range(2):
            at = p.off[i, j]
            pool[off[i, j]:off[i, j] + size] = put(p.pool[at:at + size])
    pages = kvs.LatentPages(p.ks, pool, put(off), put(p.bits), put(p.len))
    start, n = rows([40, 3])
    c, r = p.halves(n, 512), p.halves(n, 64)
    kvs.kv_latent_append_tokens(pages, 1, put(c), put(r), put(start))
    ol.append(p.os, p.pool, *p.table(), 1, c, r, start)
    for i in range(2):
        for j in range(2):
            at = p.off[i, j]
            assert np.array_equal(pool[off[i, j]:off[i, j] + size].cpu().numpy(), p.pool[at:at + size])
    c_got, r_got = torch.zeros((n, 512), dtype=torch.float16, device="cuda"), torch.zeros((n, 64), dtype=torch.float16, device="cuda")
    kvs.kv_latent_read_tokens(pages, 1, c_got, r_got, put(start))
    c_want, r_want = np.zeros_like(c), np.zeros_like(r)
    ol.read(p.os, p.pool, *p.table(), 1, c_want, r_want, start)
    assert np.array_equal(c_got.cpu().numpy(), c_want) and np.array_equal(r_got.cpu().numpy(), r_want)
    q, w = p.queries(2), p.weights()
    near, _ = p.device()
    for expanded in (False, True):
        outs = []
        for held in (pages, near):
            out = torch.zeros((2, 2, 64), dtype=torch.float16, device="cuda")
            if expanded:
                kvs.kv_latent_attend_prompts(held, 1, put(q), put(w), space(p, n_tokens=300), out, 300)
            else:
                kvs.kv_latent_attend_tokens(held, 1, put(q), put(w), space(p), out)
            outs.append(out)
        assert torch.equal(*outs)


def test_append_then_read_of_many_rows():
    """Enough rows that a wavefront has several, in pages of 16 and of 1024 rows, with absent pages between."""
    for T, seed in ((16, 1), (1024, 2)):
        p = Latent((1, 1, 512, 32, 64, 64, 8192, T, 128), [8192, 1111], MIXED + (0,), seed)
        start, n = rows([8190, 1111], lead=1)
        c, r = p.halves(n + 1, 512), p.halves(n + 1, 32)
        pages, pool = p.device()
        kvs.kv_latent_append_tokens(pages, 0, put(c), put(r), put(start))
        ol.append(p.os, p.pool, *p.table(), 0, c, r, start)
        assert np.array_equal(pool.cpu().numpy(), p.pool)
        back = torch.full((n + 1, 512), 7.0, dtype=torch.float16, device="cuda"), torch.full((n + 1, 32), 7.0, dtype=torch.float16, device="cuda")
        kvs.kv_latent_read_tokens(pages, 0, *back, put(start))
        c_want, r_want = np.full_like(c, 7.0), np.full_like(r, 7.0)
        ol.read(p.os, p.pool, *p.table(), 0, c_want, r_want, start)
        assert np.array_equal(back[0].cpu().numpy(), c_want) and np.array_equal(back[1].cpu().numpy(), r_want)


def test_latent_pages_are_on_the_current_device_and_fixed():
    p = Latent((1, 1, 256, 32, 64, 64, 16, 16, 64), [4], (16,), 24)
    pages, _ = p.device()
    for name in ("pool", "off", "bits", "length", "shape", "n_seqs"):
        with pytest.raises(AttributeError):
            setattr(pages, name, getattr(pages, name))
    c, r = torch.zeros((1, 256), dtype=torch.float16, device="cuda"), torch.zeros((1, 32), dtype=torch.float16, device="cuda")
    for bad in ((c.float(), r), (c, r.cpu()), (c[:, :128], r), (c, r.repeat(2, 1)), (c.t().contiguous().t().expand(1, 256)[:, ::1].float(), r)):
        with pytest.raises((ValueError, TypeError)):
            kvs.kv_latent_append_tokens(pages, 0, *bad)
    q, w = put(p.queries(1)), put(p.weights())
    out, ws = torch.zeros((1, 1, 64), dtype=torch.float16, device="cuda"), space(p)
    for bad in ((q[:, :, :64], w, ws, out), (q, w[:, :, :64], ws, out), (q, w, ws[:64], out), (q, w, ws.cpu(), out), (q, w, ws, out.float())):
        with pytest.raises((ValueError, TypeError, kvs.KvError)):
            kvs.kv_latent_attend_tokens(pages, 0, *bad)


@pytest.mark.parametrize("heads,most", [(16, 9), (40, 4), (64, 3)])
def test_one_workspace_for_the_longest_and_all_shorter_steps(heads, most):
    """Drafts of one to `most` rows, whose query rows pass from one tile to three lower ones, in the workspace of the longest."""
    p = Latent((1, heads, 256, 32, 64, 64, 1024, 16, 64), [1000, 17, 640], MIXED, 41)
    pages, _ = p.device()
    w, shared = put(p.weights()), space(p, max_rows=most)
    for m in range(1, most + 1):
        start, n = rows([m, 1, max(m - 1, 0)])
        q, start = put(p.queries(n)), put(start)
        out = torch.zeros((2, n, heads, 64), dtype=torch.float16, device="cuda")
        kvs.kv_latent_attend_tokens(pages, 0, q, w, shared, out[0], row_start=start, max_rows=m)
        kvs.kv_latent_attend_tokens(pages, 0, q, w, space(p, max_rows=m), out[1], row_start=start, max_rows=m)
        torch.cuda.synchronize()
        assert same(out[0], out[1]) and bool(out.any())
