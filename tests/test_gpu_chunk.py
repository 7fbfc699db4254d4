"""sd_chunk_attn_paged against the plain form in 64 bits: ragged chunks from no row to hundreds, head
groups, head sizes, pages that end inside a tile, both masks; what must not change does not."""
import threading

import numpy as np
import pytest
import torch

import gpu_util as G
import paper_2606_31315_amd as sd
import prefill_ref as R

pytestmark = pytest.mark.gpu
CAUSAL, BIDIR = R.CAUSAL, R.BIDIR


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(G.dev())


def _run(b, mask, **kw):
    kw.setdefault("max_ctx", int(b["ctx"].max()))
    kw.setdefault("max_chunk", max(1, int(b["B"].max())))
    G.log(f"sd_chunk_attn_paged q={list(b['q'].shape)} pool={list(b['kp'].shape)} ctx={b['ctx'][:8].tolist()} "
          f"B={b['B'][:8].tolist()} mask={mask}")
    o = sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], _i32(b["ctx"]), _i32(b["B"]), _i32(b["off"]), mask, **kw)
    torch.cuda.synchronize()
    return o


def _check(b, mask, scale=0.0, **kw):
    o = _run(b, mask, scale=scale, **kw)
    R.assert_attended(o, b["q"], b["kp"], b["vp"], b["table"], b["ctx"], b["B"], b["off"], mask, scale)
    return o


CASES = [  # Hq, Hkv, D, page, contexts, rows
    ("one_row_over_64", 32, 8, 128, 16, [0], [65]),
    ("tile_edges", 32, 8, 128, 64, [0, 64, 63, 1], [64, 65, 128, 63]),
    ("odd_lengths", 32, 8, 128, 16, [1000, 17, 0, 333], [131, 77, 5, 200]),
    ("rows_of_every_kind", 32, 8, 128, 32, [500, 0, 2000, 129, 0, 64], [1, 0, 300, 1, 1, 64]),
    ("one_head_to_a_group", 8, 8, 128, 64, [100, 0], [300, 257]),
    ("all_heads_in_a_group", 32, 1, 128, 256, [777, 5], [70, 9]),
    ("group_of_five", 10, 2, 128, 16, [90, 0], [140, 66]),
    ("group_of_eight_small_heads", 32, 4, 64, 128, [1500, 3], [90, 100]),
    ("small_heads", 8, 8, 64, 32, [300, 0, 47], [260, 512, 1]),
    ("group_of_three_small_heads", 6, 2, 64, 16, [10, 700], [170, 86]),
    ("long_context_few_rows", 32, 8, 128, 64, [9000], [70]),
    ("single_rows_beside_a_chunk", 32, 8, 128, 16, [3000, 1999, 12, 700, 1], [1, 1, 1, 400, 1]),
]


@pytest.mark.parametrize("mask", [CAUSAL, BIDIR], ids=["causal", "bidir"])
@pytest.mark.parametrize("name,Hq,Hkv,D,page,ctx,B", CASES, ids=[c[0] for c in CASES])
def test_parity(name, Hq, Hkv, D, page, ctx, B, mask):
    _check(R.chunk_batch(len(name), Hq, Hkv, D, page, ctx, B, G.dev()), mask)


@pytest.mark.parametrize("name,Hq,Hkv,D,page,ctx,B", CASES, ids=[c[0] for c in CASES])
def test_parity_planned(name, Hq, Hkv, D, page, ctx, B):
    """The same rows beside a long context without rows, whose bound has the batch planned."""
    _check(R.chunk_batch(len(name) + 300, Hq, Hkv, D, page, ctx + [10500], B + [0], G.dev()), CAUSAL)


@pytest.mark.parametrize("mask", [CAUSAL, BIDIR], ids=["causal", "bidir"])
@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (24, 8, 64)])
def test_many_short_chunks(Hq, Hkv, D, mask):
    """More tiles of 128 rows than CUs, fewer of 256: whole tiles in one launch."""
    B = [65, 1, 90, 0, 130, 64, 65, 66, 2, 33, 100, 127, 5, 70]
    ctx = [0, 77, 300, 1000, 5, 64, 63, 640, 1, 0, 129, 400, 1000, 31]
    _check(R.chunk_batch(14, Hq, Hkv, D, 16, ctx, B, G.dev()), mask)


@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (8, 8, 64), (128, 1, 128), (129, 1, 64)])
def test_lengths_about_a_step(Hq, Hkv, D):
    """One tile, two, three and four of 64 keys, or one less or more: a step's second tile may hold one key or none."""
    for ctx in (0, 1, 54, 55, 56, 63, 64, 118, 119, 120, 183, 190):
        b = R.chunk_batch(400 + ctx, Hq, Hkv, D, 16, [ctx, 200], [9, 2], G.dev())
        _check(b, CAUSAL, max_chunk=208)
        _check(b, BIDIR, max_chunk=208)


@pytest.mark.parametrize("B", [[1, 1, 1], [5, 16, 0], [17, 64, 33]], ids=["tokens", "blocks", "to_64_rows"])
def test_short_chunks(B):
    """Batches that the block attention's kernels take."""
    _check(R.chunk_batch(11, 32, 8, 128, 32, [700, 0, 2500], B, G.dev()), CAUSAL)


@pytest.mark.parametrize("mask", [CAUSAL, BIDIR], ids=["causal", "bidir"])
@pytest.mark.parametrize("Hq,Hkv,D,most", [(32, 8, 128, 24), (32, 8, 128, 64), (32, 8, 64, 17), (8, 8, 64, 64)])
def test_blocks_of_many_sequences(Hq, Hkv, D, most, mask):
    """Blocks that the block kernels could take beside contexts short enough for the chunk kernel's halves, and the
    same beside one that is not."""
    rng = np.random.default_rng(most)
    B, ctx = rng.integers(0, most + 1, 14), rng.integers(0, 450, 14)
    B[:3], ctx[:3] = [most, 0, 1], [449, 13, 0]
    _check(R.chunk_batch(15, Hq, Hkv, D, 16, ctx, B, G.dev()), mask)
    ctx[4] = 5000
    _check(R.chunk_batch(16, Hq, Hkv, D, 16, ctx, B, G.dev()), mask)


def test_64_rows_over_many_keys():
    """Enough keys for the chunk kernel to take blocks that the block kernels could, and the same rows beside fewer keys."""
    b = R.chunk_batch(12, 16, 4, 128, 64, [13000, 12000, 9000, 20, 16000], [64, 1, 33, 64, 0], G.dev())
    _check(b, CAUSAL, max_ctx=16000)
    _check(R.chunk_batch(13, 16, 4, 128, 64, [600, 20, 0], [64, 1, 33], G.dev()), CAUSAL)


def test_many_sequences():
    """More than 64 sequences: the lookup of a workgroup's share crosses rounds, with empty ones at its edge."""
    rng = np.random.default_rng(5)
    B = rng.integers(0, 90, 150)
    B[[0, 62, 63, 64, 127, 128, 149]] = [0, 0, 0, 81, 0, 3, 0]
    _check(R.chunk_batch(6, 16, 8, 64, 16, rng.integers(0, 300, 150), B, G.dev()), CAUSAL)


@pytest.mark.parametrize("sigma,scale", [(6.0, 0.0), (1.0, 0.5), (1e-3, 0.0)], ids=["sharp", "scaled", "flat"])
def test_scores(sigma, scale):
    """Sharp and flat softmaxes, a scale of the caller's: the running maximum moves often, or not."""
    _check(R.chunk_batch(21, 16, 4, 128, 64, [600, 50], [130, 200], G.dev(), sigma=sigma), CAUSAL, scale=scale)


def test_growing_scores():
    """Keys whose scores grow along the context, by far more than any threshold at once: every step moves the
    maximum."""
    b = R.chunk_batch(22, 8, 2, 128, 64, [700], [100], G.dev())
    b["q"].copy_(b["q"].abs())
    for s in range(1):
        n = b["table"].shape[1]
        ramp = (torch.arange(n * 64, device=G.dev()) / 100.0).reshape(1, n, 64, 1).transpose(0, 1)
        b["kp"][b["table"][s].long()] = (b["kp"][b["table"][s].long()] * 0.05 + ramp).to(torch.bfloat16)
    _check(b, CAUSAL, scale=0.05)


@pytest.mark.parametrize("rows,max_chunk", [((100, 71), 5000), ((40, 1), 64)], ids=["chunk_kernel", "block_kernels"])
def test_loose_bounds_and_padding(rows, max_chunk):
    """Bounds far above the lengths, a batch padded with rows and sequences: rows behind the last sequence
    stay as they were."""
    b = R.chunk_batch(31, 32, 8, 128, 16, [300, 0, 40, 0], [rows[0], 0, rows[1], 0], G.dev())
    n = int(b["off"][-1])
    b["q"] = torch.cat([b["q"], torch.full((37, 32, 128), float("nan"), dtype=torch.bfloat16, device=G.dev())])
    table = torch.zeros(4, 1024, dtype=torch.int32, device=G.dev())
    table[:, :b["table"].shape[1]] = b["table"]
    b["table"] = table
    out = torch.full_like(b["q"], 7.0)
    o = _check(b, CAUSAL, out=out, max_ctx=9000, max_chunk=max_chunk)
    assert o is out and bool((out[n:] == 7.0).all())


def test_minus_infinite_and_lowest_scores():
    """A key that nothing may weigh (score of the type's lowest values, -inf): weight 0, as in softmax."""
    b = R.chunk_batch(41, 4, 4, 128, 64, [200], [80], G.dev())
    b["q"].copy_(b["q"].abs() + 0.5)
    t = b["table"][0].long()
    b["kp"][t[0], :, 5] = -torch.finfo(torch.bfloat16).max / 1024
    b["kp"][t[1], :, 3] = float("-inf")
    _check(b, CAUSAL)


def test_page_ids_outside_the_pool_stay_inside():
    """Ids that the contract forbids are clamped into the pool: sequences with sound ids are not touched by it."""
    b = R.chunk_batch(51, 16, 8, 128, 16, [100, 90], [70, 80], G.dev())
    good = _run(b, CAUSAL)
    b["table"] = b["table"].clone()
    b["table"][0, 1], b["table"][0, 2] = 2 ** 30, -5
    bad = _run(b, CAUSAL)
    assert torch.equal(bad[70:], good[70:])


def test_pools_past_32_bit_offsets():
    """Pages beyond 2^31 elements of the pool, the last one among them."""
    dev, page, Hkv, D = G.dev(), 256, 8, 128
    n = (1 << 31) // (Hkv * page * D) + 40
    b = R.chunk_batch(61, 16, Hkv, D, page, [700], [100], dev)
    kp, vp = (torch.empty((n, Hkv, page, D), dtype=torch.bfloat16, device=dev) for _ in range(2))
    ids = torch.tensor([n - 1, n - 30, 3, n - 2], device=dev)[:b["table"].shape[1]]
    for big, x in ((kp, b["kp"]), (vp, b["vp"])):
        big[ids] = x[b["table"][0].long()]
    b.update(kp=kp, vp=vp, table=ids.to(torch.int32)[None].contiguous())
    _check(b, CAUSAL)


def test_same_call_same_bits_on_another_stream_and_workspace():
    b = R.chunk_batch(71, 32, 8, 128, 64, [3000, 0, 511], [200, 333, 1], G.dev())
    ref = _run(b, CAUSAL)
    sh = sd._lib.SdAttnShape(3, 32, 8, 128, b["table"].shape[1] * 64, b["q"].shape[0], 3000, 333, sd.SD_BF16, 0.0)
    ws = torch.full((sd.chunk_attn_workspace_size(sh),), 255, dtype=torch.uint8, device=G.dev())  # NaN throughout
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = _run(b, CAUSAL, workspace=ws)
    assert torch.equal(got, ref)
    assert torch.equal(_run(b, CAUSAL, stream=st), ref)


@pytest.mark.parametrize("max_chunk", [64, 400], ids=["block_kernels", "chunk_kernel"])
def test_graph_replays(max_chunk):
    """Captured once, replayed with other lengths and contents inside the bounds: equal to eager calls."""
    dev = G.dev()
    b = R.chunk_batch(81, 16, 8, 128, 32, [2000, 1500, 64], [64 if max_chunk == 64 else 300, 20, 1], dev)
    lens = [(b["ctx"], b["B"]), (b["ctx"] // 3, np.minimum(b["B"], [40, 20, 1])), (b["ctx"] * 0 + 5, b["B"] * 0 + 1)]
    ctx, B, off = _i32(b["ctx"]), _i32(b["B"]), _i32(b["off"])
    outs = {x: torch.zeros_like(b["q"]) for x in ("graph", "eager")}
    sh = sd._lib.SdAttnShape(3, 16, 8, 128, b["table"].shape[1] * 32, b["q"].shape[0], 2000, max_chunk, sd.SD_BF16, 0.0)
    ws = {x: torch.empty(sd.chunk_attn_workspace_size(sh), dtype=torch.uint8, device=dev) for x in outs}

    def call(x):
        sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], ctx, B, off, CAUSAL, max_ctx=2000,
                            max_chunk=max_chunk, out=outs[x], workspace=ws[x])

    call("eager")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call("graph")
    for i in range(6):
        c, n = lens[i % 3]
        o = np.concatenate([[0], np.cumsum(n)])
        ctx.copy_(_i32(c)), B.copy_(_i32(n)), off.copy_(_i32(o))
        outs["graph"].zero_(), outs["eager"].zero_()
        call("eager")
        torch.cuda.synchronize()
        G.log(f"  replay {i}")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs["graph"], outs["eager"]), i


def test_empty_calls():
    dev = G.dev()
    b = R.chunk_batch(91, 16, 8, 128, 16, [10, 0], [0, 0], dev)
    assert _run(b, CAUSAL, max_chunk=16).shape[0] == 0
    b = R.chunk_batch(92, 16, 8, 128, 16, [10], [80], dev)  # rows, but every sequence empty on the device
    out = torch.full_like(b["q"], 3.0)
    b["B"], b["off"] = b["B"] * 0, b["off"] * 0
    assert bool((_run(b, CAUSAL, out=out, max_chunk=80) == 3.0).all())


def test_capture_needs_a_workspace():
    b = R.chunk_batch(93, 16, 8, 128, 16, [10], [80], G.dev())
    ctx, B, off = _i32(b["ctx"]), _i32(b["B"]), _i32(b["off"])
    out = torch.empty_like(b["q"])
    x = torch.zeros(1, device=G.dev())
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        x.add_(1)
        with pytest.raises(ValueError, match="workspace"):
            sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], ctx, B, off, CAUSAL, max_ctx=10, max_chunk=80, out=out)


def test_a_captured_stream_that_is_not_the_current_one_needs_a_workspace():
    b = R.chunk_batch(94, 16, 8, 128, 16, [10], [80], G.dev())
    lens = [_i32(b[x]) for x in ("ctx", "B", "off")]
    out, x, other = torch.empty_like(b["q"]), torch.zeros(1, device=G.dev()), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        x.add_(1)
        captured = torch.cuda.current_stream()
        with torch.cuda.stream(other), pytest.raises(ValueError, match="workspace"):
            sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], *lens, CAUSAL, max_ctx=10, max_chunk=80, out=out,
                                stream=captured)


def test_two_streams_at_once_without_workspaces():
    """Calls on two streams that run at the same time, growing their buffers: each as alone."""
    batches = [R.chunk_batch(101 + i, 32, 8, 128, 64, [2000 + 900 * i, 0, 64], [150 + 70 * i, 200, 1], G.dev()) for i in range(4)]
    refs = [_run(b, CAUSAL) for b in batches]
    lens = [[_i32(b[x]) for x in ("ctx", "B", "off")] for b in batches]
    outs = [torch.zeros_like(b["q"]) for b in batches]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    G.log("sd_chunk_attn_paged on two streams at once")
    for i, (b, l, o) in enumerate(zip(batches, lens, outs)):
        sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], *l, CAUSAL, max_ctx=int(b["ctx"].max()),
                            max_chunk=int(b["B"].max()), out=o, stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, r) for o, r in zip(outs, refs))


def test_two_threads_on_one_stream_without_workspaces():
    batches = [R.chunk_batch(111 + i, 32, 8, 128, 64, [2500 + 900 * i, 0], [150 + 70 * i, 200], G.dev()) for i in range(2)]
    refs = [_run(b, CAUSAL) for b in batches]
    lens = [[_i32(b[x]) for x in ("ctx", "B", "off")] for b in batches]
    torch.cuda.synchronize()
    G.log("sd_chunk_attn_paged from two threads on one stream")
    outs = [[], []]

    def work(i):
        b = batches[i]
        for _ in range(20):
            outs[i].append(sd.chunk_attn_paged(b["q"], b["kp"], b["vp"], b["table"], *lens[i], CAUSAL,
                                               max_ctx=int(b["ctx"].max()), max_chunk=int(b["B"].max())))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(o, refs[i]) for i in range(2) for o in outs[i]) and [len(o) for o in outs] == [20, 20]


@pytest.mark.parametrize("S", [1025, 1500], ids=["just_past", "well_past"])
def test_more_sequences_than_the_plan_orders(S):
    """Batches past the plan's sorting, most of them single rows, on the planned path."""
    rng = np.random.default_rng(S)
    B = np.where(rng.random(S) < 0.05, rng.integers(60, 100, S), rng.integers(0, 3, S))
    B[[3, 1024]] = [300, 77]
    _check(R.chunk_batch(S, 8, 2, 64, 16, rng.integers(0, 60, S), B, G.dev()), CAUSAL)


@pytest.mark.parametrize("D", [64, 128])
def test_cut_tiles_over_long_contexts(D):
    """Tiles cut into many pieces, rows that see nothing of the last ones, short sequences beside them."""
    _check(R.chunk_batch(111 + D, 8, 2, D, 64, [20000, 0, 333], [100, 65, 1], G.dev()), CAUSAL)
    _check(R.chunk_batch(112 + D, 4, 4, D, 64, [0], [2500], G.dev()), CAUSAL)


def test_whole_batches_of_every_path_agree_with_their_chunks():
    """One prompt in one chunk and in uneven chunks: each within its tolerance of the plain form."""
    b = R.chunk_batch(121, 16, 4, 128, 64, [0], [900], G.dev())
    _check(b, CAUSAL)
    done = 0
    for n in (1, 64, 65, 300, 470):
        c = dict(b, q=b["q"][done:done + n].contiguous(), ctx=np.array([done], np.int32), B=np.array([n], np.int32),
                 off=np.array([0, n], np.int32))
        _check(c, CAUSAL)
        done += n
    assert done == 900
