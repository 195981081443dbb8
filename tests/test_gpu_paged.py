"""The paged cache and attention over it on the GPU against float64 (tests/paged_ref.py)."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paged_ref as ref

pytestmark = pytest.mark.gpu

OK, SHAPE, INDEX = 0, 2, 4


@pytest.fixture(scope="module")
def pa():
    import paper_2605_03110_amd as mod
    assert torch.cuda.is_available()
    return mod


# ------------------------------------------------------------------------------------------------ attention
# name, case, causal
ATTEND = {
    "one_token": lambda: ref.Case("bf16", 4, 1, 64, 16, [1], [0]),
    "one_token_17": lambda: ref.Case("bf16", 8, 8, 128, 16, [1], [16]),
    "tokens_ragged": lambda: ref.Case("bf16", 8, 2, 128, 16, [1, 1, 1, 1, 1], [0, 1, 127, 128, 1000], spare_columns=3),
    "tokens_group_7": lambda: ref.Case("bf16", 14, 2, 64, 32, [1, 1, 1], [95, 300, 63]),
    "tokens_group_20": lambda: ref.Case("bf16", 40, 2, 64, 64, [1, 1], [200, 5]),
    "tokens_256": lambda: ref.Case("bf16", 4, 2, 256, 128, [1, 1], [511, 40]),
    "tokens_f32": lambda: ref.Case("f32", 6, 2, 64, 16, [1, 1, 1], [700, 2, 33]),
    "tokens_f32_128": lambda: ref.Case("f32", 5, 5, 128, 256, [1, 1], [255, 600]),
    "chunk": lambda: ref.Case("bf16", 8, 2, 128, 16, [77], [100]),
    "chunk_long": lambda: ref.Case("bf16", 4, 4, 128, 64, [600], [37]),
    "chunk_64": lambda: ref.Case("bf16", 6, 2, 64, 32, [200, 129], [0, 511], order="slots"),
    "chunk_256": lambda: ref.Case("bf16", 2, 2, 256, 64, [150], [333]),
    "chunk_f32": lambda: ref.Case("f32", 4, 2, 64, 32, [97], [64], order="slots"),
    "chunk_f32_128": lambda: ref.Case("f32", 2, 1, 128, 16, [40, 3], [0, 130]),
    "mixed": lambda: ref.Case("bf16", 8, 2, 128, 16, [1, 0, 33, 300, 1, 0, 2], [40, 9, 0, 17, 513, 0, 64], pad_rows=5),
    "large_scores": lambda: ref.Case("bf16", 4, 2, 128, 32, [130, 1], [70, 400], scale=8.0),
    "many_tokens": lambda: ref.Case("bf16", 4, 1, 64, 16, [1] * 150, [(37 * b) % 331 for b in range(150)]),
    "many_chunks": lambda: ref.Case("bf16", 4, 2, 64, 32, [(b * 7) % 23 for b in range(130)], [(37 * b) % 200 for b in range(130)]),
    "many_chunks_f32": lambda: ref.Case("f32", 4, 2, 64, 16, [(b * 7) % 9 for b in range(70)], [(37 * b) % 90 for b in range(70)]),
    "long_token": lambda: ref.Case("bf16", 2, 1, 128, 256, [1], [70000]),
    "long_chunk": lambda: ref.Case("bf16", 16, 1, 64, 16, [9], [20000]),
    "values_off_zero": lambda: ref.Case("bf16", 4, 2, 64, 16, [64, 1], [0, 900], value_shift=3.0),
}


def step_of(c):
    """How exactly the products take a weight: bf16 caches as one bf16 number (half a step: 2^-8) at worst, fp32 exactly."""
    return 0.0 if c.dtype == torch.float32 else 2.0 ** -8


def check_attend(c, got, causal, lists=None, drop=()):
    want, weight, err = ref.attend(c, causal, lists, drop)
    n = int(c.start[-1])
    off = (got.double().cpu()[:n] - want[:n]).abs()
    room = ref.tolerance(c, want, weight, err, step_of(c))[:n]
    assert bool((off <= room).all()), "off by %.3g where %.3g is allowed" % (float(off[off > room].max()), float(room[off > room].max()))


@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("name", ATTEND)
def test_attention(pa, name, causal):
    c = ATTEND[name]()
    cache, chunk = c.on_gpu(pa)
    out = torch.full((c.rows, c.H * c.d_h), 7.0, dtype=c.dtype, device="cuda")
    res = pa.ada_attention_paged(cache, chunk, c.Q.cuda(), out=out, flags=pa.FLAG_ATTN_CAUSAL if causal else 0)
    assert res["status"].item() == OK
    assert bool((out[int(c.start[-1]):] == 7.0).all()), "rows behind the last sequence"
    check_attend(c, out, causal)


# enough rows for the tiles of 128 rows on any number of CUs up to 256 (more than half as many tiles of 16 rows as CUs)
TILES = {
    "group_4": lambda: ref.Case("bf16", 32, 8, 128, 16, [77], [100], pad_rows=3),
    "heads_64": lambda: ref.Case("bf16", 12, 2, 64, 32, [200, 129], [0, 511], order="slots"),
    "heads_256": lambda: ref.Case("bf16", 8, 4, 256, 64, [150], [333]),
    "heads_256_many_parts": lambda: ref.Case("bf16", 8, 2, 256, 16, [101], [3000], order="slots"),
    "mixed": lambda: ref.Case("bf16", 16, 4, 128, 16, [1, 0, 33, 300, 1, 0, 2], [40, 9, 0, 17, 513, 0, 64], pad_rows=5),
    "large_scores": lambda: ref.Case("bf16", 16, 8, 128, 32, [160, 1], [70, 400], scale=8.0),
    "many_parts": lambda: ref.Case("bf16", 64, 4, 64, 16, [40], [9000]),
    "many_sequences": lambda: ref.Case("bf16", 16, 2, 64, 32, [(b * 7) % 23 for b in range(130)], [(37 * b) % 200 for b in range(130)]),
    "values_off_zero": lambda: ref.Case("bf16", 16, 4, 128, 16, [164, 1], [0, 900], value_shift=3.0),
}


@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("name", TILES)
def test_attention_in_tiles(pa, name, causal):
    """Twice over one workspace, which is found as it was left: a batch with chunks of more rows."""
    c = TILES[name]()
    cache, chunk = c.on_gpu(pa)
    ws = pa.paged_workspace(cache, chunk, c.H)
    ws[pa.PAGED_ZERO_BYTES:].fill_(255)
    first = None
    for _ in range(2):
        out = torch.full((c.rows, c.H * c.d_h), 7.0, dtype=c.dtype, device="cuda")
        res = pa.ada_attention_paged(cache, chunk, c.Q.cuda(), out=out, ws=ws, flags=pa.FLAG_ATTN_CAUSAL if causal else 0)
        assert res["status"].item() == OK
        assert bool((out[int(c.start[-1]):] == 7.0).all()), "rows behind the last sequence"
        assert bool((ws[:pa.PAGED_ZERO_BYTES] == 0).all())
        assert first is None or torch.equal(first, out)
        first = out
    check_attend(c, first, causal)


def test_tiles_of_strided_rows_with_pages_outside_the_pool(pa):
    c = ref.Case("bf16", 32, 8, 128, 16, [1, 1, 90], [100, 15, 0])
    c.table[0, 2] = c.pages
    c.table[1, 0] = -1                                     # all that this row sees
    c.table[2, 1] = 2 ** 31 - 1
    cache, chunk = c.on_gpu(pa)
    wide = torch.full((c.rows, 34 * 128), math.nan, dtype=c.dtype, device="cuda")
    wide[:, 128:33 * 128] = c.Q.cuda()
    out = torch.full((c.rows, 33 * 128), 7.0, dtype=c.dtype, device="cuda")
    res = pa.ada_attention_paged(cache, chunk, wide[:, 128:33 * 128], out=out[:, 128:], flags=pa.FLAG_ATTN_CAUSAL)
    assert res["status"].item() == INDEX
    assert bool((out[:, :128] == 7.0).all()) and bool((out[1, 128:] == 0).all())
    check_attend(c, out[:, 128:], True, drop=((0, 2), (1, 0), (2, 1)))


def test_attention_of_strided_rows(pa):
    c = ref.Case("bf16", 4, 2, 64, 16, [20, 1], [33, 80])
    cache, chunk = c.on_gpu(pa)
    wide = torch.full((c.rows, 6 * 64), math.nan, dtype=c.dtype, device="cuda")
    wide[:, 64:5 * 64] = c.Q.cuda()
    out = torch.full((c.rows, 5 * 64), 7.0, dtype=c.dtype, device="cuda")
    pa.ada_attention_paged(cache, chunk, wide[:, 64:5 * 64], out=out[:, 64:], flags=pa.FLAG_ATTN_CAUSAL)
    assert bool((out[:, :64] == 7.0).all())
    check_attend(c, out[:, 64:], True)


def test_attention_is_the_same_on_every_run(pa):
    c = ATTEND["tokens_ragged"]()
    cache, chunk = c.on_gpu(pa)
    ws = pa.paged_workspace(cache, chunk, c.H)
    first = pa.ada_attention_paged(cache, chunk, c.Q.cuda(), ws=ws)["out"]
    for fill in (0, 255):
        ws[pa.PAGED_ZERO_BYTES:].fill_(fill)               # nothing is expected of the rest of a workspace
        assert torch.equal(first, pa.ada_attention_paged(cache, chunk, c.Q.cuda(), ws=ws)["out"])
        assert bool((ws[:pa.PAGED_ZERO_BYTES] == 0).all())


def test_pages_outside_the_pool_count_as_masked(pa):
    c = ref.Case("bf16", 4, 2, 128, 16, [1, 1, 40], [100, 15, 0])
    c.table[0, 2] = c.pages
    c.table[1, 0] = -1                                     # all that this row sees
    c.table[2, 1] = 2 ** 31 - 1
    cache, chunk = c.on_gpu(pa)
    res = pa.ada_attention_paged(cache, chunk, c.Q.cuda(), flags=pa.FLAG_ATTN_CAUSAL)
    assert res["status"].item() == INDEX
    assert bool((res["out"][1] == 0).all())
    check_attend(c, res["out"], True, drop=((0, 2), (1, 0), (2, 1)))


@pytest.mark.parametrize("make", (lambda: ref.Case("bf16", 8, 2, 128, 16, [1] * 6, [100, 300, 15, 7, 1000, 40]),
                                  lambda: ref.Case("f32", 4, 2, 64, 16, [1] * 6, [100, 300, 15, 7, 1000, 40]),
                                  lambda: ref.Case("bf16", 32, 8, 128, 16, [30, 20, 1, 50, 2, 3], [100, 300, 15, 7, 1000, 40])))
def test_numbers_that_are_none_stay_in_their_sequence(pa, make):
    c = make()
    cache, chunk = c.on_gpu(pa)
    for b, value in ((1, math.nan), (4, math.inf)):
        for pages in (cache.K, cache.V):
            pages[c.table[b, 0].item()][:, 3] = value
            pages[c.table[b, 0].item()][:, 5] = -value
    out = pa.ada_attention_paged(cache, chunk, c.Q.cuda(), flags=pa.FLAG_ATTN_CAUSAL)["out"].double().cpu()
    want, weight, err = ref.attend(c, True)
    room = ref.tolerance(c, want, weight, err, step_of(c))
    for b in (0, 2, 3, 5):
        rows = slice(int(c.start[b]), int(c.start[b + 1]))
        assert bool(((out - want).abs() <= room)[rows].all()), b


def test_sequences_that_do_not_fit_are_left_out(pa):
    c = ref.Case("bf16", 4, 2, 64, 16, [3, 1, 2], [20, 7, 30])
    for what in ("past", "long", "behind"):
        cache, chunk = c.on_gpu(pa)
        if what == "past":
            chunk.past[1] = -1
        elif what == "long":
            chunk.past[1] = chunk.table.shape[1] * 16
        else:
            chunk.start[2:] = 2 ** 30
        out = torch.full((c.rows, c.H * c.d_h), 7.0, dtype=c.dtype, device="cuda")
        res = pa.ada_attention_paged(cache, chunk, c.Q.cuda(), out=out, flags=pa.FLAG_ATTN_CAUSAL)
        assert res["status"].item() == SHAPE
        assert bool((out[3] == 7.0).all())
        want, weight, err = ref.attend(c, True)
        room = ref.tolerance(c, want, weight, err, step_of(c))
        keep = [0, 1, 2] + ([] if what == "behind" else [4, 5])
        assert bool(((out.double().cpu() - want).abs() <= room)[keep].all())


@pytest.mark.parametrize("longest", (1, 8, 40))
def test_sequences_that_overlap_stay_in_bounds(pa, longest):
    """Starts that go back and forth: more tiles than rows make.  Whatever is written, it is written inside, and the call says so."""
    c = ref.Case("bf16", 4, 2, 64, 16, [longest] * 3, [20, 7, 30])
    cache, _ = c.on_gpu(pa)
    B = 600
    start = torch.tensor([0, longest] * (B // 2) + [0], dtype=torch.int32, device="cuda")
    table = c.table[:1].repeat(B, 1).cuda()
    chunk = pa.Chunk(table, start, torch.full((B,), 3, dtype=torch.int32, device="cuda"), rows=longest, longest=longest)
    ws = pa.paged_workspace(cache, chunk, c.H)
    guard = torch.full((ws.numel() + 4096,), 77, dtype=torch.uint8, device="cuda")
    guard[:ws.numel()] = ws
    out = torch.full((longest + 1, c.H * 64), 7.0, dtype=c.dtype, device="cuda")
    res = pa.ada_attention_paged(cache, chunk, c.Q[:longest].cuda(), ws=guard[:ws.numel()], out=out, flags=pa.FLAG_ATTN_CAUSAL)
    assert res["status"].item() == SHAPE
    assert bool((out[longest] == 7.0).all()) and bool((guard[ws.numel():] == 77).all())
    assert bool((guard[:pa.PAGED_ZERO_BYTES] == 0).all())


def test_status_is_raised_and_never_cleared(pa):
    c = ATTEND["chunk"]()
    cache, chunk = c.on_gpu(pa)
    word = torch.full((1,), INDEX, dtype=torch.int32, device="cuda")
    pa.ada_attention_paged(cache, chunk, c.Q.cuda(), status=word)
    assert word.item() == INDEX


# ------------------------------------------------------------------------------------------------ appending
APPEND = {
    "tokens": (lambda: ref.Case("bf16", 4, 2, 128, 16, [1, 1, 1, 1], [0, 15, 16, 100]), 128, False, True),
    "tokens_pairs": (lambda: ref.Case("bf16", 3, 1, 256, 32, [1, 1], [31, 32]), 64, True, False),
    "tokens_f32": (lambda: ref.Case("f32", 2, 2, 64, 16, [1, 1, 1], [0, 3, 47]), 32, False, True),
    "chunk": (lambda: ref.Case("bf16", 8, 2, 128, 64, [100, 1, 0, 63], [30, 64, 5, 0], pad_rows=3), 128, False, True),
    "chunk_pairs": (lambda: ref.Case("bf16", 4, 4, 256, 16, [50, 16], [0, 31], order="slots"), 64, True, True),
    "chunk_part": (lambda: ref.Case("bf16", 2, 1, 128, 16, [40, 7], [9, 0]), 32, False, False),
    "chunk_f32": (lambda: ref.Case("f32", 4, 2, 128, 32, [33, 64], [1, 0], order="slots"), 128, True, True),
    "chunk_f32_part": (lambda: ref.Case("f32", 6, 3, 64, 256, [300], [77]), 16, False, True),
    "two_launches": (lambda: ref.Case("bf16", 16, 8, 128, 32, [1500, 1, 333, 50], [70, 31, 0, 5], pad_rows=9), 128, False, True),
    "two_launches_f32": (lambda: ref.Case("f32", 16, 16, 64, 128, [1400], [333], order="slots"), 32, True, False),
    "no_rotation": (lambda: ref.Case("bf16", 2, 2, 64, 16, [5, 1], [14, 0]), 0, False, True),
    "copy": (lambda: ref.Case("f32", 2, 2, 64, 16, [5, 1], [14, 0]), 0, False, False),
}


def rows_in(c):
    g = torch.Generator().manual_seed(99)
    qkv = torch.randn(max(c.rows, 1), (c.H + 2 * c.H_kv) * c.d_h, generator=g).to(c.dtype)
    weights = [(1 + 0.2 * torch.randn(c.d_h, generator=g)).to(c.dtype) for _ in range(2)]
    return qkv, weights


@pytest.mark.parametrize("with_q", (True, False))
@pytest.mark.parametrize("name", APPEND)
def test_append(pa, name, with_q):
    make, rot, pairs, norm = APPEND[name]
    c = make()
    c.K, c.V, c.bounds = c.pool()                          # what is there already: the tokens in front
    for b in range(c.B):
        c.fill(b, 0, c.past[b])
    before_K, before_V, before_bounds = c.K.clone(), c.V.clone(), c.bounds.clone()
    cache, chunk = c.on_gpu(pa)
    qkv, (wq, wk) = rows_in(c)
    table = ref.rope_table(max(c.total), rot) if rot else None
    eps = 1e-5
    q, k, v = qkv.cuda().split((c.H * c.d_h, c.H_kv * c.d_h, c.H_kv * c.d_h), dim=1)
    out = torch.full((max(c.rows, 1), c.H * c.d_h), 7.0, dtype=c.dtype, device="cuda") if with_q else None
    res = pa.ada_cache_append(cache, chunk, q if with_q else None, k, v, rope=None if table is None else table.cuda(),
                              q_norm=wq.cuda() if norm else None, k_norm=wk.cuda() if norm else None, eps=eps, out=out,
                              flags=pa.FLAG_ROPE_PAIRS if pairs else 0)
    assert res["status"].item() == OK
    half = torch.finfo(c.dtype).eps / 2
    qc, kc, vc = qkv.split((c.H * c.d_h, c.H_kv * c.d_h, c.H_kv * c.d_h), dim=1)
    K, V, bounds = cache.K.cpu(), cache.V.cpu(), cache.bounds.cpu()
    want_K, want_V = before_K, before_V
    for b in range(c.B):
        r0, r1 = c.rows_of(b)
        pos = torch.arange(c.past[b], c.total[b])
        for x, heads, w, what in ((qc, c.H, wq, "q"), (kc, c.H_kv, wk, "k")):
            y, size = ref.head(x[r0:r1].view(r1 - r0, heads, c.d_h), w if norm else None, eps, table, pos, pairs)
            # one rounding to the type; in fp32 a sum of d_h squares (its relative error is halved by the root), root, quotient, two
            # factors, the table's cosines and sines, the products and their sum: (d_h / 2 + 8) half steps of what goes into a column
            room = half * y.abs() + (c.d_h / 2 + 8) * 2.0 ** -24 * size * (1 + half)
            if what == "q":
                if with_q:
                    got = out[r0:r1].cpu().view(r1 - r0, heads, c.d_h)
                    assert bool(((got.double() - y).abs() <= room).all()), "q of sequence %d" % b
                continue
            for i in range(r1 - r0):
                p = c.past[b] + i
                at, slot = int(c.table[b, p // c.page]), p % c.page
                assert bool(((K[at, :, slot].double() - y[i]).abs() <= room[i]).all()), "key %d of sequence %d" % (i, b)
                want_K[at, :, slot] = K[at, :, slot]
                want_V[at, :, slot] = vc[r0 + i].view(c.H_kv, c.d_h)
        # bounds are those of the keys that are there, to the bit
        for j in range(-(-c.total[b] // c.page)):
            at, n = int(c.table[b, j]), min(c.page, c.total[b] - j * c.page)
            keys = K[at, :, :n]
            if (j + 1) * c.page > c.past[b] and r1 > r0:
                assert torch.equal(bounds[at, :, 0], keys.amin(1)) and torch.equal(bounds[at, :, 1], keys.amax(1)), "bounds of page %d" % j
            else:
                assert torch.equal(bounds[at], before_bounds[at])
    same = lambda x, y: torch.equal(torch.nan_to_num(x, nan=123.0), torch.nan_to_num(y, nan=123.0))  # noqa: E731
    assert same(V, want_V) and same(K, want_K), "slots of nobody's"
    if with_q:
        assert bool((out[int(c.start[-1]):] == 7.0).all())


def test_append_in_place_and_of_one_row(pa):
    c = ref.Case("bf16", 4, 2, 128, 16, [1], [5])
    cache, chunk = c.on_gpu(pa)
    qkv, (wq, wk) = rows_in(c)
    table = ref.rope_table(6, 128).cuda()
    q, k, v = (x.cuda() for x in qkv.split((512, 256, 256), dim=1))
    apart = pa.ada_cache_append(cache, chunk, q, k, v, rope=table, q_norm=wq.cuda(), k_norm=wk.cuda())["q"]
    inside = pa.ada_cache_append(cache, chunk, q, k, v, rope=table, q_norm=wq.cuda(), k_norm=wk.cuda(), out=q)["q"]
    assert inside is q and torch.equal(apart, inside)


def test_append_refuses_pages_and_positions(pa):
    c = ref.Case("bf16", 2, 2, 64, 16, [2, 2, 1], [15, 3, 40])
    c.table[0, 1] = c.pages + 5
    cache, chunk = c.on_gpu(pa)
    before = [cache.K.clone(), cache.V.clone(), cache.bounds.clone()]
    qkv, _ = rows_in(c)
    q, k, v = (x.contiguous() for x in qkv.cuda().split((128, 128, 128), dim=1))
    res = pa.ada_cache_append(cache, chunk, q, k, v, rope=ref.rope_table(40, 64).cuda())
    assert res["status"].item() == INDEX
    differ = lambda x, y: (torch.nan_to_num(x, nan=9.0) != torch.nan_to_num(y, nan=9.0)).any(3)  # noqa: E731
    for x, y in zip((cache.K, cache.V), before):
        changed = differ(x, y).any(1).nonzero().tolist()
        assert sorted(changed) == sorted([int(c.table[0, 0]), 15] if p == 15 else [int(c.table[1, 0]), p] for p in (15, 3, 4))
    widened = set(differ(cache.bounds, before[2]).any(2).any(1).nonzero().flatten().tolist())
    assert widened == {int(c.table[0, 0]), int(c.table[1, 0])}


# ------------------------------------------------------------------------------------------------ selection
SELECT = {
    "tokens": (lambda: ref.Case("bf16", 8, 2, 128, 16, [1, 1, 1], [600, 100, 3]), 8, 1, 1),
    "tokens_group_7": (lambda: ref.Case("bf16", 14, 2, 64, 32, [1, 1], [1500, 640]), 5, 1, 2),
    "tokens_group_20": (lambda: ref.Case("bf16", 20, 1, 64, 16, [1], [900]), 6, 0, 1),
    "tokens_256": (lambda: ref.Case("bf16", 4, 4, 256, 64, [1, 1], [2000, 64]), 4, 1, 1),
    "tokens_f32": (lambda: ref.Case("f32", 6, 2, 64, 16, [1, 1], [500, 321]), 7, 2, 0),
    "chunk": (lambda: ref.Case("bf16", 8, 2, 128, 16, [50], [300]), 6, 1, 1),
    "chunk_mixed": (lambda: ref.Case("bf16", 12, 4, 64, 32, [1, 0, 40, 3], [700, 4, 0, 250], pad_rows=3), 4, 0, 0),
    "chunk_f32": (lambda: ref.Case("f32", 3, 1, 128, 16, [37, 5], [64, 200]), 5, 1, 1),
    "group_24": (lambda: ref.Case("f32", 24, 1, 64, 16, [9], [200]), 3, 1, 1),
    "all_of_them": (lambda: ref.Case("bf16", 2, 1, 64, 16, [20], [100]), 64, 1, 1),
    "one_page": (lambda: ref.Case("bf16", 4, 2, 128, 64, [3, 1], [500, 900]), 1, 0, 1),
    "only_forced": (lambda: ref.Case("bf16", 4, 2, 64, 16, [6], [400]), 4, 2, 2),
    "long_chunk": (lambda: ref.Case("bf16", 6, 2, 64, 16, [70, 33], [3000, 100]), 12, 1, 1),
    "many_pages": (lambda: ref.Case("bf16", 2, 1, 64, 16, [1], [20000]), 40, 1, 1),
}


def check_lists(c, res, budget, want):
    pages, counts = res["pages"].cpu(), res["counts"].cpu()
    for row, mine in enumerate(want):
        for kv in range(c.H_kv):
            if mine is None:
                continue
            n = int(counts[row, kv])
            got = pages[row, kv].tolist()
            assert got[:n] == mine[kv] and got[n:] == [-1] * (budget - n), "row %d, head %d" % (row, kv)


@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("name", SELECT)
def test_select(pa, name, causal):
    make, budget, first, last = SELECT[name]
    c = make()
    cache, chunk = c.on_gpu(pa)
    out = dict(pages=torch.full((c.rows, c.H_kv, budget), 77, dtype=torch.int32, device="cuda"),
               counts=torch.full((c.rows, c.H_kv), 77, dtype=torch.int32, device="cuda"))
    res = pa.ada_select_pages(cache, chunk, c.Q.cuda(), budget, first=first, last=last, out=out, flags=pa.FLAG_ATTN_CAUSAL if causal else 0)
    assert res["status"].item() == OK
    check_lists(c, res, budget, ref.select(c, budget, first, last, causal))
    n = int(c.start[-1])
    assert bool((out["pages"][n:] == 77).all()) and bool((out["counts"][n:] == 77).all())


def test_select_ties_and_near_ties(pa):
    """Pages alike to the bit, scores that differ in fp32's last places only, and queries of zeros: as in float64, ties to the smaller page."""
    for kind, past in [(k, 700) for k in ("alike", "near", "zero", "f32")] + [("alike", 1700), ("zero", 1700), ("near", 10000), ("zero", 10000)]:
        c = ref.Case("f32" if kind == "f32" else "bf16", 4, 2, 128, 16, [3, 1] if past < 9000 else [1], [past, 500] if past < 9000 else [past])
        g = torch.Generator().manual_seed(5)
        if kind == "alike":
            c.bounds[:] = c.bounds[int(c.table[0, 0])].clone()
        elif kind in ("near", "f32"):
            base = 30 * torch.randn(1, c.H_kv, 2, c.d_h, generator=g)
            wiggle = torch.randn(c.pages, c.H_kv, 2, c.d_h, generator=g) * (2.0 ** -21 if kind == "f32" else 1e-4)
            b = base.to(c.dtype) + torch.where(torch.arange(c.d_h) < 2, wiggle, torch.zeros(1)).to(c.dtype)
            b[..., :2] = (base[..., :2] * 0 + wiggle[..., :2] if kind == "near" else (base + wiggle)[..., :2]).to(c.dtype)
            c.bounds = torch.stack((b.amin(2), b.amax(2)), dim=2).to(c.dtype)
        else:
            c.Q.zero_()
        cache, chunk = c.on_gpu(pa)
        for budget in (1, 5, 20):
            res = pa.ada_select_pages(cache, chunk, c.Q.cuda(), budget, first=0, last=1, flags=pa.FLAG_ATTN_CAUSAL)
            check_lists(c, res, budget, ref.select(c, budget, 0, 1, True))


def test_select_leaves_out_pages_that_are_not_there(pa):
    c = ref.Case("bf16", 4, 2, 64, 16, [2], [300])
    c.table[0, 0], c.table[0, 7] = -1, c.pages
    bad = ((0, 0), (0, 7))
    c2 = ref.Case("bf16", 4, 2, 64, 16, [2], [300])        # bounds of the pages as they were
    cache, chunk = c.on_gpu(pa)
    res = pa.ada_select_pages(cache, chunk, c.Q.cuda(), 17, flags=pa.FLAG_ATTN_CAUSAL)
    assert res["status"].item() == INDEX
    check_lists(c, res, 17, ref.select(c2, 17, 1, 1, True, bad))


# ------------------------------------------------------------------------------------------------ attention over listed pages
PAGES = {
    "tokens": (lambda: ref.Case("bf16", 8, 2, 128, 16, [1, 1, 1], [600, 100, 3]), 8),
    "tokens_64": (lambda: ref.Case("bf16", 8, 1, 64, 64, [1, 1], [2000, 640]), 9),
    "tokens_256": (lambda: ref.Case("bf16", 4, 4, 256, 32, [1, 1], [1000, 31]), 4),
    "tokens_group_20": (lambda: ref.Case("bf16", 40, 2, 64, 16, [1], [333]), 5),
    "tokens_f32": (lambda: ref.Case("f32", 6, 2, 64, 16, [1, 1], [500, 321]), 7),
    "chunk": (lambda: ref.Case("bf16", 8, 2, 128, 64, [50, 1], [300, 900], order="slots", pad_rows=2), 4),
    "chunk_f32": (lambda: ref.Case("f32", 2, 2, 128, 128, [20], [700]), 3),
}


def some_lists(c, budget, causal):
    """Any ascending pages that a row can see, its own among them; every third row has none."""
    g = torch.Generator().manual_seed(3)
    pages, counts = torch.full((c.rows, c.H_kv, budget), 1 << 29, dtype=torch.int32), torch.zeros(c.rows, c.H_kv, dtype=torch.int32)
    lists = [[[] for _ in range(c.H_kv)] for _ in range(c.rows)]
    for b in range(c.B):
        for row in range(*c.rows_of(b)):
            have = (c.past[b] + row - c.rows_of(b)[0] if causal else c.total[b] - 1) // c.page + 1
            for kv in range(c.H_kv):
                if (row + kv) % 3 == 2:
                    continue
                some = sorted(set(torch.randperm(have, generator=g)[:budget - 1].tolist()) | {have - 1})
                lists[row][kv] = some
                pages[row, kv, :len(some)] = torch.tensor(some, dtype=torch.int32)
                counts[row, kv] = len(some)
    return lists, pages.cuda(), counts.cuda()


@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("name", PAGES)
def test_attention_pages(pa, name, causal):
    make, budget = PAGES[name]
    c = make()
    cache, chunk = c.on_gpu(pa)
    lists, pages, counts = some_lists(c, budget, causal)
    out = torch.full((c.rows, c.H * c.d_h), 7.0, dtype=c.dtype, device="cuda")
    res = pa.ada_attention_pages(cache, chunk, c.Q.cuda(), pages, counts, out=out, flags=pa.FLAG_ATTN_CAUSAL if causal else 0)
    assert res["status"].item() == OK
    check_attend(c, out, causal, lists)
    n = int(c.start[-1])
    assert bool((out[n:] == 7.0).all())
    for row in range(n):
        for kv in range(c.H_kv):
            if not lists[row][kv]:
                assert bool((out[row].view(c.H, c.d_h)[kv * c.G:(kv + 1) * c.G] == 0).all()), "a row that sees nothing"


def test_lists_that_name_no_page(pa):
    c = ref.Case("bf16", 4, 1, 64, 16, [1, 1, 1, 1], [100, 100, 100, 100])
    cache, chunk = c.on_gpu(pa)
    given = [[0, 3, 3, 5], [2, 1, 4, 6], [-1, 2, 900, 3], [0, 1, 2, 6]]
    taken = [[0, 3, 5], [2, 4, 6], [2], [0, 1, 2, 6]]      # not larger than the one in front, or out of range: masked
    for row, (g, t) in enumerate(zip(given, taken)):
        pages = torch.tensor(given, dtype=torch.int32, device="cuda")[:, None].contiguous()
        counts = torch.full((4, 1), 4, dtype=torch.int32, device="cuda")
        res = pa.ada_attention_pages(cache, chunk, c.Q.cuda(), pages, counts, flags=pa.FLAG_ATTN_CAUSAL)
        assert res["status"].item() == INDEX
    check_attend(c, res["out"], True, [[t] for t in taken])


# ------------------------------------------------------------------------------------------------ together
def test_prompt_and_steps_together(pa):
    """Two sequences: a prompt in two chunks, then single tokens, appended, selected and attended to as a program does, on a stream of its own;
    lists with room for all pages give what attention over everything gives."""
    c = ref.Case("bf16", 8, 2, 128, 16, [60, 90], [0, 0], spare_columns=2)
    for b, n in enumerate((70, 100)):                      # room for ten more
        used = set(c.table[c.table >= 0].tolist())
        need = -(-n // c.page)
        free = [p for p in range(c.pages) if p not in used]
        have = -(-c.total[b] // c.page)
        c.table[b, have:need] = torch.tensor(free[:need - have], dtype=torch.int32)
    c.K, c.V, c.bounds = c.pool()
    g = torch.Generator().manual_seed(11)
    total = [70, 100]
    raw = [torch.randn(t, (c.H + 2 * c.H_kv) * c.d_h, generator=g).to(c.dtype) for t in total]
    wq, wk = [(1 + 0.2 * torch.randn(c.d_h, generator=g)).to(c.dtype) for _ in range(2)]
    table = ref.rope_table(max(total), 128)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        cache = pa.PagedCache(c.K.cuda(), c.V.cuda(), c.bounds.cuda())
        tab, rope, wq_, wk_ = c.table.cuda(), table.cuda(), wq.cuda(), wk.cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        past, outs = [0, 0], [[], []]
        for new in ([40, 90], [20, 0]) + ([1, 1],) * 10:
            start = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
            chunk = pa.Chunk(tab, start, torch.tensor(past, dtype=torch.int32, device="cuda"), rows=sum(new), longest=max(new))
            x = torch.cat([raw[b][past[b]:past[b] + new[b]] for b in range(2)]).cuda()
            q, k, v = x.split((c.H * c.d_h, c.H_kv * c.d_h, c.H_kv * c.d_h), dim=1)
            q = pa.ada_cache_append(cache, chunk, q, k, v, rope=rope, q_norm=wq_, k_norm=wk_, status=status)["q"]
            full = pa.ada_attention_paged(cache, chunk, q, status=status, flags=pa.FLAG_ATTN_CAUSAL)["out"]
            chosen = pa.ada_select_pages(cache, chunk, q, 12, status=status, flags=pa.FLAG_ATTN_CAUSAL)
            listed = pa.ada_attention_pages(cache, chunk, q, chosen["pages"], chosen["counts"], status=status, flags=pa.FLAG_ATTN_CAUSAL)["out"]
            for b in range(2):
                rows = slice(0, new[0]) if b == 0 else slice(new[0], sum(new))
                outs[b].append((full[rows], listed[rows], q[rows]))
                past[b] += new[b]
    stream.synchronize()
    assert status.item() == OK
    whole = ref.Case("bf16", 8, 2, 128, 16, total, [0, 0])
    kv = cache.K.cpu(), cache.V.cpu()
    for b in range(2):
        where = [(int(c.table[b, p // 16]), p % 16) for p in range(total[b])]
        whole.k[b] = torch.stack([kv[0][at, :, s] for at, s in where])
        whole.v[b] = torch.stack([kv[1][at, :, s] for at, s in where])
        y, size = ref.head(raw[b][:, c.H * c.d_h:(c.H + c.H_kv) * c.d_h].reshape(total[b], c.H_kv, c.d_h), wk, 1e-6, table, torch.arange(total[b]), False)
        assert bool(((whole.k[b].double() - y).abs() <= 2.0 ** -8 * y.abs() + 80 * 2.0 ** -24 * size).all())
        whole.Q[whole.rows_of(b)[0]:whole.rows_of(b)[1]] = torch.cat([o[2] for o in outs[b]]).cpu()
    for i in (0, 1):
        check_attend(whole, torch.cat([o[i] for o in outs[0]] + [o[i] for o in outs[1]]), True)


def test_steps_in_graphs_that_share_a_workspace(pa):
    """One captured step serves every later one: lengths are on the device.  Two graphs with the same workspace, replayed in turns between
    eager calls."""
    c = ref.Case("bf16", 8, 2, 128, 16, [1, 1, 1], [0, 30, 200], spare_columns=2)
    cache, chunk = c.on_gpu(pa)
    tables = chunk.table
    qkv = torch.randn(c.rows, (c.H + 2 * c.H_kv) * c.d_h, generator=torch.Generator().manual_seed(2)).to(c.dtype).cuda()
    q, k, v = qkv.split((c.H * c.d_h, c.H_kv * c.d_h, c.H_kv * c.d_h), dim=1)
    rope = ref.rope_table(256, 128).cuda()
    ws, status = pa.paged_workspace(cache, chunk, c.H), torch.zeros(1, dtype=torch.int32, device="cuda")
    qo, out = torch.zeros(c.rows, c.H * c.d_h, dtype=c.dtype, device="cuda"), torch.zeros(c.rows, c.H * c.d_h, dtype=c.dtype, device="cuda")
    lists = dict(pages=torch.zeros(c.rows, c.H_kv, 4, dtype=torch.int32, device="cuda"), counts=torch.zeros(c.rows, c.H_kv, dtype=torch.int32, device="cuda"))
    out2 = torch.zeros_like(out)

    def step():
        pa.ada_cache_append(cache, chunk, q, k, v, rope=rope, out=qo, status=status)
        pa.ada_attention_paged(cache, chunk, qo, ws=ws, out=out, status=status, flags=pa.FLAG_ATTN_CAUSAL)

    def step_listed():
        pa.ada_select_pages(cache, chunk, qo, 4, out=lists, status=status, flags=pa.FLAG_ATTN_CAUSAL)
        pa.ada_attention_pages(cache, chunk, qo, lists["pages"], lists["counts"], ws=ws, out=out2, status=status, flags=pa.FLAG_ATTN_CAUSAL)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        step_listed()
    torch.cuda.current_stream().wait_stream(stream)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, f in zip(graphs, (step, step_listed)):
        with torch.cuda.graph(graph, stream=stream):
            f()
    for turn in range(4):
        chunk.past.copy_(torch.tensor([0 + turn, 12 + turn, 200 - turn], dtype=torch.int32))
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(50 + turn)))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (qo, out, lists["pages"], out2)]
        for x in (qo, out, out2):
            x.fill_(7.0)
        step()
        step_listed()
        torch.cuda.synchronize()
        for x, y in zip(got, (qo, out, lists["pages"], out2)):
            assert torch.equal(x, y), "replay %d" % turn
    assert status.item() == OK


def test_two_calls_at_once(pa):
    """Two streams, a workspace each."""
    cases = [ref.Case("bf16", 8, 2, 128, 16, [1] * 6, [900, 10, 300, 77, 1024, 0], seed=1), ref.Case("bf16", 4, 4, 64, 64, [130], [500], seed=2)]
    streams, got = [torch.cuda.Stream() for _ in cases], []
    on = [c.on_gpu(pa) for c in cases]
    qs = [c.Q.cuda() for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for (cache, chunk), q, st in zip(on, qs, streams):
            with torch.cuda.stream(st):
                got.append(pa.ada_attention_paged(cache, chunk, q, flags=pa.FLAG_ATTN_CAUSAL))
        torch.cuda.synchronize()
    for c, r in zip(cases, got):
        check_attend(c, r["out"], True)


def test_calls_on_a_given_stream_make_what_they_need_on_it(pa):
    """The current stream is busy and its memory was used before: status, workspace and outputs of calls on another stream do not wait for it."""
    c = ref.Case("bf16", 8, 2, 128, 32, [1] * 4, [900, 10, 300, 1024], seed=3)
    cache, chunk = c.on_gpu(pa)
    q, side, busy = c.Q.cuda(), torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    want = pa.ada_select_pages(cache, chunk, q, 4)
    want = [want["pages"].clone(), want["counts"].clone(), pa.ada_attention_pages(cache, chunk, q, want["pages"], want["counts"])["out"].clone()]
    n = pa.ada_paged_workspace_bytes(cache, chunk, c.H)
    used = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    del used
    for _ in range(20):
        busy = busy @ busy * 1e-3
    sel = pa.ada_select_pages(cache, chunk, q, 4, stream=side)
    res = pa.ada_attention_pages(cache, chunk, q, sel["pages"], sel["counts"], stream=side)
    full = pa.ada_attention_paged(cache, chunk, q, stream=side)
    side.synchronize()
    assert [r["status"].item() for r in (sel, res, full)] == [OK] * 3
    for a, b in zip(want, (sel["pages"], sel["counts"], res["out"])):
        assert torch.equal(a, b)
    check_attend(c, full["out"], False)
    torch.cuda.synchronize()


def test_offsets_past_32_bits(pa):
    """Pages far into a pool whose elements need more than 32 bits to count."""
    pages, page, d_h = 70000, 256, 128
    K = torch.empty(pages, 1, page, d_h, dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    assert K.numel() > 1 << 31
    c = ref.Case("bf16", 2, 1, d_h, page, [3, 1], [500, 300])
    far = {int(p): pages - 1 - 17 * i for i, p in enumerate(sorted(set(c.table[c.table >= 0].tolist())))}
    cache, chunk = c.on_gpu(pa)
    for old, new in far.items():
        K[new], V[new] = cache.K[old], cache.V[old]
        chunk.table[chunk.table == old] = -100 - new
    chunk.table.copy_(torch.where(chunk.table <= -100, -100 - chunk.table, chunk.table))
    res = pa.ada_attention_paged(pa.PagedCache(K, V), chunk, c.Q.cuda(), flags=pa.FLAG_ATTN_CAUSAL)
    assert res["status"].item() == OK
    check_attend(c, res["out"], True)


def test_no_rows(pa):
    c = ref.Case("bf16", 2, 1, 64, 16, [0, 0], [5, 0])
    cache, _ = c.on_gpu(pa)
    chunk = pa.Chunk(c.table.cuda(), c.start.cuda(), c.past_t.cuda(), rows=0)
    ws = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
    some = torch.zeros(1, 128, dtype=torch.bfloat16, device="cuda")
    assert pa.ada_attention_paged(cache, chunk, some, ws=ws)["status"].item() == OK
    chunk = pa.Chunk(c.table.cuda(), c.start.cuda(), c.past_t.cuda(), rows=1)      # one row, nobody's
    out = torch.full((1, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    assert pa.ada_attention_paged(cache, chunk, some, out=out)["status"].item() == OK
    assert bool((out == 7.0).all())


def test_append_of_a_large_chunk(pa):
    """17000 tokens at once and in pieces of 5000 that end inside pages: the same to the bit."""
    H, H_kv, d_h, page, n = 32, 8, 128, 64, 17000
    rows, heads = torch.arange(n, device="cuda"), H + 2 * H_kv
    gen = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn(n, heads * d_h, generator=gen, device="cuda").bfloat16()
    rope = ref.rope_table(n, d_h).cuda()
    w = (1 + 0.2 * torch.randn(d_h, generator=gen, device="cuda")).bfloat16()
    pages = -(-n // page)
    table = torch.randperm(pages, generator=gen, device="cuda").int()[None].contiguous()
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    got = []
    for step in (n, 5000):
        K = torch.zeros(pages, H_kv, page, d_h, dtype=torch.bfloat16, device="cuda")
        cache = pa.PagedCache(K, torch.zeros_like(K), torch.zeros(pages, H_kv, 2, d_h, dtype=torch.bfloat16, device="cuda"))
        qs = []
        for lo in range(0, n, step):
            hi = min(lo + step, n)
            q, k, v = qkv[lo:hi].split((H * d_h, H_kv * d_h, H_kv * d_h), dim=1)
            res = pa.ada_cache_append(cache, pa.Chunk(table, ints(0, hi - lo), ints(lo), rows=hi - lo), q, k, v, rope=rope, q_norm=w, k_norm=w)
            assert res["status"].item() == OK
            qs.append(res["q"])
        got.append((torch.cat(qs), cache.K, cache.V, cache.bounds))
    for x, y in zip(*got):
        assert torch.equal(x, y)
    assert torch.equal(got[0][2][table[0, rows // page].long(), :, rows % page], qkv[:, -H_kv * d_h:].view(n, H_kv, d_h))
