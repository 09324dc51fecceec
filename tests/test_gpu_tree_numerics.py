"""Drafted trees where the other tests' tolerances say little: logits of any size, weights in as many bits as a decode step holds them
in, every row of a unit counted once, and node rows of any alignment in an accepted path."""
import numpy as np
import pytest
import torch

from tests import serving_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tb():
    import paper_2512_09238_amd.binding as tb
    return tb


@pytest.fixture(scope="module")
def bufs():
    import paper_2512_09238_amd.buffers as bufs
    return bufs


def shape(hq, hkv, d, b, w, rows, share=False):
    return dict(hq=hq, hkv=hkv, d=d, b=b, w=w, rows=rows, share=share)


def attend(tb, bufs, prm, c, q, k, v, parent, ws_bytes=None):
    n = q.shape[1]
    ws = bufs.workspace(ws_bytes or tb.tca_decode_tree_workspace_bytes(prm, c.batch, n, c.max_head_rows))
    O = torch.full_like(q, 7.0)
    tb.tca_decode_tree(prm, c.view, c.offs, n, parent, q, k, v, O, ws)
    torch.cuda.synchronize()
    return O


def forked(n):
    """Two chains from one node."""
    return [-1] + [i - 1 if i < n // 2 else 0 if i == n // 2 else i - 1 for i in range(1, n)]


# ---------------------------------------------------------------------------------------------- logits of any size --
def ties_far_above(tb, bufs, case, lengths, n, size, seed):
    """Every query is `size` times its KV head's own direction and a little else, and so are some K rows of every kind (the direction,
    that is): in a region, at its window's edge, in the ring, among the nodes.  Their logits tie, far above all others: a query's result
    is the mean of those rows' V."""
    prm, c = R.filled_cache(tb, bufs, case, lengths, seed, fill=0.6)
    q, k, v, parent = R.draft(case, len(lengths), n, seed + 1, [forked(n)] * len(lengths))
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    G = case["hq"] // case["hkv"]
    to = torch.randn(case["hkv"], case["d"], generator=g, device="cuda").sign()          # +-1, so that products and sums are exact
    some = 1.0 + torch.randint(0, 8, q.shape[:3], generator=g, device="cuda")[..., None] / 8.0
    q = (size * some * to.repeat_interleave(G, 0)).to(q.dtype)
    k[:, ::3] = to.to(k.dtype)
    # (as a row of the nodes is stored: amax / 448 and the codes of 448)
    row = (448 * to).to(torch.float8_e4m3fn).view(torch.uint8) if case["rows"] == "fp8" else to.to(k.dtype)
    scale = 1.0 / np.float32(448.0)
    Hs, w = c.n_rows.shape[1], case["w"]
    for s, T in enumerate(lengths):
        for hs in range(Hs):
            o, rows, kv = int(c.offs[hs]), int(c.n_rows[s, hs]), hs // (Hs // case["hkv"])
            seen = int((c.idx[s, o:o + rows] <= T - w).sum())
            at = torch.tensor([o + r for r in (0, rows // 3, seen - 1, seen, rows - 1) if 0 <= r < rows], dtype=torch.long, device="cuda")
            c.Kg[s, at] = row[kv]
            if case["rows"] == "fp8":
                c.Kg_scale[s, at] = float(scale)
        for pos in (T - 1, T - 7, T - w + 1, T - w + 3):
            if 0 <= pos:
                c.ringK[s, :, pos % w] = row
                if case["rows"] == "fp8":
                    c.ringK_scale[s, :, pos % w] = float(scale)
    return prm, c, q, k, v, parent


# size times sqrt(d) log2 e in the middle: 2^24.5 .. 2^38, where neighbours in fp32 are 2 to 16384 apart, and a size of no trouble
@pytest.mark.parametrize("size", [1.0, 2.0 ** 21, 2.0 ** 27, 2.0 ** 29, 2.0 ** 31, 2.0 ** 34])
@pytest.mark.parametrize("rows,d,share", [("f32", 128, False), ("f32", 64, True), ("bf16", 128, False), ("bf16", 64, True), ("fp8", 128, True),
                                          ("fp8", 64, False)])
def test_logits_of_any_size(tb, bufs, rows, d, share, size):
    case = shape(8, 2, d, 16, 160, rows, share)
    prm, c, q, k, v, parent = ties_far_above(tb, bufs, case, (2600, 300, 31), 11, size, 700)
    want, tol = R.tree_reference(case, c, q, k, v, parent)
    O = attend(tb, bufs, prm, c, q, k, v, parent).double().cpu().numpy()
    assert not np.isnan(want).any()
    if size > 1.0:
        # Rows that tie have the same products in the same order, here and there, so that their logits are equal whatever their errors;
        # all others are 10^6 and more below.  What is left of the tolerance is the weights' rounding, the sums' and the result's: of
        # fewer than 64 terms, as in `tol` without its logits.
        half = 0.0 if rows == "f32" else 2.0 ** -8
        values = [R.read_back(c, x, s) for s in range(3) for x in ("Vg", "ringV")] + [R.stored(case, v)]
        largest = max(np.abs(x).max() for x in values)
        tol = half * np.abs(want) + (half + 2 * 72 * 2.0 ** -24) * largest
    off = np.abs(O - want) / tol
    print("worst error over tolerance %.3f" % off.max(), flush=True)
    assert off.max() <= 1.0


# ------------------------------------------------------------------------------------------------- bits of weights --
def visible(case, c, q, k, v, parent):
    """Per node and head: (sequence, node, head), the weights of the rows that it sees and these rows of V in float64, and how far fp32
    logits may be off (a sum of d products: d 2^-24 of its terms' magnitudes; fp32 rows have fp64 logits)."""
    B, n, Hq, d = q.shape
    Hs, Hkv, w = c.n_rows.shape[1], case["hkv"], case["w"]
    qf, kf, vf, par = q.double().cpu().numpy(), R.stored(case, k), R.stored(case, v), parent.cpu().numpy()
    for s in range(B):
        T, idx = int(c.length[s]), c.idx[s].cpu().numpy()
        Kg, Vg, rK, rV = (R.read_back(c, x, s) for x in ("Kg", "Vg", "ringK", "ringV"))
        for i in range(n):
            line = R.line_to(par[s], i)
            P = T + len(line) - 1
            old = np.arange(max(0, P - w + 1), T) % w
            for h in range(Hq):
                hs, kv = h // (Hq // Hs), h // (Hq // Hkv)
                o = int(c.offs[hs])
                at = o + np.nonzero(idx[o:o + int(c.n_rows[s, hs])] <= P - w)[0]
                keys = np.concatenate([Kg[at], rK[kv, old], kf[s, line, kv]])
                x = keys @ qf[s, i, h] / np.sqrt(d)
                e = np.exp(x - x.max())
                off = d * 2.0 ** -24 * (np.abs(keys) @ np.abs(qf[s, i, h])).max() / np.sqrt(d)
                yield (s, i, h), e / e.sum(), np.concatenate([Vg[at], rV[kv, old], vf[s, line, kv]]), 0.0 if case["rows"] == "f32" else off


def sharp(case, c, q, k, v, parent):
    """(O, tolerance) in float64 where a weight is held in 16 bits or more (off by 2^-17 of itself): numerator and denominator twice the
    logits' error, sums of N terms in fp32 and exponentials (8 times 2^-24), and the result's rounding."""
    O, tol = np.empty(q.shape), np.empty(q.shape)
    half = 2.0 ** -24 if case["rows"] == "f32" else 2.0 ** -8
    for at, p, vals, off in visible(case, c, q, k, v, parent):
        O[at] = p @ vals
        tol[at] = half * np.abs(O[at]) + (2.0 ** -17 + 2 * off + 2 * (len(p) + 8) * 2.0 ** -24) * (p @ np.abs(vals))
    return O, tol


@pytest.mark.parametrize("rows,d,share,n", [("bf16", 128, False, 1), ("bf16", 64, True, 9), ("bf16", 64, False, 40), ("bf16", 128, True, 20),
                                            ("bf16", 64, True, 64), ("fp8", 128, False, 1), ("fp8", 64, True, 9), ("fp8", 64, False, 40),
                                            ("fp8", 128, True, 20), ("fp8", 64, True, 64), ("f32", 64, False, 9)])
def test_weights_have_the_bits_of_a_decode_step(tb, bufs, rows, d, share, n):
    """Elements that are near zero, where the terms cancel, show the weights' error bare of the result's rounding."""
    case = shape(8, 2, d, 16, 160, rows, share)
    prm, c = R.filled_cache(tb, bufs, case, (500, 170, 0), 721)
    q, k, v, parent = R.draft(case, 3, n, 722, [forked(n)] * 3)
    q = (q.float() / 3).to(q.dtype)
    want, tol = sharp(case, c, q, k, v, parent)
    O = attend(tb, bufs, prm, c, q, k, v, parent).double().cpu().numpy()
    off = np.abs(O - want) / tol
    print("worst error over tolerance %.3f" % off.max(), flush=True)
    assert off.max() <= 1.0


@pytest.mark.parametrize("rows,share", [("bf16", False), ("bf16", True), ("fp8", False), ("fp8", True), ("f32", False)])
def test_a_tree_of_one_node_is_as_exact_as_a_decode_step(tb, bufs, rows, share):
    case = shape(8, 2, 128, 16, 160, rows, share)
    prm, c = R.filled_cache(tb, bufs, case, (900, 333), 731)
    q, k, v, parent = R.draft(case, 2, 1, 732, [[-1]] * 2)
    want, tol = sharp(case, c, q, k, v, parent)
    O = attend(tb, bufs, prm, c, q, k, v, parent)
    P = np.stack([tb.tca_config_from_budget(16, 1.0, 0.4)] * tb.tca_selection_heads(prm))
    Od = torch.empty_like(q[:, 0])
    tb.tca_decode(prm, c.view, c.offs, q[:, 0].contiguous(), k[:, 0].contiguous(), v[:, 0].contiguous(), P, Od,
                  bufs.workspace(tb.tca_decode_workspace_bytes(prm, 2, c.max_head_rows)))
    torch.cuda.synchronize()
    for name, x in (("tree", O[:, 0]), ("decode", Od)):
        off = np.abs(x.double().cpu().numpy() - want[:, 0]) / tol[:, 0]
        print("%s: worst error over tolerance %.3f" % (name, off.max()), flush=True)
        assert off.max() <= 1.0


# ------------------------------------------------------------------------------------------------ every row once --
EVERY = [
    # shape, lengths, nodes, rows kept: chunks of every length, windows and regions that end inside tiles and chunks
    (shape(4, 2, 128, 16, 160, "bf16"), (5000, 1999, 161), 9, 0.5),
    (shape(4, 1, 64, 16, 640, "bf16"), (640, 700, 1279, 639, 120, 2000), 40, 0.5),
    (shape(8, 1, 128, 16, 384, "bf16", True), (2500, 385), 33, 0.6),
    (shape(2, 1, 64, 16, 64, "bf16"), (21000,), 5, 0.6),
    (shape(4, 2, 128, 16, 160, "fp8"), (5000, 1999, 161), 9, 0.5),
    (shape(8, 1, 64, 16, 640, "fp8", True), (640, 1279, 639, 2000), 40, 0.5),
    (shape(4, 2, 128, 16, 160, "f32"), (2600, 161), 9, 0.6),
    (shape(4, 1, 64, 16, 640, "f32"), (640, 1279, 639, 2000), 24, 0.5),
    (shape(2, 1, 64, 16, 64, "f32"), (13000,), 5, 0.6),
]


@pytest.mark.parametrize("i", range(len(EVERY)))
def test_every_row_counts_once(tb, bufs, i):
    """Nearly even weights, and V rows that are columns of a unit matrix (in long regions those next to a chunk's end, the others zero):
    an element of the result is the sum of the weights of its column's rows, of which one too many or too few is more than the tolerance."""
    case, lengths, n, fill = EVERY[i]
    print("case", EVERY[i], flush=True)
    d, w, fp8 = case["d"], case["w"], case["rows"] == "fp8"
    prm, c = R.filled_cache(tb, bufs, case, lengths, 740 + i, room=37 * (i % 3), fill=fill)
    if fp8:                                                              # K between 1/8 and 2, scales of 1
        g = torch.Generator(device="cuda").manual_seed(i)
        for t in (c.Kg, c.ringK):
            t.copy_(torch.randint(0x20, 0x40, t.shape, device="cuda", generator=g))
        for t in (c.Kg_scale, c.Vg_scale, c.ringK_scale, c.ringV_scale):
            t.fill_(1.0)
    q, k, v, parent = R.draft(case, len(lengths), n, 750 + i, [forked(n)] * len(lengths))
    q = (q.float() / (32 * d ** 0.5)).to(q.dtype)
    # a region's row r, counted from its head's first, and the ring's slot r in column r mod d; node r in column - r - 1
    in_head = torch.cat([torch.arange(int(r), device="cuda") for r in np.diff(c.offs)])
    far = (in_head + 24) % 4096 > 48 if max(lengths) > 10000 else torch.zeros_like(in_head, dtype=torch.bool)
    for s, T in enumerate(lengths):
        for h in range(c.n_rows.shape[1]):                               # the rows around the window's edge and the last ones
            o, rows = int(c.offs[h]), int(c.n_rows[s, h])
            edge = int((c.idx[s, o:o + rows] <= T - w).sum())
            far[o + max(0, edge - 24):o + rows] = False
    for t in (c.Vg, c.ringV):
        at = in_head if t is c.Vg else torch.arange(w, device="cuda")
        t.zero_()
        t.scatter_(-1, (at % d).expand(t.shape[:-1])[..., None], 0x38 if fp8 else 1.0)              # (E4M3: 0x38 is 1)
    c.Vg[:, :len(far)][:, far] = 0
    v.zero_()
    v.scatter_(-1, (d - 1 - torch.arange(n, device="cuda"))[None, :, None, None].expand(*v.shape[:3], 1), 1.0)
    want, lightest = np.empty(q.shape), 1.0
    for at, p, vals, _ in visible(case, c, q, k, v, parent):
        want[at] = p @ vals
        one = vals.any(1)
        lightest = min(lightest, ((p * vals.max(1))[one] / want[at][vals.argmax(1)[one]]).min())
    # A sum of weights, none negative: off by 2^-17 of itself for theirs, by their sums' roundings (numerator and denominator), by twice
    # the logits' error (they are below 1/4, and so is the sum of their terms' magnitudes over 4: d 2^-24), and by the result's rounding.
    most = int(c.n_rows.max()) + w + n
    rel = (0.0 if case["rows"] == "f32" else 2.0 ** -8) + 2.0 ** -17 + 2 * d * 2.0 ** -24 + 2 * (most + 8) * 2.0 ** -24
    print("lightest row %.4f of its column, tolerance %.4f" % (lightest, rel), flush=True)
    assert lightest > 2 * rel
    for size in (None, len(lengths) * n * case["hq"] * (2 + int(c.max_head_rows) // 4096) * (d + 4) * 4 + 256):
        got = attend(tb, bufs, prm, c, q, k, v, parent, ws_bytes=size).double().cpu().numpy()
        off = np.abs(got - want) - rel * want
        print("worst %.3g" % off.max(), flush=True)
        assert (off <= 0).all()


# --------------------------------------------------------------------------------------- node rows of any alignment --
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,share", [("bf16", False), ("bf16", True), ("fp8", False), ("fp8", True), ("f32", False)])
def test_accepted_rows_of_any_alignment(tb, bufs, rows, share, d):
    """Acceptance takes q, k_new and v_new at any address of their type, one after the other and all at once, and leaves the same bytes."""
    case = shape(4, 2, d, 8, 64, rows, share)
    prm, c = R.filled_cache(tb, bufs, case, (200, 63, 5), 771)
    n = 30
    q, k, v, parent = R.draft(case, 3, n, 772, [list(range(-1, n - 1))] * 3)
    last = torch.tensor([29, 12, 20], dtype=torch.int32, device="cuda")
    P = np.stack([tb.tca_config_from_budget(8, 1.0, 0.4)] * tb.tca_selection_heads(prm))

    def moved(x):
        flat = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:]
        y = flat.view(x.shape)
        y.copy_(x)
        assert y.data_ptr() % 16 == x.element_size()
        return y

    want = R.clone_cache(tb, bufs, prm, c)
    tb.tca_tree_accept(prm, want.view, want.offs, n, parent, last, q, k, v, P)
    for which in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 1)):
        got = R.clone_cache(tb, bufs, prm, c)
        rows_in = [moved(x) if m else x for x, m in zip((q, k, v), which)]
        tb.tca_tree_accept(prm, got.view, got.offs, n, parent, last, *rows_in, P)
        torch.cuda.synchronize()
        assert not R.same_cache(got, want), which
