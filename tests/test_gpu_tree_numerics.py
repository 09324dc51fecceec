"""Drafted trees: logits of any size."""
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
