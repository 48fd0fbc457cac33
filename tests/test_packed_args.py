"""Packings and the refusals of the operators on packed batches and 8-bit checkpoints: nothing here reaches a GPU."""
import numpy as np
import pytest

import paper_2506_06472_amd as tio

P = 1 << 20                     # an aligned address that no refused call looks at


@pytest.mark.parametrize("lens", [[1], [0], [5, 0, 7], [64, 128, 1, 1000, 0], list(range(40))])
def test_packing_export(lens):
    off = np.concatenate([[0], np.cumsum(lens)])
    for heads in ((), ("bf16", 8, 2, 64), ("bf16", 6, 2, 128), ("fp32", 4, 4, 32), ("bf16", 4, 1, 32)):
        e = tio.tio_packing_build(off, *heads).export()
        assert (e["n_seqs"], e["rows"], e["max_len"]) == (len(lens), sum(lens), max(lens))
        assert np.array_equal(e["data"][:len(off)], off)


@pytest.mark.parametrize("lens,heads", [([700, 0, 33, 1, 64, 65], ("bf16", 12, 4, 64)), ([5000, 3], ("bf16", 4, 1, 128)), ([257, 255], ("bf16", 10, 2, 128)),
                                        ([100, 31], ("fp32", 4, 2, 32)), ([4096], ("bf16", 64, 1, 64))])
def test_items_cover_the_batch_once(lens, heads):
    """The lists behind the offsets (see packing.h): every query row of a group's heads in one block of either query list, every tile of every
    block of keys in one item, the pieces of a shared block side by side among the partial sums; longest first."""
    off = np.concatenate([[0], np.cumsum(lens)])
    data = tio.tio_packing_build(off, *heads).export()["data"]
    at = (len(off) + 3) // 4 * 4
    dtype, H, Hkv, dh = heads
    mfma = dtype == "bf16" and dh > 32
    G = H // Hkv if mfma else 1
    per_tile = 64 // G if mfma else 32
    lists = data[at:]
    where = {int(o): n for o, n in zip(off[:-1], lens) if n}

    def is_query(w):
        return w[3] == 0 and where.get(int(w[0])) == w[1] and w[2] < w[1] * G
    # query lists: until every (sequence, block) of one block size has been seen
    i, seen = 0, []
    total = sum(lens) * G
    while len(seen) < 2 and i + 4 <= len(lists):
        for rows in ((64, 128, 256) if mfma else (32,)):
            n = sum((k * G + rows - 1) // rows for k in lens)
            items = lists[i:i + 4 * n].reshape(-1, 4)
            got = {(int(w[0]), int(w[2])) for w in items}
            if len(items) == n and all(is_query(w) for w in items) and got == {(o, v) for o, k in where.items() for v in range(0, k * G, rows)}:
                last = [min((w[2] + rows - 1) // G, w[1] - 1) for w in items]
                assert last == sorted(last, reverse=True)
                seen.append(rows)
                i += 4 * n
                break
        else:
            break
    assert seen and total
    rest = lists[i:].reshape(-1, 8)
    items, sums = rest[rest[:, 6] == 0], rest[rest[:, 6] > 0]
    keys = min([int(k) for k in items[:, 2] if k] + [256])                  # of a block: the second one of some sequence begins behind it
    assert keys in ((64, 128, 256) if mfma else (32,)) or max(lens) <= 256
    tiles = {}
    for first, n, kv0, t0, t1, part, _, _ in items:
        assert where[int(first)] == n and t0 < t1
        for t in range(t0, t1):
            assert tiles.setdefault((int(first), int(kv0), t), part) == part
    assert set(tiles) == {(o, kv0, t) for o, n in where.items() for kv0 in range(0, n, keys) for t in range((n - kv0 + per_tile - 1) // per_tile)}
    assert len(tiles) == sum(t1 - t0 for _, _, _, t0, t1, *_ in items)
    length = [t1 - t0 for _, _, _, t0, t1, *_ in items]
    assert length == sorted(length, reverse=True)
    parts = []
    for first, n, kv0, _, _, part, pieces, _ in sums:
        mine = sorted((t0, p) for f, _, k, t0, _, p, _, _ in items if (f, k) == (first, kv0))
        assert [p for _, p in mine] == list(range(part, part + pieces)) and pieces > 1
        parts += [p for _, p in mine]
    assert sorted(parts) == sorted(p for *_, p, _, _ in items if p >= 0)


@pytest.mark.parametrize("off,heads", [([0], ()), ([1, 4], ()), ([0, 5, 4], ()), ([0, 4], ("bf16", 3, 2, 64)), ([0, 4], ("bf16", 0, 2, 64)),
                                       ([0, 4], ("bf16", 4, 2, 48)), ([0, 4], ("bf16", 130, 2, 64)), ([0, 4], ("bf16", 4, 0, 64)),
                                       ([0, 1 << 29], ("bf16", 4, 2, 64)), (range(0, 1 << 22), ("fp32", 4, 2, 32)), ([0, 4], ("fp32", -4, -2, 32))])
def test_packings_that_are_refused(off, heads):
    with pytest.raises(tio.TioError) as e:
        tio.tio_packing_build(off, *heads)
    assert e.value.code == -1


def _attention(packing, qkv=P, ld=512, o=P, ldo=256, lse=P, dev=P, bwd=None):
    if bwd is None:
        tio.tio_op_attention_packed(0, packing, dev, qkv, ld, o, ldo, lse)
    else:
        tio.tio_op_attention_packed_bwd(0, packing, dev, qkv, ld, o, bwd[0], ldo, lse, bwd[1], bwd[2])


@pytest.mark.parametrize("bad", [dict(qkv=0), dict(o=0), dict(lse=0), dict(dev=0), dict(qkv=P + 8), dict(o=P + 2), dict(dev=P + 4), dict(ld=511), dict(ld=504),
                                 dict(ldo=248), dict(ldo=260), dict(ld=1 << 24), dict(lse=P + 2)])
@pytest.mark.parametrize("bwd", [None, (P, P, P)])
def test_attention_refusals(bad, bwd):
    with pytest.raises(tio.TioError) as e:
        _attention(tio.tio_packing_build([0, 40], "bf16", 4, 2, 64), **bad, bwd=bwd)
    assert e.value.code == -1


@pytest.mark.parametrize("bwd", [(0, P, P), (P, 0, P), (P, P, 0), (P + 8, P, P), (P, P + 8, P), (P, P, P + 8)])
def test_attention_backward_refusals(bwd):
    with pytest.raises(tio.TioError):
        _attention(tio.tio_packing_build([0, 40], "bf16", 4, 2, 64), bwd=bwd)


def test_attention_needs_heads_and_offsets_within_reach():
    with pytest.raises(tio.TioError, match="without heads"):
        _attention(tio.tio_packing_build([0, 40]))
    with pytest.raises(tio.TioError, match="without heads"):
        tio.tio_op_attention_packed_work(tio.tio_packing_build([0, 40]))
    with pytest.raises(tio.TioError, match="2 GiB"):
        _attention(tio.tio_packing_build([0, 2100000], "bf16", 4, 2, 64))
    _attention(tio.tio_packing_build([0, 0, 0], "bf16", 4, 2, 64))                      # no rows: nothing to do
    _attention(tio.tio_packing_build([0, 0], "fp32", 4, 2, 64), bwd=(P, P, P))


def _preference(n_seqs=4, dtype="bf16", V=1000, logits=P, ld=1000, labels=P, ref=P, beta=0.1, smoothing=0.0, seq=P, losses=P, loss=P, work=P, d=0, dev=P,
                total=0):
    p = tio.tio_packing_build(list(range(0, 10 * n_seqs + 1, 10)))
    tio.tio_op_preference_loss(0, dtype, p, dev, V, logits, ld, labels, ref, beta, smoothing, seq, losses, loss, work, d, total)


@pytest.mark.parametrize("bad", [dict(n_seqs=3), dict(V=0), dict(V=1001), dict(ld=992), dict(ld=1004), dict(dtype="fp32", ld=1002), dict(V=(1 << 28) + 8, ld=1 << 30),
                                 dict(logits=0), dict(labels=0), dict(ref=0), dict(seq=0), dict(losses=0), dict(loss=0), dict(work=0), dict(dev=0),
                                 dict(logits=P + 8), dict(d=P + 8), dict(work=P + 8), dict(labels=P + 2), dict(beta=0.0), dict(beta=-1.0),
                                 dict(beta=float("nan")), dict(beta=float("inf")), dict(smoothing=-0.1), dict(smoothing=1.5),
                                 dict(smoothing=float("nan")), dict(total=1), dict(total=-2)])
def test_preference_refusals(bad):
    with pytest.raises(tio.TioError) as e:
        _preference(**bad)
    assert e.value.code == -1


def test_preference_batches_beyond_a_launch():
    p = tio.tio_packing_build([0, 1 << 21, 1 << 22])
    with pytest.raises(tio.TioError, match="2.22"):
        tio.tio_op_preference_loss(0, "bf16", p, P, 8, P, 8, P, P, 0.1, 0.0, P, P, P, P, P)


def test_preference_pairs_beyond_a_launch():
    """Empty sequences: few rows do not mean few pairs."""
    p = tio.tio_packing_build(np.zeros((1 << 23) + 1, np.int32))
    with pytest.raises(tio.TioError, match="pairs"):
        tio.tio_op_preference_loss(0, "bf16", p, P, 8, P, 8, P, P, 0.1, 0.0, P, P, P, P, P)


@pytest.mark.parametrize("rows,cols,want", [(1, 1, 48), (1, 32, 48), (3, 33, 208), (128, 512, 128 * 512 + 128 * 16), (1021, 2730, (1021 * 86 * 33 + 15) // 16 * 16)])
def test_checkpoint_bytes(rows, cols, want):
    assert tio.tio_ckpt8_bytes(rows, cols) == want


@pytest.mark.parametrize("rows,cols", [(0, 4), (4, 0), (-1, 4), (1 << 40, 1 << 40), (1 << 31, 32), (1, 1 << 35)])
def test_checkpoint_sizes_that_are_refused(rows, cols):
    with pytest.raises(tio.TioError):
        tio.tio_ckpt8_bytes(rows, cols)
    with pytest.raises(tio.TioError):
        tio.tio_op_ckpt8_store(0, "bf16", rows, cols, P, 8, P)


@pytest.mark.parametrize("x,ld,kept", [(0, 104, P), (P, 104, 0), (P + 8, 104, P), (P, 104, P + 4), (P, 100, P), (P, 96, P)])
def test_checkpoint_refusals(x, ld, kept):
    for call in (tio.tio_op_ckpt8_store, lambda s, t, r, c, x, ld, k: tio.tio_op_ckpt8_load(s, t, r, c, k, x, ld)):
        with pytest.raises(tio.TioError) as e:
            call(0, "bf16", 4, 100, x, ld, kept)
        assert e.value.code == -1


@pytest.mark.parametrize("bad", [dict(act="gelu", up=P), dict(up=0), dict(gate=0), dict(y=0), dict(kept=0), dict(ldu=100), dict(ldy=96), dict(gate=P + 8),
                                 dict(up=P + 2), dict(y=P + 8), dict(kept=P + 8), dict(rows=0), dict(f=0)])
def test_activation_refusals(bad):
    a = dict(act="swiglu", rows=4, f=100, gate=P, up=P, ldu=104, y=P, ldy=104, kept=P)
    a.update(bad)
    with pytest.raises(tio.TioError):
        tio.tio_op_act_ckpt8(0, "bf16", a["act"], a["rows"], a["f"], a["gate"], a["up"], a["ldu"], a["y"], a["ldy"], a["kept"])
    if "y" not in bad:                                     # its gradient's y is optional, dy is not
        with pytest.raises(tio.TioError):
            tio.tio_op_act_ckpt8_bwd(0, "bf16", a["act"], a["rows"], a["f"], a["kept"], P, 104, a["gate"], a["up"], a["ldu"], a["y"], a["ldy"])
    with pytest.raises(tio.TioError):
        tio.tio_op_act_ckpt8_bwd(0, "bf16", "swiglu", 4, 100, P, 0, 104, P, P, 104)


@pytest.mark.parametrize("dtype,H,Hkv,dh,rows", [("bf16", 64, 1, 128, 1 << 22), ("bf16", 64, 1, 64, 1 << 23), ("bf16", 7, 7, 128, 38400000)])
def test_backward_passes_beyond_a_launch(dtype, H, Hkv, dh, rows):
    """The launch for delta has a thread for every 16 bytes of dO, and a grid fewer than 2^32: refused before anything is launched."""
    p = tio.tio_packing_build(np.arange(0, rows + 1, 12800 if rows % 12800 == 0 else 1 << 14), dtype, H, Hkv, dh)
    ld, ldo = (H + 2 * Hkv) * dh, H * dh
    with pytest.raises(tio.TioError, match="backward") as e:
        tio.tio_op_attention_packed_bwd(0, p, P, P, ld, P, P, ldo, P, P, P)
    assert e.value.code == -1


@pytest.mark.parametrize("heads", [("fp32", 1, 1, 32), ("bf16", 1, 1, 32), ("bf16", 1, 1, 64), ("bf16", 1, 1, 128)])
@pytest.mark.parametrize("rows", [(1 << 31) - 1, (1 << 31) - 200, (1 << 30) + 77])
def test_one_sequence_of_nearly_all_rows_is_refused(heads, rows):
    """Before any list is built: the lists of such a batch would take gigabytes, and its last block ends past 32 bits."""
    import resource
    before = resource.getrusage(resource.RUSAGE_SELF).ru_maxrss
    with pytest.raises(tio.TioError, match="cut the batch") as e:
        tio.tio_packing_build([0, rows], *heads)
    assert e.value.code == -1
    assert resource.getrusage(resource.RUSAGE_SELF).ru_maxrss - before < 1 << 16          # KiB


def test_more_sequences_than_words_are_refused():
    """By their number: no offset is looked at."""
    import ctypes as C
    off, out = (C.c_int32 * 1)(0), C.c_void_p()
    for n in (1 << 28, (1 << 31) - 1):
        assert tio.binding.lib().tio_packing_build(off, C.c_int32(n), 1, C.c_int64(0), C.c_int64(0), C.c_int64(0), C.byref(out)) == -1


@pytest.mark.parametrize("rows,cols,fits", [(8, (1 << 31) - 1024, True), (8, (1 << 31) - 1023, False), (9, (1 << 31) - 1024, False), ((1 << 29) - 256, 32, True),
                                            ((1 << 29) - 256, 33, False), ((1 << 29) - 255, 32, False), ((1 << 28) - 128, 64, True), ((1 << 31) - 1024, 1, False)])
def test_largest_checkpoints(rows, cols, fits):
    """The limits that the header gives: 2^34 - 2^13 values in whole blocks of 32."""
    assert fits == (rows * ((cols + 31) // 32 * 32) <= (1 << 34) - (1 << 13) and max(rows, cols) <= (1 << 31) - 1024)
    if fits:
        assert tio.tio_ckpt8_bytes(rows, cols) == (rows * ((cols + 31) // 32) * 33 + 15) // 16 * 16
    else:
        with pytest.raises(tio.TioError, match="2.34"):
            tio.tio_ckpt8_bytes(rows, cols)
