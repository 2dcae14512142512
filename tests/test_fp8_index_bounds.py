"""A CPU model of the index arithmetic of the 8-bit cache's kernels (no GPU): the
places that the wide kernel's staging and epilogue use in LDS, the transposed reads,
the tiles' pieces, the work items that workgroups pick by themselves, and the shares of
head rows, each over their whole ranges."""
import numpy as np
import pytest

import fp8_reference as ref

WAVE = 64


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("W", [2, 4])
def test_wide_staging_fills_every_place_once(D, W):
    threads, TP, RP = W * WAVE, 2 * D, D // 8
    BP = 2 * TP
    NP = 2 * 2 * D // threads
    assert NP >= 1 and D % WAVE == 0
    written, read = np.zeros(2 * BP, int), np.zeros((2, 2, 16 * D), int)
    one_side = NP >= 2
    for k in range(NP):
        for tid in range(threads):
            x = k * threads + tid
            side = k // (NP // 2 + (1 if NP < 2 else 0)) if one_side else x // (2 * D)
            assert side == x // (2 * D)
            blk, pc = x // D % 2, x % D
            # uniform for the wavefront
            first = k * threads + tid // WAVE * WAVE
            assert first // D % 2 == blk and first // (2 * D) == side
            assert 16 * pc + 16 <= 16 * D
            read[side, blk, 16 * pc:16 * pc + 16] += 1
            if side == 0:
                slot, kg, c = pc % 16, pc // 16 % 4, pc // 64
                s_off = slot
                dst = [blk * BP + (8 * c + 4 * h + kg) * 16 + slot for h in range(2)]
                # a 16-byte piece is elements 64 c + 32 h + 8 kg .. of the slot
                for h in range(2):
                    d = 64 * c + 32 * h + 8 * kg
                    assert np.ravel_multi_index(ref.k_place(d, slot), (D // 64, 4, 16, 2, 8)) == 16 * pc + 8 * h
            else:
                piece, kg, j = pc % RP, pc // RP % 4, pc // (4 * RP)
                s_off = 16 + 4 * kg + 2 * j
                dst = []
                for e in range(2):
                    r = 4 * kg + 2 * j + e
                    perm = 4 * (r & 3) if D == 128 else 4 * ((r >> 1) & 1)
                    assert (piece ^ perm) < RP
                    dst.append(blk * BP + TP + r * RP + (piece ^ perm))
                    assert np.ravel_multi_index(ref.v_place(8 * piece, r), (2, 4, D // 8, 2, 8)) == 16 * pc + 8 * e
            assert s_off + (1 if side == 0 else 2) <= 32 and (side == 0 or s_off % 2 == 0)
            for x in dst:
                written[x] += 1
    assert (written == 1).all() and (read == 1).all()


@pytest.mark.parametrize("D", [64, 128])
def test_wide_reads_stay_in_their_tiles(D):
    TP, RP, KS, VT = 2 * D, D // 8, D // 16, D // 32
    BP = 2 * TP
    rows = np.zeros((16, D), int)
    for lane in range(WAVE):
        hh, col = lane >> 5, lane & 31
        for c in range(KS):
            piece = (col >> 4) * BP + hh * 16 + (lane & 15) + 32 * c
            blk, within = divmod(piece, BP)
            assert blk == col >> 4 and within < TP and within // 16 == 2 * c + hh and within % 16 == col % 16
        s16 = lane & 15
        tr_row = (4 * hh + s16 // 4) * D + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3)
        for t in range(VT):
            off = tr_row + 32 * (t ^ (s16 // 4 if D == 128 else s16 // 8))
            for more in (0, 8 * D):
                at = off + more
                assert 0 <= at and at + 4 <= 16 * D
                r, e = divmod(at, D)
                perm = 4 * (r & 3) if D == 128 else 4 * ((r >> 1) & 1)
                d = 8 * ((e // 8) ^ perm) + e % 8
                rows[r, d:d + 4] += 1
                assert r == 4 * hh + s16 // 4 + (8 if more else 0)
                assert 32 * t <= d < 32 * t + 32  # the tile's own columns
    assert (rows == 1).all()


@pytest.mark.parametrize("D", [64, 128])
def test_wide_epilogue_places(D):
    UH, VT = D // 8, D // 32
    for half in range(2):
        at = np.zeros((32, UH), int)
        for lane in range(WAVE):
            hh, col = lane >> 5, lane & 31
            for t in range(VT // 2):
                for k in range(4):
                    u = 8 * t + 2 * k + hh
                    assert u < UH
                    at[col, u ^ (col & (UH - 1))] += 1
        assert (at == 1).all()
    # what the epilogue holds fits where the staging buffers were
    for W in (2, 4):
        buffers = 3 if W == 4 else 2
        assert W * 32 * UH * 16 <= buffers * 2 * 2 * 2 * D * 16


@pytest.mark.parametrize("D", [64, 128])
def test_decode_pieces(D):
    """The lane's K pieces are its MFMA fragments (elements 32 c + 8 kg of its token), its V pieces its four rows' 8
    columns."""
    seen_k, seen_v = np.zeros((16, D), int), np.zeros((16, D), int)
    for lane in range(WAVE):
        n, kg = lane & 15, lane >> 4
        for c in range(D // 64):
            at = 16 * lane + 1024 * c
            assert at + 16 <= 16 * D
            for h in range(2):  # k-step 2 c + h
                d = 32 * (2 * c + h) + 8 * kg
                assert np.ravel_multi_index(ref.k_place(d, n), (D // 64, 4, 16, 2, 8)) == at + 8 * h
                seen_k[n, d:d + 8] += 1
        for j in range(2):
            at = ((4 * j + kg) * (D // 8) + n % (D // 8)) * 16
            assert at + 16 <= 16 * D
            for e in range(2):
                r, d = 4 * kg + 2 * j + e, 8 * (n % (D // 8))
                assert np.ravel_multi_index(ref.v_place(d, r), (2, 4, D // 8, 2, 8)) == at + 8 * e
                seen_v[r, d:d + 8] += 1
    assert (seen_k == 1).all() and (seen_v == 128 // D).all()


def picked(B, P, H, lens, Tp):
    """(pair, head) of every workgroup of a step that picks its items."""
    pairs = B * P
    cls = []
    for x in range(pairs):
        p, b = divmod(x, B)
        tok = min(max(lens[b] - p * Tp, 0), Tp)
        cls.append(255 - min(-(-tok // 16), 255))
    order = sorted(range(pairs), key=lambda x: (cls[x], x))  # what ranking by class, then index, finds
    for slot in range(pairs * H):
        if H % 8 == 0:
            pos, g = divmod(slot, H)
        else:
            first = slot // (8 * H) * 8
            c = min(8, pairs - first)
            within = slot - first * H
            pos, g = first + within % c, within // c
        yield order[pos], g


def test_picked_items_are_a_permutation():
    rng = np.random.RandomState(0)
    for _ in range(60):
        P, H = int(rng.randint(1, 9)), int(rng.choice([1, 2, 3, 5, 8, 16, 24]))
        B = int(rng.randint(1, 256 // P + 1))
        Tp = 16 * int(rng.randint(1, 40))
        lens = rng.randint(0, P * Tp + 1, B)
        got = sorted(picked(B, P, H, lens, Tp))
        assert got == [(x, g) for x in range(B * P) for g in range(H)]


def test_row_shares_cover_a_row_once():
    for D in range(8, 513, 8):
        for R in [0] + list(range(16, D + 1, 16)):
            for inter in (False, True):
                shares = (D + 15) // 16
                seen, turned = np.zeros(D, int), np.zeros(D, int)
                for u in range(shares):
                    if inter or R == 0:
                        d0, d1 = 8 * u, 8 * (u + shares)
                        t = 2 if d1 < R else 1 if d0 < R else 0
                    elif u < R // 16:
                        d0, d1, t = 8 * u, R // 2 + 8 * u, 2
                    else:
                        d0 = R + 8 * (u - R // 16)
                        d1, t = d0 + 8 * (shares - R // 16), 0
                    assert d0 + 8 <= D
                    seen[d0:d0 + 8] += 1
                    turned[d0:d0 + 8] += t > 0
                    if d1 < D:
                        assert d1 + 8 <= D
                        seen[d1:d1 + 8] += 1
                        turned[d1:d1 + 8] += t > 1
                    else:
                        assert t < 2
                assert (seen == 1).all(), (D, R, inter)
                assert (turned[:R] == 1).all() and (turned[R:] == 0).all()
