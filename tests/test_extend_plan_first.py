"""The extend plan that a program asks for is the one that runs, first tokens
beside the window included (metadata-only store, CPU)."""

import math
import os
import random

import pytest


@pytest.fixture(scope="module")
def sq():
    from paper_2602_22603_amd import build_lib, sq as sqmod
    if not os.path.exists(sqmod.LIB_PATH):
        build_lib.build()
    sqmod.lib()
    return sqmod


def _plans(sq, hq, hkv, d, n, base, *opts):
    s = sq.Store(num_layers=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, num_pages=(n + base + 15) // 16,
                 max_seqs=1, max_pages_per_seq=(n + base + 15) // 16, metadata_only=True)
    a = s.seq_create()
    s.append(a, n=n + base)
    out = [s.extend_plan_info(a, n, **o) for o in opts]
    s.close()
    return out


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (64, 8, 64), (8, 8, 64), (8, 1, 128)])
def test_splits_cover_the_window_and_the_first_tokens(sq, hq, hkv, d):
    """A query block's list: the first tokens' blocks in front of its window's."""
    rng = random.Random(hq + d)
    for _ in range(120):
        n = int(round(math.exp(rng.uniform(0, math.log(2000)))))
        base = int(round(math.exp(rng.uniform(0, math.log(60000))))) - 1
        w = rng.choice([1, 64, 300, 5000])
        first = rng.choice([1, 64, 3001, 9000, 70000, 2 ** 31 - 1])
        p, = _plans(sq, hq, hkv, d, n, base, dict(window=w, first=first))
        tq, total = p["rows"] // (hq // hkv), n + base
        assert p["n_qblocks"] == -(-n // tq)
        for qb in range(p["n_qblocks"]):
            begin = max(0, base + qb * tq - w + 1) // 64
            blocks = -(-min(total, base + (qb + 1) * tq) // 64) - begin + min(-(-min(first, total) // 64), begin)
            assert p["n_split"] * p["split_blocks"] >= blocks, (n, base, w, first, p)
        if p["n_split"] > 1:
            assert p["n_split"] <= 64 and p["n_qblocks"] * hkv * p["n_split"] * p["rows"] <= 8192 * 16


def test_first_tokens_count_with_a_window_only(sq):
    """Without a window they change nothing; all of them are as if there were
    none (every key is seen), and more keys mean other splits."""
    none, alone, window, both, far = _plans(
        sq, 32, 8, 128, 5, 20000, dict(), dict(first=9000), dict(window=300), dict(window=300, first=9000),
        dict(window=300, first=2 ** 31 - 1))
    assert alone == none and both != window
    assert far["n_split"] * far["split_blocks"] >= -(-20005 // 64)


def test_arguments(sq):
    s = sq.Store(1, 8, 2, 64, 8, 2, 8, metadata_only=True)
    a = s.seq_create()
    s.append(a, n=20)
    for kw in (dict(window=4, first=-1), dict(window=-1, first=1), dict(window=1 << 32), dict(window=4, first=1 << 32)):
        with pytest.raises(sq.SqError):
            s.extend_plan_info(a, 4, **kw)
    import ctypes as C
    o, out = sq.AttnOpts(), sq.ExtendInfo()
    assert sq.lib().sq_extend_plan_info_opts(s._handle, a, 4, None, C.byref(out)) == sq.OK
    assert sq.lib().sq_extend_plan_info_opts(s._handle, a, 4, C.byref(o), None) == sq.ERR_INVALID
    o.reserved = 1
    assert sq.lib().sq_extend_plan_info_opts(s._handle, a, 4, C.byref(o), C.byref(out)) == sq.ERR_INVALID
    s.close()
