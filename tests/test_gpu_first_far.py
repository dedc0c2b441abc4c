"""First tokens beside a window, as many as an int32 holds: every key, in decode,
steps, extend and drafts.  Against float64; tolerance 5e-4, as for every
attention output from N(0, 1) inputs."""

import math

import pytest

from oracle import draft as odr
from paper_2602_22603_amd import workload as wl

pytestmark = pytest.mark.gpu
TOL = 5e-4
FAR = [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 65]


@pytest.fixture(scope="module")
def sq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_22603_amd import sq as sqmod
    sqmod.lib()
    return sqmod


def _attend(q, k, v, seen):
    """q [n, Hq, D] over k, v [L, Hkv, D]; seen: bool [n, L]; float64."""
    import torch
    n, hq, d = q.shape
    out = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
    for h in range(hq):
        g = h // (hq // k.shape[1])
        s = (q[:, h].double() @ k[:, g].double().T.contiguous()) / math.sqrt(d)
        out[:, h] = torch.softmax(s.masked_fill(~seen, -math.inf), 1) @ v[:, g].double().contiguous()
    return out


def _store(sq, n):
    s = sq.Store(1, 16, 4, 128, num_pages=60, max_seqs=1, max_pages_per_seq=50)
    h = s.seq_create()
    k, v = (wl.device_normal_bf16((1, n, 4, 128), j, "cuda") for j in (0, 1))
    s.append(h, k, v)
    return s, h, k, v


def _causal(n, total):
    import torch
    return torch.arange(total, device="cuda")[None] <= (total - n + torch.arange(n, device="cuda"))[:, None]


@pytest.mark.parametrize("first", FAR)
@pytest.mark.parametrize("n", [1, 70, 300])
def test_extend(sq, n, first):
    s, h, k, v = _store(sq, 613)
    q = wl.device_normal_bf16((n, 16, 128), 5, "cuda")
    for window in (1, 20, 2 ** 31 - 1):
        got = s.extend(0, h, q, window=window, first=first)
        assert (got.double() - _attend(q, k[0], v[0], _causal(n, 613))).abs().max() <= TOL


@pytest.mark.parametrize("first", FAR)
def test_decode_and_step(sq, first):
    import torch
    s, h, k, v = _store(sq, 613)
    q = wl.device_normal_bf16((1, 16, 128), 5, "cuda")
    for mode in (sq.ATTN_AUTO, sq.ATTN_STREAM):
        got = s.decode(0, [h], q, mode=mode, window=20, first=first)
        assert (got.double() - _attend(q, k[0], v[0], _causal(1, 613))).abs().max() <= TOL
    kn, vn = (wl.device_normal_bf16((1, 4, 128), j, "cuda") for j in (7, 8))
    s.step_begin([h], window=20, first=first)
    got = s.step_attn(0, kn, vn, q, window=20, first=first)
    want = _attend(q, torch.cat([k[0], kn]), torch.cat([v[0], vn]), _causal(1, 614))
    assert (got.double() - want).abs().max() <= TOL


@pytest.mark.parametrize("first", FAR)
def test_draft(sq, first):
    import torch
    s, h, k, v = _store(sq, 613)
    tree = [-1, 0, 0, 1, 3, 2, -1]
    n = len(tree)
    q = wl.device_normal_bf16((n, 16, 128), 5, "cuda")
    kn, vn = (wl.device_normal_bf16((n, 4, 128), j, "cuda") for j in (7, 8))
    s.draft_begin([h], [tree], window=2, first=first)
    s.qkv_store(0, q, kn, vn)
    got = s.draft_attn(0, q, window=2, first=first)
    seen = torch.zeros(n, 613 + n, dtype=torch.bool)
    for i, slots in enumerate(odr.visible(tree, 613, 2, first)):
        seen[i, slots] = True
    want = _attend(q, torch.cat([k[0], kn]), torch.cat([v[0], vn]), seen.cuda())
    assert (got.double() - want).abs().max() <= TOL
    s.draft_accept([[]])
