"""The plan of a drafted batch (csrc/draft_plan.hpp) on the CPU: a small program
around it, compiled by g++ with AddressSanitizer and UndefinedBehaviorSanitizer,
prints the plans of random batches.  Checked here: every node sees what the
oracle says it sees, and in blocks that its tile reads; every key block of every
(tile, KV head) is dealt to exactly one piece, every piece to one workgroup's
chain, which ends; pieces, rows and partial rows stay inside their arrays."""

import os
import random
import subprocess

import pytest

from oracle import draft as odr

# the arrays' sizes: rows and workgroups of a plan, partial rows of the workspace
ROWS, WGS, PARTIAL = 4096, 1024, 8192 * 16

PROGRAM = r"""
#include <cstdio>
#include <memory>
#include "draft_plan.hpp"
using namespace sq;
int main() {
  int hkv, G, D, cus, kv8, batch, window, first;
  auto nodes = std::make_unique<DraftNode[]>(kMaxBatch * kMaxDraft);
  auto sp = std::make_unique<DraftSplit>();
  printf("%d %d %d\n", kDraftRows, kDraftWgs, kMaxItems * kRows);
  while (scanf("%d %d %d %d %d %d %d %d", &hkv, &G, &D, &cus, &kv8, &batch, &window, &first) == 8) {
    std::vector<int32_t> counts(batch), base(batch), parents;
    for (int b = 0; b < batch; ++b) {
      if (scanf("%d %d", &base[b], &counts[b]) != 2) return 1;
      for (int i = 0, p; i < counts[b]; ++i) {
        if (scanf("%d", &p) != 1) return 1;
        parents.push_back(p);
      }
    }
    std::vector<int32_t> depth(parents.size());
    const DraftModel m{hkv, G, D, cus, kv8 != 0};
    const DraftShape shape = draft_shape(m, counts.data(), batch);
    std::vector<DraftTile> tiles[2];
    int tok0 = 0;
    printf("S %d %d %d\n", shape.rows, shape.n_wg, shape.shared);
    for (int b = 0; b < batch; ++b) {
      if (!tree_depths(parents.data() + tok0, counts[b], depth.data() + tok0)) return 2;
      const DraftEntry e{b, (base[b] + counts[b] + kPage - 1) / kPage, base[b], counts[b], tok0, 0,
                         parents.data() + tok0, depth.data() + tok0};
      printf("E %lld\n", (long long)draft_entry(e, window, first, shape, G, nodes.get(), tiles));
      tok0 += counts[b];
    }
    for (int i = 0; i < tok0; ++i)
      printf("N %llu %llu %d %d %d\n", (unsigned long long)nodes[i].anc[0], (unsigned long long)nodes[i].anc[1],
             nodes[i].lo, nodes[i].tile, nodes[i].in_tile);
    for (int w = 0; w < (window > 0 ? 2 : 1); ++w) {
      const int n = draft_split(tiles[w], m, shape, sp.get());
      printf("P %d %d %d %d\n", sp->n_used, sp->rows, sp->total, n);
      for (const DraftTile &t : tiles[w])
        printf("T %d %d %d %d %d %d %d %d %d %lld\n", t.as.row, t.as.base, t.as.n, t.as.n_pages, t.as.node0,
               t.as.n_nodes, t.as.nf, t.as.skip, t.as.lo_max, (long long)t.blocks);
      for (size_t r = 0; r < tiles[w].size() * hkv; ++r) printf("M %d %d\n", sp->merge[r].row0, sp->merge[r].n);
      for (int i = 0; i < n; ++i) {
        const DraftPiece &p = sp->pieces[i];
        printf("I %d %d %d %d %d %d %d %d %d %d %d %d %d %d\n", p.g, p.row, p.base, p.n, p.n_pages, p.node0, p.n_nodes,
               p.nf, p.skip, p.lo_max, p.b_lo, p.b_hi, p.slot, p.next);
      }
    }
    printf("X\n");
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_2602_22603_amd import build_lib
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build_lib._hipcc())))
    out = tmp_path_factory.mktemp("plan")
    (out / "plan.cpp").write_text(PROGRAM)
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
           "-I", build_lib.CSRC, *build_lib.SAN_FLAGS, str(out / "plan.cpp"), "-o", str(out / "plan")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    return str(out / "plan")


def _plans(program, cases):
    """[(shape, first keys, nodes, plans)]; a plan: (header, tiles, merges, pieces)."""
    text = []
    for c in cases:
        text.append(f"{c['hkv']} {c['G']} {c['D']} {c['cus']} {int(c['kv8'])} {len(c['trees'])} {c['window']} {c['first']}")
        for base, tree in zip(c["bases"], c["trees"]):
            text.append(f"{base} {len(tree)} " + " ".join(map(str, tree)))
    res = subprocess.run([program], input="\n".join(text), capture_output=True, text=True, timeout=200)
    assert res.returncode == 0, res.stderr[-4000:]
    lines = [line.split() for line in res.stdout.splitlines()]
    assert [int(x) for x in lines[0]] == [ROWS, WGS, PARTIAL]
    out, cur = [], None
    for line in lines[1:]:
        kind, v = line[0], [int(x) for x in line[1:]]
        if kind == "S":
            cur = (v, [], [], [])
        elif kind == "E":
            cur[1].append(v[0])
        elif kind == "N":
            cur[2].append(v)
        elif kind == "P":
            cur[3].append((v, [], [], []))
        elif kind in "TMI":
            cur[3][-1]["TMI".index(kind) + 1].append(v)
        else:
            out.append(cur)
    assert len(out) == len(cases)
    return out


def _tree(rng, n):
    return [-1] + [rng.randrange(max(-1, i - 6), i) for i in range(1, n)]


def _case(rng, longest, seqs, **kw):
    n = rng.randrange(1, seqs + 1)
    small = rng.choice([1, 5, 16, 64])
    return dict(dict(hkv=rng.choice([1, 2, 8, 8, 16]), G=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128]), cus=256,
                     kv8=rng.random() < 0.5, window=rng.choice([0, 1, 3, 16, 100, 4096]),
                     first=rng.choice([0, 1, 4, 64, 131, 10 ** 6, 2 ** 31 - 1]),
                     bases=[rng.choice([0, 1, rng.randrange(longest)]) for _ in range(n)],
                     trees=[_tree(rng, rng.randrange(1, rng.choice([small, 64]) + 1)) for _ in range(n)]), **kw)


def _check_split(c, shape, plan, trees):
    rows, n_wg, shared = shape
    (n_used, p_rows, p_total, n_pieces), tiles, merges, pieces = plan
    assert (p_rows, p_total) == (rows, sum(map(len, trees)))
    assert 1 <= n_used <= n_wg <= min(WGS, c["cus"] * 3) and len(tiles) * c["hkv"] == len(merges) <= ROWS
    assert n_used <= n_pieces == len(pieces) <= ROWS + WGS
    # chains: every piece has one owner
    seen, by_row = set(), {}
    for w in range(n_used):
        at = w
        while at >= 0:
            assert at not in seen and at < n_pieces
            seen.add(at)
            p = pieces[at]
            if p[10] < p[11]:
                by_row.setdefault((p[5], p[0]), []).append(p)
            else:
                assert at == w and p[13] == -1  # (a workgroup without work)
            at = p[13]
    assert len(seen) == n_pieces
    # rows: every block dealt once; parts have partial rows of their own
    slots = []
    for t, tile in enumerate(tiles):
        row, base, n, n_pages, node0, n_nodes, nf, skip, lo_max, blocks = tile
        assert 1 <= n_nodes * c["G"] <= rows and n == len(trees[row]) and base == c["bases"][row]
        for g in range(c["hkv"]):
            mine = sorted(by_row.pop((node0, g)), key=lambda p: p[10])
            assert [p[10] for p in mine] == [0] + [p[11] for p in mine[:-1]] and mine[-1][11] == blocks
            for p in mine:
                assert p[1:10] == [row, base, n, n_pages, node0, n_nodes, nf, skip, lo_max]
            row0, parts = merges[t * c["hkv"] + g]
            if len(mine) == 1:
                assert parts == 0 and mine[0][12] == -1
            else:
                assert parts == len(mine)
                assert sorted(p[12] for p in mine) == [row0 + i * rows for i in range(parts)]
                slots += [p[12] for p in mine]
    assert not by_row
    assert len(set(slots)) == len(slots) and all(s >= 0 and s % rows == 0 and s + rows <= PARTIAL for s in slots)
    assert shared or all(len(t) * c["G"] <= rows for t in trees)


def _blocks(tile):
    nf, skip, blocks = tile[6], tile[7], tile[9]
    return [i if i < nf else i + skip for i in range(blocks)]


def test_every_block_is_dealt_once(program):
    rng = random.Random(1)
    cases = [_case(rng, 150000, rng.choice([1, 2, 12])) for _ in range(160)]
    cases += [_case(rng, 3000, 64, hkv=rng.choice([1, 8, 16])) for _ in range(25)]
    cases += [_case(rng, 150000, 8, cus=cus) for cus in (1, 3, 64, 304, 1500) for _ in range(4)]
    # the most rows, and the longest caches of the fewest rows
    cases += [dict(hkv=64, G=8, D=128, cus=256, kv8=kv8, window=0, first=0, bases=[20000] * 16, trees=[_tree(rng, 64)] * 16)
              for kv8 in (False, True)]
    cases += [dict(hkv=1, G=G, D=64, cus=256, kv8=False, window=100, first=4, bases=[2 ** 24], trees=[_tree(rng, n)])
              for G in (1, 8) for n in (1, 5, 64)]
    cases = [c for c in cases
             if sum(-(-len(t) * c["G"] // 16) for t in c["trees"]) * c["hkv"] <= ROWS or c["hkv"] == 64]
    for c, (shape, _, nodes, plans) in zip(cases, _plans(program, cases)):
        n_rows = sum(-(-len(t) // (shape[0] // c["G"])) for t in c["trees"]) * c["hkv"]
        assert n_rows <= ROWS
        for plan in plans:
            _check_split(c, shape, plan, c["trees"])
            at = 0
            for t, tile in enumerate(plan[1]):  # the tiles hold the nodes in order
                assert tile[4] == at
                for i in range(tile[5]):
                    assert nodes[at + i][3:] == [t, i]
                at += tile[5]
            assert at == len(nodes)


def test_nodes_see_what_the_oracle_says(program):
    rng = random.Random(2)
    cases = [_case(rng, 700, 5, window=rng.choice([0, 1, 2, 5, 40, 300, 10 ** 6]),
                   first=rng.choice([0, 1, 63, 64, 65, 200, 10 ** 6])) for _ in range(120)]
    for c, (shape, firsts, nodes, plans) in zip(cases, _plans(program, cases)):
        at = 0
        for base, tree, lo_seq in zip(c["bases"], c["trees"], firsts):
            for w, plan in enumerate(plans):
                window, first = (c["window"], c["first"]) if w else (0, 0)
                want = odr.visible(tree, base, window, first)
                for i, slots in enumerate(want):
                    anc, lo, t = nodes[at + i][w], nodes[at + i][2] if w else 0, nodes[at + i][3]
                    got = [k for k in range(base) if k >= lo or k < first] + \
                          [base + j for j in range(len(tree)) if anc >> j & 1]
                    assert sorted(got) == sorted(slots), (c, i)
                    assert set(s // 64 for s in slots) <= set(_blocks(plan[1][t])), (c, i)
                    if w:
                        assert lo <= plan[1][t][8] and min([s for s in slots if s >= first] or [lo_seq]) >= lo_seq
            at += len(tree)
        for plan in plans:  # a list of blocks goes to the last key, without a repetition
            for tile in plan[1]:
                b = _blocks(tile)
                assert b == sorted(set(b)) and b[-1] == (tile[1] + tile[2] - 1) // 64


def test_the_same_counts_take_the_same_launches(program):
    """A captured layer is replayed for any draft of its counts, so tile and
    launch may not follow from lengths, trees or windows."""
    rng = random.Random(3)
    for _ in range(10):
        c = _case(rng, 5000, 8)
        others = [dict(c, bases=[rng.randrange(90000) for _ in c["bases"]], trees=[_tree(rng, len(t)) for t in c["trees"]],
                       window=w) for w in (0, 7, 4096)]
        shapes = [p[0] for p in _plans(program, others)]
        assert shapes[0] == shapes[1] == shapes[2]
