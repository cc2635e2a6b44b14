"""The prompt path without a GPU: the numbering of the attention's work units (csrc/prompt_geometry.cuh, compiled
for the host) against a sort, the host's refusals, and the oracle's own examples."""
import ctypes
import os
import random
import re
import subprocess

import numpy as np
import pytest

import oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include "prompt_geometry.cuh"
// stdin: width batch max_ctx max_tokens, then (ctx, tokens) per sequence; prints every block in order (found from
// the start, and from where the one before was found), and whether the first number past them is refused.
int main() {
  int width, batch, max_ctx, max_tokens;
  while (std::scanf("%d %d %d %d", &width, &batch, &max_ctx, &max_tokens) == 4) {
    static int ctx[4096], n[4096];
    int total = 0;
    for (int b = 0; b < batch; ++b) {
      if (std::scanf("%d %d", ctx + b, n + b) != 2) return 1;
      total += ptd::prompt_blocks(ctx[b], n[b], width, ptd::index_divisor(width)).count;
    }
    auto load = [&](int b) { return ptd::PromptSequence{7 * b, n[b], ctx[b], ptd::prompt_blocks(ctx[b], n[b], width, ptd::index_divisor(width))}; };
    const int step = ptd::prompt_level_step(max_ctx, max_tokens, width);
    auto from = [&](int level) {
      int c = 0;
      for (int b = 0; b < batch; ++b) c += ptd::blocks_from(load(b).blocks, level * step);
      return c;
    };
    auto level_of = [&](int u, int& upto, int& above) {
      int level = 31;
      while (level > 0 && from(level) <= u) --level;
      upto = from(level), above = level < 31 ? from(level + 1) : 0;
      return level;
    };
    ptd::PromptCursor on = {0, 0, 0, 0, 0};
    ptd::PromptSequence s;
    int b, i, b2, i2;
    for (int u = 0; u <= total; ++u) {
      ptd::PromptCursor fresh = {0, 0, 0, 0, 0};
      const bool found = ptd::find_prompt_block(ptd::OneLane{}, load, level_of, batch, step, u, fresh, b, i, s);
      if (found != (u < total)) return 1;
      if (u % 3 == 1 && u < total) continue;   // (a CTA does not get every number)
      if (ptd::find_prompt_block(ptd::OneLane{}, load, level_of, batch, step, u, on, b2, i2, s) != found) return 1;
      if (found && (b2 != b || i2 != i || s.row0 != 7 * b || s.tokens != n[b] || s.ctx != ctx[b])) return 1;
      if (found) std::printf("%d,%d ", b, i);
    }
    for (int u = 1; u < total; u += 3) {
      ptd::PromptCursor fresh = {0, 0, 0, 0, 0};
      if (!ptd::find_prompt_block(ptd::OneLane{}, load, level_of, batch, step, u, fresh, b, i, s)) return 1;
      std::printf("%d,%d ", b, i);
    }
    ptd::PromptCursor fresh = {0, 0, 0, 0, 0};
    std::printf("%d\n", ptd::find_prompt_block(ptd::OneLane{}, load, level_of, batch, step, -1, fresh, b, i, s));
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    from paper_2607_10661_gb300 import ptd

    __graft_entry__.build()
    return ptd.lib()


def test_blocks_are_numbered_longest_first(tmp_path):
    rng = random.Random(5)
    cases = [(64, [(0, 0)]), (64, [(5, 1)]), (64, [(100, 640)]), (1, [(3, 4), (0, 9), (5, 0), (2, 2)]),
             (256, [(0, 0), (0, 0)]), (2, [(rng.randrange(4000), 1) for _ in range(128)]),
             (2, [(rng.randrange(4000), rng.randrange(3)) for _ in range(129)]),
             (32, [(1000, 1)] * 64), (2, [(9, 1)] * 100)]
    for _ in range(60):
        seqs = [(rng.choice([0, rng.randrange(5000)]), rng.choice([0, 1, rng.randrange(3000)]))
                for _ in range(rng.randrange(1, 70))]
        cases.append((rng.choice([2, 10, 25, 36, 64, 256]), seqs))
    src, exe = tmp_path / "geometry.cpp", tmp_path / "geometry"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    bounds = [(max(c for c, _ in s) + rng.choice([0, 700]), max(1, max(n for _, n in s))) for _, s in cases]
    text = "\n".join(f"{w} {len(s)} {mc} {mn} " + " ".join(f"{c} {n}" for c, n in s)
                     for (w, s), (mc, mn) in zip(cases, bounds))
    r = subprocess.run([str(exe)], input=text, capture_output=True, text=True)
    assert r.returncode == 0
    for (width, seqs), (mc, mn), line in zip(cases, bounds, r.stdout.strip("\n").split("\n")):
        step = (mc // width + mn // width + 2) // 32 + 1
        level = lambda c, i: (c // width + i) // step if 1 < len(seqs) <= 128 else 0
        blocks = sorted((-level(c, i), b, -i) for b, (c, n) in enumerate(seqs) for i in range(-(-n // width)))
        assert all(-l < 32 for l, _, _ in blocks)
        order = [f"{b},{-i}" for _, b, i in blocks]
        want = [x for u, x in enumerate(order) if u % 3 != 1] + order[1::3] + ["0"]
        assert line.split() == want, (width, seqs)


def test_even_shares_cover_every_unit_once(tmp_path):
    """The shares cut the units' key tiles without gaps; the merge finds a unit's pieces where their CTAs put them, at
    places of their own."""
    src, exe = tmp_path / "shares.cpp", tmp_path / "shares"
    src.write_text(r"""
#include <cstdio>
#include <vector>
#include "prompt_geometry.cuh"
int main() {
  int ctas, units, own, cut = 0;   // own: a unit's cells besides its key tiles
  while (std::scanf("%d %d %d", &ctas, &own, &units) == 3) {
    std::vector<int> n(units), first(units);
    int cells = 0, longest = 0, there = 0, shortest = 1 << 24;
    for (int i = 0; i < units; ++i) {
      if (std::scanf("%d", &n[i]) != 1) return 1;
      first[i] = cells;
      if (n[i] == 0) continue;
      cells += n[i] + own, ++there;
      longest = n[i] + own > longest ? n[i] + own : longest;
      shortest = n[i] + own < shortest ? n[i] + own : shortest;
    }
    const ptd::PromptCut c0 = ptd::prompt_cut(cells, there, longest, shortest, ctas, ctas, {1, own});
    const int shares = c0.shares;
    if (shares == 0) continue;
    ++cut;
    if (shares < 0 || shares > ctas || shares > cells / 2 || c0.cells != cells) return 2;
    std::vector<std::vector<int>> pieces(units);   // places, in order
    std::vector<int> taken(2 * shares, 0), tiles(units, 0);
    int next = 0;
    for (int c = 0; c < shares; ++c) {
      const int x0 = ptd::share_begin(c, c0), x1 = ptd::share_begin(c + 1, c0);
      if (x0 != next || x1 <= x0) return 3;
      for (int i = 0; i < units; ++i) {
        const int a = x0 > first[i] ? x0 : first[i], b = x1 < first[i] + n[i] ? x1 : first[i] + n[i];
        if (a >= b) continue;
        tiles[i] += b - a;
        if (a == first[i] && b == first[i] + n[i]) continue;   // whole
        const int place = 2 * c + (a > x0 ? 1 : 0);
        if (taken[place]++) return 4;
        pieces[i].push_back(place);
      }
      next = x1;
    }
    if (next != cells) return 5;
    for (int i = 0; i < units; ++i) {
      if (tiles[i] != n[i]) return 6;
      if (n[i] == 0) continue;
      const int c = ptd::share_of(first[i], c0), count = ptd::share_of(first[i] + n[i] - 1, c0) - c + 1;
      if (count == 1) {
        if (!pieces[i].empty()) return 7;
        continue;
      }
      if ((int)pieces[i].size() != count) return 8;
      for (int s = 0; s < count; ++s)
        if (pieces[i][s] != (s ? 2 * (c + s) : 2 * c + (ptd::share_begin(c, c0) < first[i] ? 1 : 0))) return 9;
      const int at = ptd::share_begin(c + 1, c0);   // the boundary at which the merge looks for it
      if (at <= first[i] || at >= first[i] + n[i]) return 10;
    }
  }
  if (ptd::prompt_cut(0, 0, 0, 1 << 24, 152, 152, {1, 1}).shares != 0 || ptd::prompt_cut(1, 1, 1, 1, 152, 152, {0, 0}).shares != 0) return 11;
  const int most = ptd::kMostCutCells;   // (no product leaves 32 bits)
  for (int units : {8, 100, 300, 510}) {
    const ptd::PromptCut c = ptd::prompt_cut(most, units, most / 2, 1, 255, 255, {4, 3});
    if (c.shares != 255 || ptd::share_begin(255, c) != most || ptd::share_of(most - 1, c) != 254 || ptd::share_of(0, c) != 0)
      return 12;
    if (ptd::prompt_cut(most, units, most / 2, 1, 255, 9, {4, 3}).shares != 9) return 14;   // (no room for more)
    if (ptd::prompt_cut(most + 1, units, most / 2, 1, 255, 255, {4, 3}).shares != 0) return 13;
  }
  std::printf("%d\n", cut);
  return 0;
}
""")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    rng = random.Random(9)
    cases = [(152, [20]), (152, [5000] * 8), (152, [33, 0, 1, 2] * 16), (3, [7, 8]), (1, [5, 6]), (152, [33] * 256),
             (255, [1 << 19] * 16), (152, [63] * 8), (152, [9] * 75), (152, [9] * 77)]
    for _ in range(400):
        top = rng.choice([2, 8, 40, 300])
        cases.append((rng.choice([1, 2, 7, 148, 152]), [rng.randrange(top + 1) for _ in range(rng.randrange(1, 400))]))
    r = subprocess.run([str(exe)], input="\n".join(f"{c} {rng.randrange(4)} {len(n)} " + " ".join(map(str, n)) for c, n in cases),
                       capture_output=True, text=True)
    assert r.returncode == 0 and int(r.stdout) > 50, (r.returncode, r.stdout)


TURNS = r"""
#include <cstdio>
#include <unordered_set>
#include <vector>
#include "prompt_geometry.cuh"
// Every interleaving of the two issuers and two softmax warps an M tile over a few units (n0, n1 key tiles), without the
// ring, which only holds them back.  Barriers count arrivals; an arrival carries the phase that it is meant for, and a
// wait passes on the phase's parity, as the hardware's does.  1: an arrival in another phase, or a wait let through by
// another phase; 2: a state that nobody leaves.
enum { kP = 0, kF = 2, kS = 4, kO = 6, kEntry = 8, kBars = 9 };
struct Op { bool wait; int bar, phase; };
const int counts[kBars] = {3, 3, 2, 2, 1, 1, 1, 1, 1};   // kP: two warps and the turn
int main() {
  const int kinds[8][2] = {{1, 0}, {2, 0}, {0, 1}, {0, 2}, {1, 1}, {1, 2}, {2, 2}, {2, 3}};
  long states = 0;
  for (int x = 0; x < 8 * 8 * 8; ++x) {
    std::vector<Op> ops[6];
    int first[2] = {0, 0}, outs[2] = {0, 0}, entries = 0;
    for (int u = 0; u < 3; ++u) {
      const int* n = kinds[u == 0 ? x % 8 : u == 1 ? x / 8 % 8 : x / 64];
      const int both = n[0] < n[1] ? n[0] : n[1], all = n[0] < n[1] ? n[1] : n[0];
      for (int t = 0; t < 2; ++t) {
        std::vector<Op>& o = ops[t];
        if (ptd::tells_entry(t, both)) o.push_back({false, kEntry, entries});
        if (n[t] > 0) o.push_back({false, kS + t, first[t]});
#ifndef PTD_NO_ENTRY
        if (ptd::awaits_entry(t, both)) o.push_back({true, kEntry, entries});
#endif
        for (int j = 0; j < all; ++j) {
          if (j >= n[t]) continue;
          if (ptd::own_turn(t, j, both)) o.push_back({false, kP + t, first[t] + j});
          o.push_back({true, kP + t, first[t] + j});
          o.push_back({true, kF + t, first[t] + j});
          if (ptd::passes_turn(t, j, both)) o.push_back({false, kP + (t ^ 1), first[t ^ 1] + j + t});
          if (j + 1 < n[t]) o.push_back({false, kS + t, first[t] + j + 1}); else o.push_back({false, kO + t, outs[t]});
        }
        for (int w = 0; w < 2 && n[t] > 0; ++w) {
          std::vector<Op>& q = ops[2 + 2 * t + w];
          for (int j = 0; j < n[t]; ++j) {
            q.push_back({true, kS + t, first[t] + j});
            q.push_back({false, kP + t, first[t] + j});
            q.push_back({false, kF + t, first[t] + j});
          }
          q.push_back({true, kO + t, outs[t]});
        }
      }
      for (int t = 0; t < 2; ++t) first[t] += n[t], outs[t] += n[t] > 0;
      entries += both > 0;
    }
    std::unordered_set<unsigned long long> seen = {0};
    std::vector<unsigned long long> todo = {0};   // the processes' places, a byte each
    while (!todo.empty()) {
      const unsigned long long at = todo.back();
      todo.pop_back();
      ++states;
      int arrived[kBars] = {};
      for (int i = 0; i < 6; ++i)
        for (int k = 0; k < (int)(at >> 8 * i & 255); ++k)
          if (!ops[i][k].wait) ++arrived[ops[i][k].bar];
      bool done = true, moved = false;
      for (int i = 0; i < 6; ++i) {
        const int k = (int)(at >> 8 * i & 255);
        if (k == (int)ops[i].size()) continue;
        done = false;
        const Op& o = ops[i][k];
        const int phase = arrived[o.bar] / counts[o.bar];
        if (o.wait) {
          if ((phase & 1) == (o.phase & 1)) continue;   // (the phase of this parity is open)
          if (phase != o.phase + 1) return 1;
        } else if (phase != o.phase) {
          return 1;
        }
        moved = true;
        const unsigned long long next = at + (1ull << 8 * i);
        if (seen.insert(next).second) todo.push_back(next);
      }
      if (!moved && !done) return 2;
    }
  }
  std::printf("%ld\n", states);
  return 0;
}
"""


def test_issuers_turns_meet_their_own_phase(tmp_path):
    """No turn of one unit counts for a wait of another, whatever the order in which the warps run; and the model finds
    the turn that comes early where issuer 0 does not wait for issuer 1 to begin a unit."""
    src = tmp_path / "turns.cpp"
    src.write_text(TURNS)
    for name, flags, code in (("turns", [], 0), ("early", ["-DPTD_NO_ENTRY"], 1)):
        exe = tmp_path / name
        subprocess.run(["g++", "-O2", "-std=c++17", *flags, "-I", os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), str(src),
                        "-o", str(exe)], check=True)
        r = subprocess.run([str(exe)], capture_output=True, text=True)
        assert r.returncode == code, (name, r.returncode, r.stdout)
        assert code or int(r.stdout) > 10 ** 5


def test_index_division_is_exact(tmp_path):
    src, exe = tmp_path / "divide.cpp", tmp_path / "divide"
    src.write_text(r"""
#include <cstdio>
#include "row_division.cuh"
int main() {
  for (int64_t d = 1; d < (1ll << 31); d += d < 5000 ? 1 : d / 97 + 1) {
    const ptd::IndexDivisor x = ptd::index_divisor((int)d);
    const int64_t top = (1ll << 31) - 1;
    const int64_t qs[] = {0, 1, 2, 1000, 65535, top / d - 1, top / d};
    for (int64_t q : qs) {
      const int64_t ns[] = {q * d - 1, q * d, q * d + d / 2, q * d + d - 1, top};
      for (int64_t n : ns)
        if (n >= 0 && n <= top && ptd::divide((int)n, x) != n / d) return std::printf("%ld / %ld\n", (long)n, (long)d), 1;
    }
  }
  return 0;
}
""")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_sequences_out_of_bounds(tmp_path):
    src, exe = tmp_path / "ok.cpp", tmp_path / "ok"
    src.write_text(r"""
#include <cstdio>
#include "prompt_geometry.cuh"
int main() {
  const ptd::PromptBounds p = {100, 40, 1000, 1020};
  const int c[][4] = {{0, 40, 0, 1},   {0, 41, 0, 0},    {60, 100, 980, 1}, {60, 100, 981, 0}, {61, 101, 0, 0},
                      {-1, 3, 0, 0},   {5, 4, 0, 0},     {5, 5, 1000, 1},   {5, 5, 1001, 0},   {5, 6, -1, 0},
                      {0, 0, 0, 1},    {2147483647, -2147483647, 0, 0},     {0, 20, 1000, 1},  {0, 21, 1000, 0}};
  for (auto& x : c)
    if (ptd::prompt_sequence_ok(p, x[0], x[1], x[2]) != (x[3] == 1)) return std::printf("%d %d %d\n", x[0], x[1], x[2]), 1;
  return 0;
}
""")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


A = 1 << 24   # stands for device memory: host checks never read it


def _prompt(ptd, batch=2, total=10, max_tokens=8, max_ctx=100, offsets=A, ctx=A + 4096):
    return ptd._Prompt(batch, total, max_tokens, max_ctx, offsets, ctx)


def _cache(ptd, page=16, dtype=None, hkv=8, d=128, layers=2, num_pages=40, max_pages=10, k=2 * A):
    dt = ptd.BF16 if dtype is None else dtype
    return ptd._Cache(k, 3 * A, dt, layers, hkv, d, page, 0 if page else 300, num_pages if page else 0,
                      A + 8192 if page else None, max_pages if page else 0)


def test_prompt_slots_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    def call(prompt, cache, pool="default", slots=4 * A, positions=5 * A, status=6 * A):
        if pool == "default":
            pool = ptd._PagePool(7 * A, 8 * A, 9 * A, 10 * A, 11 * A, cache.block_table)
        return lib.ptd_prompt_slots(ctypes.byref(prompt) if prompt else None, ctypes.byref(cache),
                                    ctypes.byref(pool) if pool else None, slots, positions, status, None)

    ok_p, ok_c = _prompt(ptd), _cache(ptd)
    bad = ptd.INVALID_ARG
    assert call(None, ok_c) == bad
    for p in (_prompt(ptd, batch=0), _prompt(ptd, total=0), _prompt(ptd, max_tokens=0), _prompt(ptd, max_ctx=-1),
              _prompt(ptd, offsets=None), _prompt(ptd, ctx=None)):
        assert call(p, ok_c) == bad
    for p in (_prompt(ptd, batch=8193), _prompt(ptd, max_tokens=2**31 - 1), _prompt(ptd, max_ctx=2**30 - 7),
              _prompt(ptd, total=2**30 + 1)):
        assert call(p, ok_c) == ptd.UNSUPPORTED
    for pool in (None, "default"):   # slots on positions, the offsets, the contexts, the block table
        assert call(ok_p, ok_c, pool=pool, positions=4 * A + 36) == bad
        for at in (A + 8, A + 4096 - 36, A + 8192 + 76):
            assert call(ok_p, ok_c, pool=pool, slots=at) == bad and call(ok_p, ok_c, pool=pool, positions=at) == bad
    assert call(ok_p, ok_c, slots=None) == bad and call(ok_p, ok_c, positions=None) == bad
    assert call(ok_p, ok_c, status=None) == bad
    assert call(ok_p, _cache(ptd, page=0), pool=ptd._PagePool(7 * A, 8 * A, 9 * A, 10 * A, 11 * A, None)) == bad
    assert call(ok_p, _cache(ptd, page=24)) == ptd.UNSUPPORTED
    assert call(ok_p, _cache(ptd, num_pages=1 << 28)) == ptd.UNSUPPORTED            # 2^32 rows a layer
    assert call(_prompt(ptd, batch=4096), _cache(ptd, max_pages=1 << 20)) == ptd.UNSUPPORTED
    for i in range(6):   # each member missing
        m = [7 * A, 8 * A, 9 * A, 10 * A, 11 * A, ok_c.block_table]
        m[i] = None
        assert call(ok_p, ok_c, pool=ptd._PagePool(*m)) == bad
    t = ok_c.block_table
    for m in ((7 * A, 8 * A, 9 * A, 9 * A, 11 * A, t), (7 * A, 8 * A, 9 * A, 9 * A + 4, 11 * A, t),   # new_held on held
              (7 * A, 8 * A, 9 * A, 10 * A, 8 * A, t),                                                # new count on count
              (7 * A, 7 * A + 8, 9 * A, 10 * A, 11 * A, t),                                           # count in the stack
              (7 * A, 8 * A, 9 * A, 10 * A, 11 * A, 12 * A),                                          # another table
              (4 * A + 8, 8 * A, 9 * A, 10 * A, 11 * A, t)):                                          # slots on the stack
        assert call(ok_p, ok_c, pool=ptd._PagePool(*m)) == bad, m


def test_prompt_rope_append_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    def call(cache=None, layer=0, slots=4 * A, positions=5 * A, q=7 * A, qs=4096, hq=32, k=8 * A, ks=1024, v=9 * A, vs=1024,
             base=1e4, out=10 * A, outs=4096, status=6 * A):
        return lib.ptd_prompt_rope_append(ctypes.byref(_prompt(ptd)), ctypes.byref(cache or _cache(ptd)), layer, slots,
                                          positions, q, qs, hq, k, ks, v, vs, base, out, outs, status, None)

    for kw in (dict(layer=-1), dict(layer=2), dict(slots=None), dict(positions=None), dict(q=None), dict(k=None),
               dict(v=None), dict(out=None), dict(status=None), dict(qs=4095), dict(ks=1023), dict(vs=0), dict(outs=-4096),
               dict(hq=30), dict(hq=0), dict(base=1.0), dict(base=float("inf")), dict(base=float("nan")),
               dict(q=7 * A + 1), dict(out=10 * A + 1), dict(out=7 * A, qs=5000),
               dict(cache=_cache(ptd, d=127, hkv=16), qs=10**6, ks=10**6, vs=10**6),
               dict(cache=_cache(ptd, d=264), qs=10**6, outs=10**6, ks=10**6, vs=10**6)):
        assert call(**kw) == ptd.INVALID_ARG, kw
    # 2^31 elements a token
    assert call(hq=2**24 - 16, qs=2**31, outs=2**31) == ptd.UNSUPPORTED
    # cache rows of 24 bytes: not a multiple of 16
    assert call(cache=_cache(ptd, dtype=ptd.F32, hkv=1, d=6)) == ptd.UNSUPPORTED


def test_prompt_attention_refusals(lib):
    from paper_2607_10661_gb300 import ptd

    def call(prompt=None, cache=None, layer=0, q=7 * A, qs=4096, hq=32, out=8 * A, status=6 * A):
        return lib.ptd_prompt_attention(ctypes.byref(prompt or _prompt(ptd)), ctypes.byref(cache or _cache(ptd)), layer, q, qs,
                                        hq, 0.0, out, None, 0, status, None)

    for kw in (dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(status=None), dict(qs=4095), dict(qs=4097),
               dict(hq=30), dict(hq=0), dict(q=7 * A + 2), dict(out=8 * A + 8), dict(prompt=_prompt(ptd, batch=0)),
               dict(cache=_cache(ptd, k=2 * A + 8))):
        assert call(**kw) == ptd.INVALID_ARG, kw
    for kw in (dict(cache=_cache(ptd, d=64)), dict(cache=_cache(ptd, dtype=ptd.F32, d=96)), dict(cache=_cache(ptd, page=8)),
               dict(prompt=_prompt(ptd, batch=8193))):
        assert call(**kw) == ptd.UNSUPPORTED, kw
    size = lambda p, c, hq=32: lib.ptd_prompt_attention_workspace_size(ctypes.byref(p), ctypes.byref(c), hq)
    assert size(_prompt(ptd), _cache(ptd), 30) == 0 and size(_prompt(ptd), _cache(ptd, d=64)) == 0
    # a token far into a sequence: its keys are split; a prompt that fills the SMs by itself: none
    assert size(_prompt(ptd, 1, 1, 1, 30000), _cache(ptd, page=0)) > 0
    assert size(_prompt(ptd, 1, 20000, 20000, 0), _cache(ptd, page=0)) == 0


def test_oracle_pages_by_hand():
    """Pages of 16: sequence 0 (20 + 13 positions) has 2 pages and needs 3, sequence 1 is finished and gives 7 and
    9 back, sequence 2 is new and needs 2, sequence 3 stays in its page."""
    table = [[4, 2, -1], [7, 9, -1], [-1, -1, -1], [5, -1, -1]]
    t, held, free = oracle.prompt_pages([20, 0, 0, 3], [13, 0, 17, 1], [2, 2, 0, 1], table, [11, 8], 16)
    assert t == [[4, 2, 9], [7, 9, -1], [7, 8, -1], [5, -1, -1]] and held == [3, 0, 2, 1] and free == [11]
    assert oracle.prompt_pages([20, 0, 0, 3], [13, 0, 65, 1], [2, 2, 0, 1], [r + [-1] * 3 for r in table], [11, 8], 16) is None
    slots, pos = oracle.prompt_slots([20, 0, 0, 3], [13, 0, 17, 1], t, 16)
    assert slots[:13] == [2 * 16 + 4 + i for i in range(12)] + [9 * 16] and pos[:13] == list(range(20, 33))
    assert slots[13:] == [7 * 16 + i for i in range(16)] + [8 * 16, 5 * 16 + 3] and pos[-1] == 3
    assert oracle.prompt_slots([2, 5], [2, 1], None, -50)[0] == [2, 3, 55]


def test_oracle_causal_attention_is_a_chain_tree():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((9, 4, 8)), rng.standard_normal((14, 2, 8)), rng.standard_normal((14, 2, 8))
    o, size = oracle.causal_attention(q, k, v, 5)
    want = oracle.tree_attention(q, k, v, [-1] + list(range(8)), 5)
    assert np.abs(o - want).max() < 1e-14 and (size >= np.abs(o) - 1e-15).all()
    one, _ = oracle.causal_attention(q[:1], k, v, 0)
    assert np.array_equal(one[0], np.repeat(v[0], 2, axis=0))


@pytest.mark.parametrize("name,count", [("prompt_slots", 7), ("prompt_rope_append", 12), ("prompt_attention", 9)])
def test_native_prompt_calls_leave_other_arguments_alone(lib, name, count):
    """Host tensors, plain objects and wrong counts are not taken (None: nothing was enqueued)."""
    import torch

    from paper_2607_10661_gb300 import ptd

    f = getattr(ptd._native(), name)
    host = torch.zeros((2, 4), dtype=torch.int32)
    for filler in (host, None, 3, [1, 2], 0.5):
        assert f(*([filler] * count)) is None
    assert f() is None and f(*([host] * (count + 1))) is None


def _native_with(ptd, monkeypatch, tensors_on, current):
    """The native calls with a stand-in tensor type on device `tensors_on` while `current` is the current device."""
    import torch

    class Fake:
        is_cuda, dtype, nbytes, shape = True, torch.int32, 40, (10, 2, 128)

        def __init__(self, dtype=torch.int32, device=tensors_on):
            self.dtype, self.device_ = dtype, device

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return A

        def stride(self):
            return (256, 128, 1)

        def get_device(self):
            return self.device_

    calls = ptd._native()
    calls.load(ptd.LIB_PATH, Fake, torch.int32, torch.float32, torch.bfloat16, lambda d: 0, lambda: current)
    return calls, Fake


def test_native_prompt_calls_keep_to_the_current_device(lib, monkeypatch):
    """Tensors of another device than the current one, or of several, are left to the path that changes the
    device or raises (the calls that are taken here end at the library's own checks: no layer 9, no status)."""
    import torch

    from paper_2607_10661_gb300 import ptd

    class Holder:
        def __init__(self, c, k=None, ctx_lens=None):
            self.c, self.k, self.block_table, self.ctx_lens = c, k, None, ctx_lens

    try:
        for here, current, stray in ((0, 0, None), (1, 1, None), (1, 0, None), (0, 0, "k"), (0, 0, "q"), (0, 0, "ctx")):
            calls, Fake = _native_with(ptd, monkeypatch, here, current)
            prompt = Holder(_prompt(ptd), None, Fake(device=1 - here if stray == "ctx" else here))
            cache = Holder(_cache(ptd, page=0, hkv=2), Fake(torch.bfloat16, 1 - here if stray == "k" else here))
            q, x, i = Fake(torch.bfloat16, 1 - here if stray == "q" else here), Fake(torch.bfloat16), Fake()
            taken = here == current and stray is None
            want = -ptd.INVALID_ARG if taken else None
            assert calls.prompt_attention(prompt, cache, 9, q, x, i, 0.0, None, 0) == want
            # (the rotary call reads nothing of the batch on the device)
            assert calls.prompt_rope_append(prompt, cache, 9, i, i, q, x, x, x, 1e4, i, 0) == \
                (want if stray != "ctx" else -ptd.INVALID_ARG)
            prompt.c.batch = 0   # refused by the library
            assert calls.prompt_slots(prompt, cache, None, i, i, i, 0) == (want if stray != "q" else -ptd.INVALID_ARG)
    finally:
        ptd._calls = None
        ptd._native()


def test_no_call_sets_a_kernels_limits_by_its_own_size():
    """Attributes belong to the kernel: threads that set them by their call's sizes undo one another's, so that every
    limit of dynamic shared memory is a constant."""
    csrc, found = os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), 0
    for name in sorted(os.listdir(csrc)):
        text = open(os.path.join(csrc, name)).read() if name.endswith((".cu", ".cuh")) else ""
        for m in re.finditer(r"cudaFuncAttributeMaxDynamicSharedMemorySize,([^;]*);", text):
            found += 1
            value = re.sub(r"[\\\s]", "", m.group(1))
            assert re.fullmatch(r"\(int\)([\w<>,]+::)*k[A-Z]\w*\)", value), (name, value)
    assert found >= 8


def test_batches_that_are_not_the_caches_are_refused(lib, monkeypatch):
    """A contiguous cache of another number of sequences (its layers would begin elsewhere), a block table of too few
    rows: not taken natively, and a ValueError of each call otherwise."""
    import types

    import torch

    from paper_2607_10661_gb300 import ptd

    class Refuse:
        def __getattr__(self, name):
            return lambda *a: None

    shapes = ((0, (2, 2), True), (0, (2, 1), False), (0, (2, 3), False), (16, (2, 10), True), (16, (3, 10), True),
              (16, (1, 10), False))
    try:
        for page, shape, good in shapes:
            calls, Fake = _native_with(ptd, monkeypatch, 0, 0)
            i, x = Fake(), Fake(torch.bfloat16)
            prompt = types.SimpleNamespace(c=_prompt(ptd), ctx_lens=Fake(), batch=2, total_tokens=10)
            cache = types.SimpleNamespace(c=_cache(ptd, page=page, hkv=2), page_size=page, k=Fake(torch.bfloat16),
                                          block_table=Fake() if page else None, head_dim=128, num_kv_heads=2)
            (cache.block_table if page else cache.k).shape = shape if page else shape + (300, 2, 128)
            want = -ptd.INVALID_ARG if good else None   # (taken: layer 9, slots on positions)
            assert calls.prompt_attention(prompt, cache, 9, x, x, i, 0.0, None, 0) == want, shape
            assert calls.prompt_rope_append(prompt, cache, 9, i, i, x, x, x, x, 1e4, i, 0) == want, shape
            assert calls.prompt_slots(prompt, cache, None, i, i, i, 0) == want, shape
            if good:
                continue
            with monkeypatch.context() as m:
                m.setattr(ptd, "_calls", Refuse())
                for call in (lambda: ptd.prompt_attention(prompt, cache, 9, x, x, i, stream=0),
                             lambda: ptd.prompt_rope_append(prompt, cache, 9, i, i, x, x, x, x, 1e4, i, stream=0),
                             lambda: ptd.prompt_slots(prompt, cache, i, i, i, stream=0)):
                    with pytest.raises(ValueError, match="sequences"):
                        call()
    finally:
        ptd._calls = None
        ptd._native()


def test_rows_in_memory_meet(tmp_path):
    """Against the sets of bytes, for every pair of small sets of rows; only sets of different steps may be said to meet
    where they interleave."""
    src, exe = tmp_path / "rows.cpp", tmp_path / "rows"
    src.write_text(r"""
#include <cstdio>
#include <vector>
#include "memory_rows.cuh"
int main() {
  struct S { long at, bytes, step, count; };
  std::vector<S> sets;
  for (long bytes : {0, 1, 3, 5})
    for (long step : {5, 6, 7, 12})
      for (long count : {1, 2, 4})
        sets.push_back({0, bytes, step, count});
  auto covers = [](const S& s, long x) {
    for (long i = 0; i < s.count; ++i)
      if (x >= s.at + i * s.step && x < s.at + i * s.step + s.bytes) return true;
    return false;
  };
  long met = 0, apart = 0;
  for (const S& a0 : sets)
    for (const S& b0 : sets)
      for (long shift = -60; shift <= 60; ++shift) {
        S a = a0, b = b0;
        a.at = 100, b.at = 100 + shift;
        bool want = false;
        for (long x = 0; x < 300 && !want; ++x) want = covers(a, x) && covers(b, x);
        const auto rows = [](const S& s) { return ptd::memory_rows(reinterpret_cast<const void*>(s.at), s.bytes, s.step, s.count); };
        const bool got = ptd::rows_meet(rows(a), rows(b));
        const bool exact = a.count == 1 || b.count == 1 || a.step == b.step;
        if (exact ? got != want : want && !got) return std::printf("%ld+%ldx%ld/%ld %ld+%ldx%ld/%ld\n", a.at, a.bytes, a.count, a.step, b.at, b.bytes, b.count, b.step), 1;
        ++(want ? met : apart);
      }
  const auto far = ptd::memory_rows(reinterpret_cast<const void*>(1l << 40), 256, 1l << 31, 1 << 30);   // spans 2^61
  if (ptd::rows_meet(far, ptd::memory_rows(reinterpret_cast<const void*>((1l << 40) + (1l << 50) + 256), 300))) return 2;
  if (!ptd::rows_meet(far, ptd::memory_rows(reinterpret_cast<const void*>((1l << 40) + (1l << 50) + 255), 300))) return 3;
  std::printf("%ld %ld\n", met, apart);
  return 0;
}
""")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and min(map(int, r.stdout.split())) > 1000, (r.returncode, r.stdout)


def test_overlaps_are_refused(lib):
    """What a call writes on what it reads: refused before anything is launched."""
    from paper_2607_10661_gb300 import ptd

    p = _prompt(ptd)   # 10 tokens
    paged, plain = _cache(ptd), _cache(ptd, page=0)
    row, kv = 32 * 128 * 2, 1024 * 2

    def rope(q=7 * A, qs=4096, k=8 * A, ks=1024, v=9 * A, vs=1024, out=10 * A, outs=4096):
        return lib.ptd_prompt_rope_append(ctypes.byref(p), ctypes.byref(paged), 0, 4 * A, 5 * A, q, qs, 32, k, ks, v, vs, 1e4, out,
                                          outs, 6 * A, None)

    for kw in (dict(out=7 * A + row), dict(out=7 * A - 16), dict(out=7 * A + 10 * row - 16), dict(out=8 * A), dict(out=9 * A + kv),
               dict(out=8 * A + 16 - 10 * row), dict(out=7 * A, k=7 * A + 4 * row), dict(out=7 * A, qs=6144, outs=6144, v=7 * A + row - 16, vs=6144),
               dict(out=7 * A, qs=6144), dict(out=7 * A + 2 * row, qs=6144, outs=6144), dict(qs=2**62), dict(outs=2**61)):
        assert rope(**kw) == ptd.INVALID_ARG, kw

    def attention(cache=paged, q=7 * A, qs=4096, out=8 * A, ws=None, wsb=0, prompt=p):
        return lib.ptd_prompt_attention(ctypes.byref(prompt), ctypes.byref(cache), 0, q, qs, 32, 0.0, out, ws, wsb, 6 * A, None)

    layers = 2 * 40 * 16 * kv
    for kw in (dict(out=7 * A), dict(out=7 * A + 16), dict(out=7 * A + 9 * row), dict(out=7 * A - 9 * row), dict(qs=6144, out=7 * A + 6144 * 2),
               dict(out=2 * A), dict(out=2 * A + layers - 16), dict(out=3 * A + layers // 2), dict(out=A), dict(out=A + 4096), dict(out=A + 8192),
               dict(cache=plain, out=3 * A + 2 * 300 * 2 * kv - 16), dict(qs=2**62)):
        assert attention(**kw) == ptd.INVALID_ARG, kw
    far = _prompt(ptd, 1, 1, 1, 30000)   # cut into pieces
    long = _cache(ptd, max_pages=2000)
    need = lib.ptd_prompt_attention_workspace_size(ctypes.byref(far), ctypes.byref(long), 32)
    assert need > 0
    for ws in (8 * A, 7 * A, 8 * A + 16 - need, 7 * A - need + 256, 2 * A + 64, A):
        assert attention(cache=long, prompt=far, ws=ws, wsb=need) == ptd.INVALID_ARG, ws

    t = paged.block_table
    for pool in (None, ptd._PagePool(7 * A, 8 * A, 9 * A, 10 * A, 11 * A, t)):
        on = [4 * A, 5 * A + 36, A, A + 4096, t + 4] + ([] if pool is None else [7 * A + 156, 8 * A, 9 * A + 4, 10 * A, 11 * A])
        for status in on:
            assert lib.ptd_prompt_slots(ctypes.byref(p), ctypes.byref(paged), ctypes.byref(pool) if pool else None, 4 * A, 5 * A,
                                        status, None) == ptd.INVALID_ARG, status


def test_scratch_is_sized_for_the_tensors_device(monkeypatch):
    """The size is asked for while the tensors' device is the current one; tensors of two devices are refused."""
    import types

    import torch

    from paper_2607_10661_gb300 import ptd

    current = [0]

    class Guard:
        def __init__(self, device):
            self.device = device.index

        def __enter__(self):
            self.before, current[0] = current[0], self.device

        def __exit__(self, *exc):
            current[0] = self.before

    asked = []
    size = lambda *a: asked.append(current[0]) or 4096
    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(ptd, "lib", lambda: types.SimpleNamespace(ptd_prompt_attention_workspace_size=size))
    on = lambda d: types.SimpleNamespace(device=torch.device("cuda", d))
    prompt, cache = types.SimpleNamespace(c=_prompt(ptd), ctx_lens=on(1)), types.SimpleNamespace(c=_cache(ptd), k=on(1))
    assert ptd.prompt_attention_workspace_size(prompt, cache, 32) == 4096 and asked == [1] and current == [0]
    cache.k = on(0)
    with pytest.raises(ValueError, match="devices"):
        ptd.prompt_attention_workspace_size(prompt, cache, 32)


def test_a_cache_of_several_devices_is_refused():
    """The prompt calls compare the other tensors' device with k's; v and the block table are on it too."""
    import types

    import torch

    from paper_2607_10661_gb300 import ptd

    on = lambda d: types.SimpleNamespace(shape=(1, 2, 16, 2, 128), dtype=torch.bfloat16, device=torch.device("cuda", d))
    for k, v, table in ((0, 1, 0), (0, 0, 1), (1, 0, 0)):
        with pytest.raises(ValueError, match="devices"):
            ptd.KVCache(on(k), on(v), 2, 128, 16, on(table))
    with pytest.raises(ValueError, match="devices"):
        ptd.KVCache(on(0), on(1), 2, 128)


def test_partials_have_places_of_their_own(tmp_path):
    """block_place + block: distinct over a batch's blocks and below prompt_places, with padding before, behind and in
    the sequences' sizes; below it even where offsets decrease (sequences that are valid by themselves then overlap)."""
    src, exe = tmp_path / "places.cpp", tmp_path / "places"
    src.write_text(r"""
#include <cstdio>
#include <set>
#include "prompt_geometry.cuh"
int main() {
  int width, total, batch, ordered, most = 0;
  while (std::scanf("%d %d %d %d", &width, &total, &batch, &ordered) == 4) {
    static int off[5000];
    for (int b = 0; b <= batch; ++b)
      if (std::scanf("%d", off + b) != 1) return 1;
    const ptd::IndexDivisor by = ptd::index_divisor(width);
    const ptd::PromptBounds bounds = {total, total, 0, total};
    const long places = ptd::prompt_places(total, batch, width);
    std::set<long> taken;
    for (int b = 0; b < batch; ++b) {
      if (!ptd::prompt_sequence_ok(bounds, off[b], off[b + 1], 0)) {
        if (ordered) return 2;
        continue;
      }
      const int count = ptd::prompt_blocks(0, off[b + 1] - off[b], width, by).count;
      for (int i = 0; i < count; ++i) {
        const long place = ptd::block_place(off[b], b, by) + i;
        if (place < 0 || place >= places) return 3;
        if (!taken.insert(place).second && ordered) return 4;
        if (place == places - 1) ++most;
      }
    }
  }
  std::printf("%d\n", most);
  return 0;
}
""")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2607_10661_gb300", "csrc"), str(src),
                    "-o", str(exe)], check=True)
    rng = random.Random(14)
    lines = ["2 128 128 1 " + " ".join(map(str, range(129))), "64 1 1 1 0 1", "64 128 2 1 0 64 128", "7 5 3 1 5 5 5 5"]
    for _ in range(800):
        width, batch = rng.choice([1, 2, 3, 10, 16, 25, 36, 64, 256]), rng.randrange(1, 200)
        off = [rng.choice([0, rng.randrange(50)])]
        for _ in range(batch):
            off.append(off[-1] + rng.choice([0, 1, 1, rng.randrange(1, 3 * width + 2)]))
        total = max(off[-1] + rng.choice([0, 0, rng.randrange(300)]), 1)
        ordered = rng.random() < 0.7
        if not ordered:
            for _ in range(rng.randrange(1, 20)):
                off[rng.randrange(batch + 1)] = rng.randrange(-3, total + 4)
        lines.append(f"{width} {total} {batch} {int(ordered)} " + " ".join(map(str, off)))
    r = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True)
    assert r.returncode == 0 and int(r.stdout) > 20, (r.returncode, r.stdout)   # (the last place is taken too)


def test_tree_calls_refuse_batches_beyond_the_cache(lib, monkeypatch):
    """More trees than the cache's sequences, or fewer beyond the first layer of a contiguous cache: refused before
    anything is called; the others go on to the call."""
    import types

    from paper_2607_10661_gb300 import ptd

    class Reached(Exception):
        pass

    class Calls:
        def __getattr__(self, name):
            def call(*a):
                raise Reached

            return call

    monkeypatch.setattr(ptd, "_calls", Calls())
    monkeypatch.setattr(ptd, "lib", Calls)
    monkeypatch.setattr(ptd, "_dev", lambda *a, **k: 0)
    x = types.SimpleNamespace(dim=lambda: 3, c=ptd._StepArgs(), t=None)
    io = types.SimpleNamespace(c=ptd._HostIO())
    for page, sequences, batch, layers, layer, good in ((0, 3, 3, 2, 1, True), (0, 3, 4, 1, 0, False), (0, 3, 2, 1, 0, True),
                                                        (0, 3, 2, 2, 1, False), (16, 3, 2, 2, 1, True), (16, 3, 4, 2, 0, False)):
        tree = types.SimpleNamespace(batch=batch, c=ptd._Tree())
        k = types.SimpleNamespace(dtype=None)
        cache = types.SimpleNamespace(sequences=sequences, page_size=page, num_layers=layers, k=k, c=ptd._Cache())
        for call in (lambda: ptd.tree_attention(tree, cache, x, x, 8, x, layer_begin=layer, num_layers=1, stream=0),
                     lambda: ptd.tree_attention_as(1, 0, tree, cache, x, x, 8, x, layer_begin=layer, num_layers=1, stream=0),
                     lambda: ptd.tree_rope_append(tree, cache, layer, x, 8, x, x, 1e4, x, stream=0),
                     lambda: ptd.kv_compact(tree, cache, x, x, x, stream=0),
                     lambda: ptd.verify_and_compact(tree, cache, x, x, 1, x, x, x, x, x, stream=0),
                     lambda: ptd.tree_verify_step(tree, cache, x, stream=0),
                     lambda: ptd.tree_verify_step_host(tree, cache, x, io, stream=0),
                     lambda: ptd.Pipeline(cache, [tree, tree], [x, x], [types.SimpleNamespace(numel=lambda: 1, element_size=lambda: 1)] * 2,
                                          stream=0)):
            with pytest.raises(Reached if good else ValueError):
                call()
    # a lone first layer takes fewer trees
    tree = types.SimpleNamespace(batch=2, c=ptd._Tree())
    cache = types.SimpleNamespace(sequences=3, page_size=0, num_layers=2, k=k, c=ptd._Cache())
    with pytest.raises(Reached):
        ptd.tree_attention(tree, cache, x, x, 8, x, layer_begin=0, num_layers=1, stream=0)
