"""Which kernels, tiles and parts the log probabilities of given tokens and their gradients take for a size: the device's division of the
work and the products' choice of tiles from their own headers, compiled for the host, the rest restated.  Nothing here uses the library."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2601_06562_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CUS, IDS = 256, 256                                   # compute units; ids of a tile
MOST_IDS, DL_BYTES, LOW_ROWS = 1 << 18, 256 << 20, 32
STREAM_BYTES = 288 << 20

PROGRAM = r"""
#include <stdio.h>
#include "mosaic_schedule.h"
#include "mosaic_ffn_choice.h"
using namespace mosaic;
static void product(int mode, long long rows_p, long long rows_q, long long steps, long long splits) {
  const int t = ffn::choose_tile(mode, rows_p, rows_q, steps, splits).tile;
  const ffn::TileGrid g = ffn::tile_grid(mode, t, rows_p, rows_q, splits);
  printf("%d %d %d\n", t, g.n > g.blocks, g.blocks);
}
int main() {
  char what;
  long long a, b, c, e;
  while (scanf(" %c %lld %lld %lld %lld", &what, &a, &b, &c, &e) == 5) {
    if (what == 'S') {          // tiles of the vocabulary, steps of K, rows, room of the partial arrays
      ScheduleInput in{};
      in.vocab_tiles = (uint32_t)a;
      in.k_tiles = (uint32_t)b;
      in.widths = 0xff;
      in.grid = 256;
      in.slots64 = (uint32_t)e;
      const Schedule s = choose_schedule(in, (int32_t)c);
      printf("%d %d %d\n", s.width, s.row_tiles, s.splits);
    } else if (what == 'X') {   // columns, rows, steps, parts
      product(ffn::kOneDx, a, b, c, e);
    } else if (what == 'W') {   // columns, ids, steps
      product(ffn::kOneDw, a, b, c, 1);
    } else {                    // rows, columns, depth: the parts of K
      const int64_t steps = ffn::tiles(c, ffn::kStepK);
      int best = 1;
      double least = 0.0;
      for (int s = 1; s == 1 || (s <= ffn::kMostParts && s * a <= ffn::kPartRows && s * 4 <= steps); ++s) {
        const double us = ffn::choose_tile(ffn::kOneDx, b, a, steps, s).us + (double)(a * b) * 8.0 * s / ffn::kJoinBytesPerUs;
        if (s == 1 || us < least) best = s, least = us;
      }
      printf("%d 0 0\n", best);
    }
  }
}
"""


class Choice:
    def __init__(self, folder):
        src, self.exe, self.known = os.path.join(folder, "choice.hip"), os.path.join(folder, "choice"), {}
        with open(src, "w") as f:
            f.write(PROGRAM)
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                        "-o", self.exe, src], check=True, stderr=subprocess.DEVNULL)

    def ask(self, questions):
        new = [q for q in dict.fromkeys(questions) if q not in self.known]
        if new:
            lines = subprocess.run([self.exe], input="\n".join("%s %d %d %d %d" % q for q in new), text=True, check=True,
                                   stdout=subprocess.PIPE).stdout.splitlines()
            assert len(lines) == len(new)
            self.known.update((q, tuple(int(v) for v in line.split())) for q, line in zip(new, lines))
        return [self.known[q] for q in questions]


def up(n, by):
    return -(-n // by)


def four_waves(d, V):
    """Whether the 4-wave loop takes these sizes."""
    return d % 64 == 0 and V >= IDS and (V % IDS == 0 or d // 64 >= 5)


def tile_rows(rows):
    """Rows of a tile of the eight-wave kernel."""
    if rows <= 128:
        return 64 if rows <= 64 else 128
    return 128 if 92 * up(rows, 128) < 150 * up(rows, 256) else 256


def parts_of(row_tiles, vocab_tiles, steps):
    """Parts of the vocabulary there."""
    best = None
    for s in range(1, 257):
        if s > vocab_tiles or (s > 1 and row_tiles * s > 512):
            break
        cost = min(up(row_tiles * s, CUS) * (up(vocab_tiles, s) * steps + 2), 0x7fffff)
        best = (cost, s) if best is None or cost < best[0] else best
    return best[1]


def forward_question(rows, d, V, bound=None):
    vocab_tiles, row_tiles = up(V, IDS), up(bound or rows, 256)
    units = min(max(4 * row_tiles + CUS, 2 * CUS), row_tiles * min(vocab_tiles, 256))
    return ("S", vocab_tiles, d // 64, rows, 4 * units)


def forward_ways(choice, sizes):
    """Per size (rows, d, V, n_top): what it runs.  (kernel, width or rows of a tile, whether a unit has several tiles, whether the
    weights are streamed, whether a block takes several units)."""
    answers = iter(choice.ask([forward_question(r, d, V) for r, d, V, _ in sizes if four_waves(d, V)]))
    out = []
    for rows, d, V, n_top in sizes:
        name = "alternatives" if n_top else "statistics"
        vocab_tiles = up(V, IDS)
        if four_waves(d, V):
            width, row_tiles, splits = next(answers)
            out.append((name + " 4", width, up(vocab_tiles, splits) > 1, row_tiles == 1 and V * d * 2 > STREAM_BYTES, row_tiles * splits > CUS))
        else:
            tile = min(tile_rows(rows), 128) if n_top else tile_rows(rows)
            parts = parts_of(up(rows, tile), vocab_tiles, up(d, 64))
            out.append((name + " 8", tile, up(vocab_tiles, parts) > 1, False, up(rows, tile) * parts > CUS))
    return out


def ids_at_once(dl_rows, V, room):
    most = max(min(room // (2 * dl_rows) // IDS * IDS, MOST_IDS), IDS)
    return up(up(V, up(V, most)), IDS) * IDS


def gradient_ways(choice, sizes):
    """Per size (rows, d, V, whether dw has 32 bits), with the default workspace: the set of what it runs."""
    plans, questions = [], []
    for M, d, V, wide in sizes:
        questions.append(("P", 2 * M if M <= LOW_ROWS else M, d, min(V, 65536), 0))
    splits = [a[0] for a in choice.ask(questions)]
    questions = []
    for (M, d, V, wide), s in zip(sizes, splits):
        low = M <= LOW_ROWS or wide
        dl_rows, dx_rows = 2 * M if low else M, 2 * M if M <= LOW_ROWS else M
        each = ids_at_once(dl_rows, V, 4 * M * ids_at_once(2 * M, V, DL_BYTES))
        found = {("parts of dx", s > 1), ("parts of the vocabulary", each < V)}
        asked = []
        for n in {each, V % each or each} if each < V else {V}:
            whole = n // IDS * IDS if four_waves(d, IDS) else 0
            if whole:
                asked.append(("S", whole // IDS, d // 64, M, (1 << 31) - 1))
            if n > whole:
                tile, vocab_tiles = tile_rows(M), up(n - whole, IDS)
                parts = parts_of(up(M, tile), vocab_tiles, up(d, 64))
                found.add(("logits 8", low, tile, up(vocab_tiles, parts) > 1))
            asked.append(("X", d, min(dx_rows, 1 << 17), up(n, 64), s))
            asked.append(("W", d, n, up(dl_rows, 64), 1))
        plans.append((low, found, asked))
        questions += asked
    answers = dict(zip(questions, choice.ask(questions)))
    for low, found, asked in plans:
        for q in asked:
            a = answers[q]
            if q[0] == "S":
                found.add(("logits 4", low, a[0], up(q[1], a[2]) > 1))
            else:
                found.add(("dx" if q[0] == "X" else "dw", a[0], bool(a[1])))
    return [found for _, found, _ in plans]
