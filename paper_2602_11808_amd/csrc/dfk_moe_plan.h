// Which forms of the tile kernel the experts of many rows run on, and when a workgroup of it looks ahead for its next tile.  Free of device code, so that a
// host program can check it.
#pragma once

namespace dfk {

// Rows of a row tile, by the rows that an expert has on the average, and 256 only with tiles for one and a half rounds of workgroups (an expert's last tile taken as half).
// Whole call, us, with 64 / 128 / 256:
//   19 rows (300 tokens, 8 of 128 experts of 2048 x 768) 238 / 235 / 274, 25 (100, 2 of 8 of 4096 x 4096) 147 / 162 / 206, 38 (300, 4 of 32 of 2888 x 1000) 176 / 155 / 186,
//   128 (1024, 8 of 64 of 2048 x 1024) 283 / 239 / 284, 175 (1400 tokens of these) 329 / 273 / 297, 200 (3000, 4 of 60 of 2304 x 1408) 528 / 421 / 419, 256 (2048, 8 of 64 of
//   2048 x 1024) 431 / 334 / 325;
//   94 tiles of 256 rows (2000 tokens, 1 of 8 of 2048 x 1024) 89 / 85 / 100, 214 (1200, 2 of 8 of 2048 x 2048) 148 / 119 / 131, 320 (4096, 2 of 16 of 1024 x 1024) 118 / 108 / 111,
//   378 (1000, 2 of 8 of 4096 x 4096) 425 / 352 / 337.
// With rows off the cache lines, which 128 rows take by their lines: 13 rows (200, 4 of 60 of 2888 x 1000) 242 / 208 / -, 25 (400, 4 of 64 of 2056 x 1000) 211 / 174 / -, 250 (2000, 4 of 32 of
//   2888 x 1000) - / 310 / 325, 500 (4000 tokens of these) - / 510 / 475.
constexpr int experts_tile_rows(int M, int n_experts, int top_k, int d_model, int d_ff) {
    const bool on_lines = d_model % 64 == 0 && d_ff % 64 == 0;
    const long long slots = (long long)M * top_k, tiles = (slots / 256 + n_experts / 2) * ((d_ff + 127) / 128);
    return on_lines && slots < 28ll * n_experts ? 64 : slots < (on_lines ? 200ll : 300ll) * n_experts || tiles < 350 ? 128 : 256;
}

// Row tiles that there are at most.
constexpr int experts_max_tiles(int slots, int n_experts, int tile_rows) { return slots / tile_rows + (slots < n_experts ? slots : n_experts); }

// A form of k_experts: rows and columns of a tile, the steps that LDS holds, workgroups that a CU holds, rows off the cache lines by their own lines.
struct ExpertsForm { int bm, bn, ns, per_cu; bool lines; };
constexpr ExpertsForm kExpertsForms[] = {{64, 128, 3, 2, false}, {128, 128, 4, 1, true}, {128, 128, 4, 1, false}, {128, 256, 3, 1, false}, {256, 256, 2, 1, false}};
constexpr int kExpertsCus = 256;

// The form of a product with N columns (of gate, and as many of up) and K to sum over.  Half as wide where the tiles that there are at most, of 256 columns (128 of gate and up), would
// leave CUs without one.  Whole call, us, wide / narrow: 96 and 96 tiles (300 tokens, 2 of 8 experts of 2048 x 1024) 63 / 50, 176 and 88 (200, 4 of 16 of 1024 x 1024) 51 / 42,
// 176 and 176 (400, 2 of 16 of 2048 x 1024) 71 / 58; 256 tiles of gate and up (512, 2 of 8 of 2048 x 2048) 79 / 85.
constexpr int experts_form(int tile_rows, int max_tiles, int N, int K, bool gated) {
    const int columns = gated ? 128 : 256;
    return tile_rows == 64 ? 0 : tile_rows == 256 ? 4 : K % 64 != 0 ? 1 : (long long)max_tiles * ((N + columns - 1) / columns) <= 192 ? 2 : 3;
}
constexpr unsigned experts_grid(const ExpertsForm& f, int max_tiles, int N, bool gated) {
    const int columns = gated ? f.bn / 2 : f.bn;
    const long long tiles = (long long)max_tiles * ((N + columns - 1) / columns);
    return tiles < kExpertsCus * f.per_cu ? (unsigned)((tiles + 7) / 8 * 8) : (unsigned)(kExpertsCus * f.per_cu);
}

// What has to be in LDS behind a step's barrier: the next step, with lines the one after it too.  Steps whose loads may be under way when a wavefront waits for that.
constexpr int experts_newer_steps(int ns, bool lines) { return ns - (lines ? 3 : 2); }

// The look for the next tile, in four parts behind the barriers of different steps: part 0 asks for the tile's number (and
// gets it on the spot: the compiler waits where the one thread that asks joins the others), 1 for its words (one wavefront's asynchronous load into LDS), 2 reads
// them, 3 begins the tile's loads, whose first step is requested amid step steps - ns.  Each step requests one more step behind its part, and the wavefront waits by count: a wait that leaves
// the newest experts_newer_steps of them under way covers what is older, so the words are in LDS for sure only where as many steps lie between parts 1 and 2.
constexpr int experts_look_gap(int ns) { return experts_newer_steps(ns, false) > 1 ? experts_newer_steps(ns, false) : 1; }
// Steps a tile has to have; part that step s of `steps` does, or -1.
constexpr int experts_look_steps(int ns) { return ns + 2 + experts_look_gap(ns); }
constexpr int experts_look_part(int s, int steps, int ns) {
    const int gap = experts_look_gap(ns), at = s - (steps - experts_look_steps(ns));
    return at < 0 || at > 2 + gap || (at > 1 && at <= gap) ? -1 : at <= 1 ? at : at - gap + 1;
}

}  // namespace dfk
