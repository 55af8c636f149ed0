// Tiles of the group norm: which ones a call takes.
#include "norm_tile.h"
#include <algorithm>
#include <cstdint>
#include <numeric>

namespace kavg {

namespace {

constexpr int MOST_LANES = 1024;
constexpr int LANES = 512;                // two workgroups of them share a compute unit's registers
constexpr int64_t FULL = 256 * 1024;      // lanes that fill the device's 256 compute units
constexpr int64_t SUM_GROUPS = 512;       // workgroups of a round of sums: two per compute unit

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// LDS of the sums (whole tiles need no less)
size_t lds_bytes(const Tile& t, bool backward) {
    if (!backward) return (size_t)(2 * t.threads * (t.vec / t.gran) + 2 * t.units * t.groups) * sizeof(float);
    return (size_t)(2 * t.threads * t.vec + 2 * t.threads + t.units * (3 * t.channels + 2 * t.groups)) * sizeof(float);
}

bool finish(const NormCall& c, bool backward, Tile* t) {
    const int D = c.channels / c.groups;
    t->whole_rows = t->flat ? (int)(c.positions * c.channels / ((int64_t)t->cols * t->vec)) : t->rows / t->lane_rows;
    t->threads = (int)up((int64_t)t->units * t->cols * t->lane_rows, 64) * 64;
    t->by_unit = divisor(t->cols * t->lane_rows);
    t->by_cols = divisor(t->cols);
    t->by_d = divisor(D);
    t->by_per = divisor(D / t->gran);
    t->by_chunks = divisor(t->chunks);
    t->by_blocks = divisor(t->blocks);
    t->by_images = divisor((uint32_t)c.images);
    const int64_t tiles = up(c.sets * c.images, t->units) * t->blocks * t->chunks;
    if (tiles >= (int64_t)1 << 30 || c.sets * c.images >= (int64_t)1 << 30) return false;      // (the divisors' range)
    if (tiles * t->threads >= (int64_t)1 << 32) return false;                                  // (a launch's)
    t->lds = lds_bytes(*t, backward);
    return t->lds <= 160 * 1024;
}

// Packs per lane: the fewest of 1, 2, 4, .. `most` that bring an image (lanes_of packs) into a workgroup of at most `lanes`, 0 if none does;
// more of them where workgroups are plenty even so and lanes go down with it (one position has one pack per lane, however many images there are:
// 2048 vectors of 1024 in fp32, 16 packs / one, forward 19.5 us / 9.8; in bf16 11.9 / 6.9; backward, eight / one in fp32 40.0 / 32.9).
template <class LanesOf> int packs_per_lane(int most, int lanes, int64_t tiles, LanesOf lanes_of) {
    int nv = 1;
    while (nv <= most && lanes_of(nv) > lanes) nv *= 2;
    if (nv > most) return 0;
    while (nv < most && tiles * lanes_of(2 * nv) >= FULL && lanes_of(2 * nv) < lanes_of(nv)) nv *= 2;
    return nv;
}

// the two tiles of an image that is read twice, from `t`, which has everything but how an image is cut along its rows
bool twice(const NormCall& c, bool backward, const Tile& t, int64_t rows, NormTiles* n) {
    const int64_t images = c.sets * c.images;
    const int turn = backward ? GRAD_PACKS : SUM_PACKS;
    n->whole.nv = 0;
    n->sums = n->apply = t;
    n->sums.units = n->apply.units = 1;
    // Chunks: as many as make `round` rounds of the device's workgroups, for the number of rounds that costs least, in turns; a workgroup has
    // about two turns' work beside its turns.  (Four chunks of each of 132 images, 528 workgroups, are two rounds, three are one: of 11342
    // positions, 70 channels in bf16, forward 176 us and 159.)
    const int64_t turns = up(rows, (int64_t)turn * t.lane_rows), tiles = images * t.blocks, first = up(tiles, SUM_GROUPS);
    int64_t chunks = 1, least = INT64_MAX;
    for (int64_t round = first; round < first + 4; ++round) {
        const int64_t some = std::min(turns, round * SUM_GROUPS / tiles), cost = up(tiles * some, SUM_GROUPS) * (up(turns, some) + 2);
        if (cost < least) { least = cost; chunks = some; }
    }
    n->sums.nv = n->apply.nv = (int)(turn * up(turns, chunks));
    n->sums.chunks = n->apply.chunks = (int)up(rows, (int64_t)n->sums.nv * t.lane_rows);
    return finish(c, backward, &n->sums) && finish(c, backward, &n->apply);
}

bool rows_tiles(const NormCall& c, int vec, int elem, bool backward, NormTiles* n) {
    const int D = c.channels / c.groups;
    const int64_t least = std::lcm((int64_t)D, (int64_t)vec);          // channels of whole groups and whole packs
    if (least / vec > MOST_LANES || c.positions > (int64_t)1 << 30) return false;
    const int64_t images = c.sets * c.images, pieces = c.channels / least;
    Tile t = {};
    t.vec = vec;
    t.gran = std::gcd(D, vec);
    t.rows = (int)c.positions;
    const int most = backward ? backward_packs(t.gran, vec) : FORWARD_PACKS;
    // tiles of rows' segments of so many bytes, or of a piece if that is more
    const auto cut = [&](int64_t segment) {
        const int64_t blocks = up(pieces, std::max<int64_t>(1, segment / (elem * least))), per = up(pieces, blocks);
        t.channels = (int)(per * least);
        t.cols = t.channels / vec;
        t.groups = t.channels / D;
        t.blocks = (int)up(pieces, per);
    };
    const auto fit = [&](int lanes) {
        return packs_per_lane(most, lanes, images * t.blocks, [&](int nv) { return t.cols * up(c.positions, nv); });
    };
    // Short rows that are not made of lines: whole, if need be by a workgroup of all lanes (segments of them share lines; backward, us, whole /
    // in segments: 256 images of 784 positions, 40 channels in fp32 24 / 28, in bf16 20 / 25; but 64 of 196 positions, 320 in bf16 54 / 40).
    const int64_t row = (int64_t)c.channels * elem;
    if (row % 128 && row <= 256) {
        cut(row);
        t.nv = fit(MOST_LANES);
    }
    // Else segments of 128 bytes, or of 64 or 32 where only these bring an image into a workgroup of 512 lanes, so that two share a compute
    // unit (32x32x64 in bf16, backward: twice the segment for 1024 lanes 124 us against 112; 32x32x128, forward: half the segment for 256 lanes 129
    // against 111).  Then the same for 1024 lanes, but no 32 bytes: those cost more than reading the image twice (1225 positions, 64 channels in
    // groups of four, bf16, backward, us, whole / twice: 80 images 30 / 24, 1024 227 / 164; but in 64 bytes, 64 images of 1000, 256 channels,
    // 35 / 37, in 128, 64 of 2000, 512 channels, forward 73 / 90, 256 of 500, backward 119 / 141).
    for (const int lanes : {LANES, MOST_LANES})
        for (int64_t segment = 128; segment >= (lanes == LANES ? 32 : 64) && !t.nv; segment /= 2) { cut(segment); t.nv = fit(lanes); }
    if (t.nv) {
        t.lane_rows = (int)up(c.positions, t.nv);
        t.chunks = 1;
        t.units = (int)std::max<int64_t>(1, std::min<int64_t>(images, 256 / (t.cols * t.lane_rows)));
        n->whole = t;
        return finish(c, backward, &n->whole);
    }
    if (least / vec > LANES) return false;
    // Whole lines of a row (forward: two of 256x256x128 in bf16 128 bytes 24 us, 256 25).  Longer segments where no run of groups is made of lines
    // (backward: three images of 127x129, 320 channels in 32 groups, bf16: 80 bytes 52 us, 160 47, 320 44, 640 53), and in the backward pass where
    // a workgroup has many turns to go (128 bytes / 512: nineteen turns, nine images of 8964 positions, 512 channels in fp32, 183 / 167;
    // fourteen, three of 19162, 1024 in bf16, 127 / 120; eight, sixteen of 4096, 512 in bf16, 70 / 68; but four, four of 16384, 256, 34 / 37).
    const int64_t turns = images * c.positions * c.channels / vec / (SUM_GROUPS * LANES * GRAD_PACKS);
    cut(backward && turns >= 6 ? 512 : 128);
    if ((int64_t)t.channels * elem % 128) cut(512);
    t.lane_rows = std::max(1, LANES / t.cols);
    return twice(c, backward, t, c.positions, n);
}

bool flat_tiles(const NormCall& c, int vec, int most, bool backward, NormTiles* n) {
    const int period = c.channels / std::gcd(c.channels, vec);         // packs until the channels begin again
    const int64_t run = c.positions * c.channels, images = c.sets * c.images;
    if (period > LANES || images * run < vec || run > (int64_t)1 << 40) return false;
    const int64_t packs = up(run, vec);
    Tile t = {};
    t.flat = true;
    t.gran = 1;
    t.vec = vec;
    t.channels = c.channels;
    t.groups = c.groups;
    t.blocks = 1;
    t.lane_rows = 1;
    const auto lanes = [&](int nv) { return up(up(packs, nv), period) * period; };
    // (1024 lanes rather than two readings: 256 images of 784 positions, 45 channels in bf16, forward 21 us / 34; of 361, 33, backward 18.5 / 24)
    t.nv = packs_per_lane(most, LANES, images, lanes);
    if (!t.nv) t.nv = packs_per_lane(most, MOST_LANES, images, lanes);
    t.cols = (int)(t.nv ? lanes(t.nv) : LANES / period * period);
    const int64_t rows = up(packs, t.cols);
    if (rows > (int64_t)1 << 30) return false;
    t.rows = (int)rows;
    if (!t.nv) return twice(c, backward, t, rows, n);
    t.chunks = 1;
    t.units = (int)std::max<int64_t>(1, std::min<int64_t>(images, 256 / t.cols));
    n->whole = t;
    return finish(c, backward, &n->whole);
}

}  // namespace

bool norm_tiles(const NormCall& c, bool contiguous, bool backward, NormTiles* t) {
    const int elem = c.dtype == KAVG_BF16 ? 2 : 4, vec = 16 / elem;
    if (c.channels % vec == 0) return rows_tiles(c, vec, elem, backward, t);
    // packs of half the bytes rather than flat (3680 images of 85 positions, 380 channels in bf16, forward 133 us / 244; 64 of 1024, 100 channels 12.5 / 25.5,
    // backward 20 / 32; 4080 of 180, 12 channels, backward 22 / 33)
    if (c.channels % 4 == 0 && rows_tiles(c, 4, elem, backward, t)) return true;
    if (contiguous && flat_tiles(c, vec, backward ? backward_packs(1, vec) : FLAT_PACKS, backward, t)) return true;
    return rows_tiles(c, 1, elem, backward, t);
}

bool call_tiles(const NormCall& c, bool backward, NormTiles* t) {
    const int vec = c.dtype == KAVG_BF16 ? 8 : 4;
    const auto read_flat = [&](const Strides& s) { return s.row == c.channels && extent_of(c, s) >= vec; };
    return norm_tiles(c, read_flat(c.xs) && (!backward || read_flat(c.dys)) && c.outs.row == c.channels, backward, t);
}

size_t norm_workspace(const NormCall& c, const NormTiles& t, bool backward) {
    const size_t images = (size_t)(c.sets * c.images), groups = images * c.groups, chunks = t.whole.nv ? 1 : t.sums.chunks;
    if (!backward) return t.whole.nv ? 0 : (2 * groups * chunks + 2 * groups) * sizeof(float);
    return (images * chunks * 2 * c.channels + (t.whole.nv ? 0 : 2 * groups)) * sizeof(float);
}

}  // namespace kavg
