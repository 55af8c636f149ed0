// Tiles of the group norm: which one a call takes.
#include "norm_tile.h"
#include <algorithm>
#include <numeric>

namespace kavg {

namespace {

constexpr int MOST_LANES = 1024;
constexpr int64_t FULL = 256 * 1024;      // lanes that fill the device's 256 compute units

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

size_t lds_bytes(const Tile& t, bool backward) {
    if (!backward) return (size_t)(2 * t.threads * (t.whole_pack ? 1 : t.vec) + 2 * t.units * t.groups) * sizeof(float);
    return (size_t)(2 * t.threads * t.vec + 2 * t.threads + 2 * t.units * (t.channels + t.groups)) * sizeof(float);
}

bool finish(Tile* t, const NormCall& c, bool backward) {
    t->threads = (int)up((int64_t)t->units * t->cols * t->lane_rows, 64) * 64;
    fastdiv_make(t->cols * t->lane_rows, &t->unit_m, &t->unit_s);
    fastdiv_make(t->cols, &t->col_m, &t->col_s);
    fastdiv_make(c.channels / c.groups, &t->d_m, &t->d_s);
    t->lds = lds_bytes(*t, backward);
    return t->lds <= 160 * 1024;
}

// Packs per lane: the fewest of 1, 2, 4, .. `most` that bring an image (lanes_of packs) into a workgroup of at most `lanes`, 0 if none does;
// more of them where workgroups are plenty even so.
template <class LanesOf> int packs_per_lane(int most, int lanes, int64_t tiles, LanesOf lanes_of) {
    int nv = 1;
    while (nv <= most && lanes_of(nv) > lanes) nv *= 2;
    if (nv > most) return 0;
    while (nv < most && tiles * lanes_of(2 * nv) >= FULL) nv *= 2;
    return nv;
}

bool rows_tile(const NormCall& c, int vec, int elem, int most, bool backward, Tile* t) {
    const int D = c.channels / c.groups;
    const int64_t least = std::lcm((int64_t)D, (int64_t)vec);          // channels of whole groups and whole packs
    if (least / vec > MOST_LANES / 2 || c.positions > (int64_t)1 << 30) return false;
    const int64_t images = c.sets * c.images, pieces = c.channels / least;
    t->flat = false;
    t->vec = vec;
    t->whole_pack = D % vec == 0;
    t->rows = (int)c.positions;
    // tiles of rows' segments of so many bytes, or of a piece if that is more
    const auto cut = [&](int64_t segment) {
        const int64_t blocks = up(pieces, std::max<int64_t>(1, segment / (elem * least))), per = up(pieces, blocks);
        t->channels = (int)(per * least);
        t->cols = t->channels / vec;
        t->groups = t->channels / D;
        t->blocks = (int)up(pieces, per);
    };
    t->nv = 0;
    for (const int lanes : {MOST_LANES / 2, MOST_LANES}) {
        for (int64_t segment = 128; segment >= 32 && !t->nv; segment /= 2) {
            cut(segment);
            t->nv = packs_per_lane(most, lanes, images * t->blocks, [&](int nv) { return t->cols * up(c.positions, nv); });
        }
        if (t->nv) break;
    }
    if (t->nv) {
        t->lane_rows = (int)up(c.positions, t->nv);
        t->chunks = 1;
        t->units = (int)std::max<int64_t>(1, std::min<int64_t>(images, 256 / (t->cols * t->lane_rows)));
    } else {
        cut(128);
        t->nv = most;
        t->lane_rows = std::max(1, MOST_LANES / 2 / t->cols);
        t->chunks = (int)up(c.positions, (int64_t)t->nv * t->lane_rows);
        t->units = 1;
    }
    return finish(t, c, backward);
}

bool flat_tile(const NormCall& c, int vec, int most, bool backward, Tile* t) {
    const int period = c.channels / std::gcd(c.channels, vec);         // packs until the channels begin again
    const int64_t run = c.positions * c.channels, images = c.sets * c.images;
    if (period > MOST_LANES || images * run < vec || run > (int64_t)1 << 40) return false;
    const int64_t packs = up(run, vec);
    t->flat = true;
    t->vec = vec;
    t->whole_pack = false;
    t->channels = c.channels;
    t->groups = c.groups;
    t->blocks = 1;
    t->lane_rows = 1;
    const auto lanes = [&](int nv) { return up(up(packs, nv), period) * period; };
    t->nv = packs_per_lane(most, MOST_LANES / 2, images, lanes);
    if (!t->nv) t->nv = packs_per_lane(most, MOST_LANES, images, lanes);
    t->cols = (int)(t->nv ? lanes(t->nv) : std::max(1, MOST_LANES / 2 / period) * period);
    if (!t->nv) t->nv = most;
    const int64_t rows = up(packs, t->cols);
    if (rows > (int64_t)1 << 30) return false;
    t->rows = (int)rows;
    t->chunks = (int)up(rows, t->nv);
    t->units = t->chunks > 1 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(images, 256 / t->cols));
    return finish(t, c, backward);
}

size_t bytes_of(const NormCall& c, const Tile& t, bool backward) {
    const size_t images = (size_t)(c.sets * c.images), groups = images * c.groups;
    if (!backward) return t.chunks == 1 ? 0 : (2 * groups * t.chunks + 2 * groups) * sizeof(float);
    return (images * t.chunks * 2 * c.channels + (t.chunks == 1 ? 0 : 2 * groups)) * sizeof(float);
}

}  // namespace

bool norm_tile(const NormCall& c, bool contiguous, bool backward, Tile* t) {
    const int elem = c.dtype == KAVG_BF16 ? 2 : 4, vec = 16 / elem, most = backward ? BACKWARD_PACKS : 16;
    if (c.channels % vec == 0) return rows_tile(c, vec, elem, most, backward, t);
    if (contiguous && flat_tile(c, vec, std::min(most, FLAT_PACKS), backward, t)) return true;
    return rows_tile(c, 1, elem, most, backward, t);
}

size_t norm_workspace(const NormCall& c, bool backward) {
    Tile t;
    size_t most = 0;
    for (const bool contiguous : {true, false})
        if (norm_tile(c, contiguous, backward, &t)) most = std::max(most, bytes_of(c, t, backward));
    return most;
}

}  // namespace kavg
