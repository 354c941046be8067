// Selective state space scan: how a call is divided, and workspaces.
#include <algorithm>

#include "scan_common.hpp"

namespace ucd {
using namespace seq;

// The library's own buffers of states have NP of them to a channel, so that they are read in packs whatever N is.
// Segments: a launch is waves of 64 / lanes channels that walk over all tokens, and 1024 of them give every SIMD one.  With fewer, sequences are cut
// into segments that are scanned side by side, after a first launch over the states alone, which costs two thirds of the second; so much that four
// waves to a SIMD (Forward; Backward's registers leave room for two) are then worth it, down to segments of four tiles.  Times per token, channel and
// state (bf16, 16 states, 2048 tokens): Forward with 1024 waves 0.45 ps in one segment, with 512 0.90 in one and 0.54, 0.50 in four, eight; Backward 1.10,
// 2.2 and 1.13, 1.12.  The two meet at about 950 waves.
static void segments(const ucd_scan_t &d, int dir, ScanParams &p)
{
    const int lanes = scan_lanes(d);
    p.per_group = d.D / d.G;
    const int per_block = kWaves * 64 / lanes;
    p.blocks = (p.per_group + per_block - 1) / per_block;
    p.tiles = (d.L + kTile - 1) / kTile;
    const long waves = (long)d.B * d.G * ((p.per_group + 64 / lanes - 1) / (64 / lanes));
    long segs = 1;
    const long target = dir == UCD_SEQ_FWD ? 4096 : 2048;
    if (waves < 960) segs = std::max(1l, std::min({target / std::max(1l, waves), (long)p.tiles / 4, 64l}));
    p.seg_tiles = std::max(1, (int)((p.tiles + segs - 1) / segs));
    p.segs = std::max(1, (p.tiles + p.seg_tiles - 1) / p.seg_tiles);
}

static size_t round16(size_t n) { return (n + 15) / 16 * 16; }

void scan_params(const ucd_scan_t &d, const ucd_scan_in_t &in, int dir, void *ws, ScanParams &p)
{
    p.d = d;
    p.in = in;
    segments(d, dir, p);
    char *at = (char *)ws;
    if (p.segs > 1) {
        p.seg_state = (float *)at;
        at += round16((size_t)4 * d.B * p.segs * d.D * scan_states(d));
        p.seg_step = (float *)at;
        at += round16((size_t)4 * d.B * p.segs * d.D);
    }
    if (dir == UCD_SEQ_BWD) {
        p.part_bc = (float *)at;
        at += round16((size_t)4 * d.B * p.tiles * d.G * p.blocks * kTile * 2 * scan_states(d));
        p.part_w = (float *)at;
    }
}

size_t scan_ws_bytes(const ucd_scan_t &d, int dir)
{
    ScanParams p{};
    segments(d, dir, p);
    size_t n = p.segs > 1 ? round16((size_t)4 * d.B * p.segs * d.D * scan_states(d)) + round16((size_t)4 * d.B * p.segs * d.D) : 0;
    if (dir == UCD_SEQ_BWD)
        n += round16((size_t)4 * d.B * p.tiles * d.G * p.blocks * kTile * 2 * scan_states(d)) + (size_t)4 * d.B * p.segs * d.D * (d.N + 2);
    return n;
}

size_t scan_saved_bytes(const ucd_scan_t &d) { return (size_t)4 * d.B * ((d.L + kTile - 1) / kTile) * (kTile / kKeep) * d.D * scan_states(d); }

}  // namespace ucd
