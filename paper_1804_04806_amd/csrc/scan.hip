// Selective state space scan: how a call is divided, and workspaces.
#include <algorithm>

#include "scan_common.hpp"

namespace ucd {
using namespace seq;

// The library's own buffers of states have NP of them to a channel, so that they are read in packs whatever N is.
// Segments: a launch is waves of 64 / lanes channels that walk over all tokens, and 1024 of them give every SIMD one.  With fewer, sequences are cut
// into segments that are scanned side by side, after a first launch over the states alone, which costs two thirds of the second; so much that more
// waves to a SIMD are then worth it, for which the registers have room: two (Backward, and fp32) or four, of which three run at once (bf16; four and
// two measured 450 and 490 us for 16384 tokens of 4096 channels, but for fp32 564 and 577, and 43 and 39 us for 5 x 677 tokens of 770 channels).
// Segments have two tiles at least: a sequence of 256 tokens, 2048 channels takes 16 us, and 19 in segments of four tiles.  Times per token, channel
// and state (bf16, 16 states, 2048 tokens): Forward with 1024 waves 0.40 ps in one segment, with 512 0.8 in one and 0.46 in eight; Backward 0.98, 2.0
// and 1.05.  The two meet at about 950 waves.
static void segments(const ucd_scan_t &d, int dir, ScanParams &p)
{
    const int lanes = scan_lanes(d);
    p.per_group = d.D / d.G;
    const int per_block = kWaves * 64 / lanes;
    p.blocks = (p.per_group + per_block - 1) / per_block;
    p.tiles = (d.L + kTile - 1) / kTile;
    const long waves = (long)d.B * d.G * ((p.per_group + 64 / lanes - 1) / (64 / lanes)), groups = (long)d.B * d.G * p.blocks;
    long segs = 1;
    const long most = dir == UCD_SEQ_FWD && d.dtype == 1 ? 1024 : 512;      // workgroups
    if (waves < 960) segs = std::max(1l, std::min({most / std::max(1l, groups), (long)p.tiles / 2, 64l}));
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
