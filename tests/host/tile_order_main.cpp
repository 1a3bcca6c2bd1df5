// The places of tiles of many rows in the list that goes by the keys they see, against a sort in 64 bits: lengths from one token to the ends of
// int32, requests that are served and requests that are not.  Host code only.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2410_09687_amd/csrc/kv.h"

struct Tile {
    long long sees;
    int s, t, place;
};

static long long wrong = 0, steps = 0;

// kv as the caller gave it; asked: tokens as asked for; n: those that lie in the batch.
static void check(const std::vector<int> &kv, const std::vector<int> &asked, const std::vector<int> &n, const std::vector<bool> &pages, int group, int parts_most,
                  long long row_max, std::mt19937 &rng)
{
    const int S = (int)kv.size();
    std::vector<moin::KvListed> listed(S);
    std::vector<Tile> tiles;
    int total = 0;
    for (int s = 0; s < S; ++s) {
        const bool sane = kv[s] >= 0 && std::max(kv[s], 0) + (long long)asked[s] <= row_max, served = sane && pages[s];
        const int count = moin::kv_tiles_of(n[s], group), parts = served ? 1 + (int)(rng() % parts_most) : 1;
        listed[s] = moin::kv_listed(make_int4(std::max(kv[s], 0), served ? 3 : -1, 0, count > 0 ? total : -1), n[s], parts, group);
        for (int t = 0; t < count; ++t) {
            const long long rows = t ? (long long)(count - t) * moin::KV_TILE_ROWS : (long long)n[s] * group;
            tiles.push_back({(served ? kv[s] : 0) + (rows - 1) / group, s, t, 0});
        }
        total += count * parts;
    }
    std::stable_sort(tiles.begin(), tiles.end(), [](const Tile &a, const Tile &b) { return a.sees > b.sees; });   // (of equals the lower request, then the lower tile)
    int at = 0;
    for (const Tile &x : tiles) {
        int place = x.t * listed[x.s].parts;
        const int sees = moin::kv_tile_sees(listed[x.s], x.t, group);
        for (int i = 0; i < S; ++i)
            if (i != x.s) place += moin::kv_records_before(listed[i], sees, i < x.s, group);
        if (place != at && ++wrong <= 10)
            std::printf("S %d, group %d: tile %d of request %d (%d keys, %d tokens) at %d, not %d\n", S, group, x.t, x.s, kv[x.s], n[x.s], place, at);
        at += listed[x.s].parts;
    }
    ++steps;
}

int main()
{
    std::mt19937 rng(5);
    auto upto = [&](long long hi) { return (long long)(rng() % (unsigned long long)(hi + 1)); };
    const int top = 2147483647, groups[] = {1, 2, 3, 7, 8, 16, 32, 100, 255};
    for (int step = 0; step < 20000; ++step) {
        const int S = 1 + (int)upto(step % 10 ? 7 : 63), group = groups[upto(8)], most = (int)std::max<long long>(1, (step % 3 ? 700 : 20000) / group);
        const long long row_max = upto(1) ? top : 64LL * (1 + upto(200));
        std::vector<int> kv(S), asked(S), n(S);
        std::vector<bool> pages(S);
        for (int s = 0; s < S; ++s) {
            n[s] = (int)upto(most);
            asked[s] = upto(9) ? n[s] : (int)upto(top);   // (the batch ends in front of the others)
            const long long at[] = {0, upto(3000), top, top - upto(2LL * most), row_max - upto(most), row_max - n[s], top - n[s], -1 - upto(top)};
            kv[s] = (int)std::min<long long>(at[upto(step % 4 ? 7 : 1)], top);
            pages[s] = upto(5) > 0;
        }
        check(kv, asked, n, pages, group, 4, row_max, rng);
    }
    check({top, 0}, {100, 100}, {100, 100}, {true, true}, 8, 1, 1 << 20, rng);
    check({top - 100, top - 100}, {100, 100}, {100, 100}, {true, true}, 8, 1, top, rng);
    for (int group : groups)   // the most rows that a step may have, and a tile that sees all but the last token of them
        for (int back = 1; back < 300; ++back) {
            const int n = (top - moin::KV_TILE_ROWS) / group, tiles = moin::kv_tiles_of(n, group);
            const long long first = (long long)(n - back) * group / moin::KV_TILE_ROWS + 1;   // the first k whose row 128 k - 1 is of token n - back or later
            if (moin::kv_records_before(moin::KvListed{5, n, tiles, 1}, 5 + n - back, true, group) != 1 + tiles - first) ++wrong;
        }
    if (wrong) {
        std::printf("%lld places of tiles are wrong\n", wrong);
        return 1;
    }
    std::printf("tile places agree over %lld steps\n", steps);
    return 0;
}
