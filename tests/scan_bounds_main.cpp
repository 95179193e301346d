// Host program: where the selective scan reads flags of slots, over blocks on both sides of a tile's length.
#include <cstdio>

#include "bload_selective.hpp"

int main()
{
    for (int T = 1; T <= 5 * bload::kTile; ++T)
        for (int t = 0; t < (T + bload::kTile - 1) / bload::kTile * bload::kTile; ++t) {
            const bload::LookSlots look = bload::look_slots(t, T);
            const bool inside = look.own >= 0 && look.own < T && look.front >= 0 && look.front < T;
            if (!inside || (t < T && (look.own != t || (t > 0 && look.front != t - 1)))) {
                std::printf("T %d t %d: own %d front %d\n", T, t, look.own, look.front);
                return 1;
            }
        }
    std::printf("scan bounds ok\n");
    return 0;
}
