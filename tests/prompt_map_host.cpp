// Which workgroup of prompt attention takes which stretch, by the function that the kernels use: every stretch in use once, whatever part of the launch that is; the same
// number of them on every XCD, but for one; neighbours together.
#include <stdio.h>

#include <vector>

#include "../paper_2511_14617_amd/csrc/seer_prompt.h"

using namespace seer;

int main() {
    for (int launched = kXcds; launched <= 1024; launched += kXcds)
        for (int used = 0; used <= launched; ++used) {
            std::vector<int> taken(used + 1), on_xcd(kXcds), least(kXcds, used), most(kXcds, -1);
            for (int block = 0; block < launched; ++block) {
                const int w = stretch_of(block, used), xcd = block % kXcds;
                if (w < -1 || w >= used) return printf("launched %d, used %d: workgroup %d takes stretch %d\n", launched, used, block, w), 1;
                if (w < 0) continue;
                ++taken[w], ++on_xcd[xcd];
                if (w < least[xcd]) least[xcd] = w;
                if (w > most[xcd]) most[xcd] = w;
            }
            for (int w = 0; w < used; ++w)
                if (taken[w] != 1) return printf("launched %d, used %d: stretch %d taken %d times\n", launched, used, w, taken[w]), 1;
            for (int x = 0; x < kXcds; ++x) {
                if (on_xcd[x] < used / kXcds || on_xcd[x] > used / kXcds + 1) return printf("launched %d, used %d: %d on XCD %d\n", launched, used, on_xcd[x], x), 1;
                if (on_xcd[x] && most[x] - least[x] + 1 != on_xcd[x]) return printf("launched %d, used %d: gaps on XCD %d\n", launched, used, x), 1;
            }
        }
    return 0;
}
