// Prints how the gated feed-forward block cuts up the shapes on standard input, a line each: M K F and an element's bytes.
#include <stdio.h>

#include "../../paper_2001_01347_amd/csrc/tr_cut.h"

static const char* tiles(bool large) { return large ? "large" : "small"; }

int main()
{
    long long M, K, F;
    int size;
    while (scanf("%lld %lld %lld %d", &M, &K, &F, &size) == 4) {
        const ForwardCut f = forward_cut(M, K, F, size, true);
        const Cut x = dx_cut(M, K, F, size), w = dw_cut(M, K, F, size);
        if (f.few) printf("few%d 1", f.few);
        else printf("%s %d", tiles(f.large), f.parts);
        printf(" %s %d %s %d\n", tiles(x.large), x.parts, tiles(w.large), w.parts);
    }
    return 0;
}
