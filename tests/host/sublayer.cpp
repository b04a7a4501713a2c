// Whether the selective scan's forwards on stdin, one a line (B T C G N train), go along whole
// sequences in one pass or in chunks; prints "one" or "chunks".
#include <cstdio>

#include "selective.hpp"

using namespace gspn;

int main()
{
    Workspace reserve;
    int B, T, C, G, N, train;
    while (scanf("%d %d %d %d %d %d", &B, &T, &C, &G, &N, &train) == 6) {
        SelectiveProblem p{};
        p.B = B, p.T = T, p.C = C, p.G = G, p.N = N;
        p.rs = train ? &reserve : nullptr;
        printf("%s\n", sel_one_pass(p) ? "one" : "chunks");
    }
    return 0;
}
