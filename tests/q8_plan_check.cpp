// Host-side answers of the 8-bit product's rule of sizes.
//
// Test infrastructure: compiles q8/gemm_q8_plan.h for the host and reads one product a line,
//   M N K ldx ldw x w room
// (x, w: addresses; room: bytes of workspace), and prints for each
//   shape splits tail full kt phases skewed bytes
// of the launch that the library would make (splits 1 and tail 0: whole K in every tile).
#include "gemm_q8_plan.h"

#include <cstdio>

int main() {
    using namespace pb;
    using namespace pb::q8;
    long long M, N, K, ldx, ldw, x, w, room;
    while (scanf("%lld %lld %lld %lld %lld %lld %lld %lld", &M, &N, &K, &ldx, &ldw, &x, &w, &room) == 8) {
        GemmQ8Params p{};
        p.M = (int)M; p.N = (int)N; p.K = (int)K; p.ldx = ldx; p.ldw = ldw;
        p.X = (const int8_t*)x; p.W = (const int8_t*)w;
        const Plan c = plan_of(p, (size_t)room);
        const Split sp = split_of(p, c);
        printf("%d %d %d %d %d %d %d %zu\n", c.shape, sp.splits, sp.tail, sp.full, sp.kt, sp.phases, skewed(p) ? 1 : 0, bytes_of(c));
    }
}
