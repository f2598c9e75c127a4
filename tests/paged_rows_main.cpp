// The fp32 attention's view of a row, on the host: "columns shift T B q_start[0] .. q_start[B] kv_len[0] .. kv_len[B - 1]" in, a line "row branch keys tokens" out for
// every row of Q and every branch that a search may end at.  Host code only; nothing here launches.
#ifdef PAGED_ROWS_RUNTIME
extern "C" {
void* __hipRegisterFatBinary(void*) { return nullptr; }
void __hipRegisterFunction() {}
void __hipRegisterVar() {}
void __hipUnregisterFatBinary() {}
}
#else
#include "paged_attention.hip"
#include <cstdio>
#include <vector>

int main() {
    lotts::PagedParams p = {};
    while (scanf("%d %d %d %d", &p.columns, &p.shift, &p.T, &p.B) == 4) {
        std::vector<int32_t> start(p.B + 1), len(p.B);
        for (auto& v : start)
            if (scanf("%d", &v) != 1) return 1;
        for (auto& v : len)
            if (scanf("%d", &v) != 1) return 1;
        p.q_start = start.data();
        p.kv_len = len.data();
        for (int t = 0; t < p.T; ++t)
            for (int b = 0; b < p.B; ++b) {
                const lotts::Branch br = lotts::branch_at(p, b);
                printf("%d %d %d %d\n", t, b, lotts::keys_of_row(br, t), br.L);
            }
    }
    return 0;
}
#endif
