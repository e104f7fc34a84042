// Where the workgroups of attention over packed sequences find their rows: packed_attention.hpp's own find_rows and place_of for every slot of a launch.
// Reads launches from standard input, "Q causal M sequences offsets ..", and writes for each a line: "slots", then "slot start length tile alone" of every slot that has rows.
#include "lanes.hpp"

#include "packed_attention.hpp"

using namespace delta::pat;

template <int Q, bool CAUSAL>
static void slots_of_launch(const Args &a) {
    const int n = slots_of(a.M, a.seqs, Q);
    printf("%d", n);
    for (int slot = 0; slot < n; ++slot) {
        Rows found[64];
        bool there[64];
        lanes::run([&] { there[lanes::now] = find_rows<Q, CAUSAL>(a, n, slot, found[lanes::now]); });
        for (int l = 1; l < 64; ++l)
            if (there[l] != there[0] || (there[0] && memcmp(&found[l].start, &found[0].start, 3 * sizeof(int)))) { fprintf(stderr, "lanes differ\n"); abort(); }
        if (there[0]) printf(" %d %d %d %d %d", slot, found[0].start, found[0].len, found[0].tile, (int)found[0].alone);
    }
    printf("\n");
}
template <bool CAUSAL>
static void places(int units, int slots) {
    printf("places");
    for (unsigned i = 0, n = (unsigned)units * (unsigned)slots; i < n; ++i) {
        int unit, slot;
        place_of<CAUSAL>(i, n, units, slots, unit, slot);
        printf(" %d %d", unit, slot);
    }
    printf("\n");
}

int main() {
    long long q, causal, M, n;
    while (scanf("%lld %lld %lld %lld", &q, &causal, &M, &n) == 4) {
        if (q == 0) {                                    // M units, n slots
            causal ? places<true>((int)M, (int)n) : places<false>((int)M, (int)n);
            continue;
        }
        std::vector<long long> off((size_t)n + 1);
        for (long long &o : off)
            if (scanf("%lld", &o) != 1) return 1;
        Args a = {};
        a.off = off.data(); a.M = (int)M; a.seqs = (int)n;
        auto run = [&](auto size) {
            constexpr int Q = decltype(size)::value;
            causal ? slots_of_launch<Q, true>(a) : slots_of_launch<Q, false>(a);
        };
        if (q == 32) run(std::integral_constant<int, 32>());
        else if (q == 64) run(std::integral_constant<int, 64>());
        else if (q == 128) run(std::integral_constant<int, 128>());
        else if (q == 256) run(std::integral_constant<int, 256>());
        else return 1;
    }
    return 0;
}
