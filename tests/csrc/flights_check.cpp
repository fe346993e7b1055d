// Runs a CTA's copies against a model of its mbarriers (PTX: a wait for a parity
// is over when the phase of that parity is, that is unless the running phase has
// it) and gives up in the middle: prints how often a copy was still on its way
// when the waits ended, how often a lost copy was not noticed, and how often a
// wait for either parity would have waited.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "kv_flights.h"

struct Bar {
    unsigned phase = 0;      // completed phases
    bool flying = false;
    bool over(unsigned parity) const { return (phase & 1u) != parity; }
};

int main(int argc, char** argv) {
    const int runs = atoi(argv[1]);
    srand(1);
    long early = 0, unnoticed = 0, either = 0, waited = 0, lost_runs = 0;
    for (int run = 0; run < runs; ++run) {
        const int n = 1 + rand() % 4;
        std::vector<Bar> bars(n);
        soniq::Flights f;
        const int copies = rand() % 12;
        for (int j = 0; j < copies; ++j) {
            Bar& b = bars[j % n];
            if (b.flying) {      // a stage is issued again only when its copy has come
                b.flying = false;
                ++b.phase;
            }
            b.flying = true;
            f.issue(j % n, j / n & 1u);
            const int s = rand() % n;
            if (bars[s].flying && rand() % 2) {
                bars[s].flying = false;
                ++bars[s].phase;
            }
        }
        // some copies are lost for good, the others come one at a time while the CTA polls
        std::vector<bool> lost(n);
        bool any = false;
        for (int s = 0; s < n; ++s) {
            lost[s] = bars[s].flying && rand() % 8 == 0;
            any = any || lost[s];
        }
        for (int s = 0; s < n; ++s)
            if (bars[s].flying && !bars[s].over(0) && !bars[s].over(1)) ++either;
        int polls = 0;
        const bool ok = f.land([&](int s, unsigned parity) { return bars[s].over(parity); },
                               [&]() {
                                   ++waited;
                                   const int s = rand() % n;
                                   if (bars[s].flying && !lost[s]) {
                                       bars[s].flying = false;
                                       ++bars[s].phase;
                                   }
                                   return ++polls < 1000;
                               });
        lost_runs += any;
        if (any && ok) ++unnoticed;
        if (!any && !ok) ++early;
        if (ok)
            for (const Bar& b : bars)
                if (b.flying) ++early;
    }
    printf("%ld %ld %ld %ld %ld\n", early, unnoticed, either, waited, lost_runs);
}
