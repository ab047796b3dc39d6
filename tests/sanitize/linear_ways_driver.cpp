// linear_ways_driver.cpp -- the way that each call in ways.txt takes by the
// library's plans (paper_2608_23048_amd/csrc/checks.cpp): lines "operation tokens
// rows cols packed" in, the same with the way behind it out.
#include "checks.hpp"

#include <cstdio>
#include <cstring>

using namespace roi;

static void print_cut(const Cut& c, bool copied)
{
    const long long rest = c.tm * c.tn - c.full;
    std::printf("%s%s%s\n", c.full > 0 ? " whole" : "", rest > 0 ? " cut" : "",
                copied ? " copied" : "");
}

int main()
{
    std::FILE* f = std::fopen("ways.txt", "r");
    if (!f) return 1;
    char op[16];
    long long t, r, c;
    int packed;
    while (std::fscanf(f, "%15s %lld %lld %lld %d", op, &t, &r, &c, &packed) == 5) {
        std::printf("%s %lld %lld %lld %d: ", op, t, r, c, packed);
        if (!std::strcmp(op, "linear")) {
            const LinearPlan p = plan_linear(t, r, c, packed != 0);
            if (p.few) {
                std::printf("few\n");
                continue;
            }
            const long long blocks = p.cut.full + (p.cut.tm * p.cut.tn - p.cut.full) * p.cut.splits;
            std::printf(p.cut.tile == 256 ? "256" : blocks <= kUnits ? "128 alone" : "128");
            print_cut(p.cut, p.x_bytes > 0);
        } else {
            const bool weight = !std::strcmp(op, "weight");
            const GradPlan p = weight ? plan_grad(r, c, t, true) : plan_grad(t, c, r, false);
            std::printf(p.ready ? "ready" : p.deep ? "deep" : p.cut.tile == 256 ? "256" : "128");
            print_cut(p.cut, p.dy_bytes > 0 || p.q_bytes > 0);
        }
    }
    std::fclose(f);
    std::printf("linear ways ok\n");
    return 0;
}
