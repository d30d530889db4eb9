"""How attention calls are launched, from the header that plans them, compiled for the host."""
import os
import subprocess

from paper_2509_24859_amd import build

_SOURCE = r"""
#include <stdio.h>
#include "op_attention_plan.h"
using namespace harp::attention;
int main() {
    harp_attention g = {};
    long long tq, tk;
    int causal;
    while (scanf("%lld %lld %d %d %d %d %d", &tq, &tk, &g.batch, &g.heads, &g.kv_heads, &g.head, &causal) == 7) {
        g.tokens_q = tq, g.tokens_k = tk;
        const Plan plans[] = {plan_queries(256, &g, causal), plan_keys(256, &g, causal)};
        const long long joins[] = {(long long)query_joins(&g), (long long)tiles_of(tk, g.kv_heads, g.batch, kJoinRows)};
        for (int i = 0; i < 2; ++i)
            printf("%d %d %lld %lld %d %d %lld %lld\n", sizes_fit(&g), plans[i].waves, (long long)plans[i].tiles, (long long)plans[i].places(),
                   plans[i].shares, plans[i].paired, (long long)plans[i].heads_of_a_launch(g.kv_heads), joins[i]);
    }
}
"""
_NAMES = ("fits", "waves", "tiles", "places", "shares", "paired", "heads", "joins")


def plans(directory, calls):
    """For each (queries, keys, batch, heads, kv heads, head, causal): the plans of the passes over rows and over keys, on 256 compute units."""
    source, program = os.path.join(directory, "plan.cpp"), os.path.join(directory, "plan")
    with open(source, "w") as f:
        f.write(_SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(build.ROOT, "include"),
                           "-I", build.CSRC, source, "-o", program])
    lines = "\n".join(" ".join(str(int(x)) for x in call) for call in calls)
    out = subprocess.run([program], input=lines, capture_output=True, text=True, check=True).stdout.splitlines()
    rows = [dict(zip(_NAMES, map(int, line.split()))) for line in out]
    assert len(rows) == 2 * len(calls)
    return [(rows[2 * i], rows[2 * i + 1]) for i in range(len(calls))]
