"""How attention over shared prefixes shares its work out, walked on the CPU: the header that the kernel takes it from also compiles
for the host.  Every share of a prefix and of a sequence is taken once, no workgroup is without work, and shares that the plan lays side by
side are not taken one behind the other."""
import os
import random
import subprocess

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("share_walk") / "share_walk")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-Wno-unknown-pragmas", "-I" + os.path.join(ROOT, "include"),
                           "-I" + os.path.join(ROOT, "paper_2509_10798_amd", "csrc"), os.path.join(ROOT, "tests", "share_walk.cpp"), "-o", exe])

    def run(calls):
        """calls: (n_layers, h_kv, query rows of a sequence, prefixes, members, sequences); (prefix shares, own shares, workgroups, tiles) of each."""
        text = "".join("%d %d %d %d %s %s\n" % (nl, h, rows, len(pre), " ".join("%d %d" % x for x in zip(pre, members)), " ".join(map(str, own)))
                       for nl, h, rows, pre, members, own in calls)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300)
        lines = r.stdout.splitlines()
        assert r.returncode == 0 and len(lines) == len(calls), "ended (%d) at %s" % (r.returncode, str(calls[min(len(lines), len(calls) - 1)])[:200])
        for call, line in zip(calls, lines):
            assert line.startswith("ok"), (line, str(call)[:300])
        return [tuple(map(int, line.split()[1:])) for line in lines]
    return run


def _call(rng):
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    members = [log(1, 30) for _ in range(log(1, 40))]
    while sum(members) > 128:
        members.pop()
    members = members or [1]
    return (rng.choice([1, 1, 1, 2, 7, 32]), rng.choice([1, 2, 3, 4, 5, 8, 16]), log(1, 100), [log(1, 60000) for _ in members], members,
            [log(1, 4000) for _ in range(sum(members))])


@pytest.mark.parametrize("h_kv", [1, 2, 4, 5])
def test_several_prefixes_of_few_heads(walk, h_kv):
    """Shares that do not come in eights: counted with room for eight each, three prefixes of 2 heads took more workgroups than run at a time, and
    shares planned side by side came one behind the other."""
    rng = random.Random(h_kv)
    walk([(1, h_kv, 4, [rng.randint(3000, 40000) for _ in range(3)], [4, 8, 2], [rng.randint(30, 900) for _ in range(14)]) for _ in range(300)])


def test_one_prefix_a_sequence(walk):
    """128 prefixes of one head: 128 shares side by side with those of the sequences, not a thousand workgroups of which one in eight has work."""
    assert walk([(1, 1, 4, [200] * 128, [1] * 128, [100] * 128)]) == [(128, 128, 256, 1)]


def test_any_call(walk):
    rng = random.Random(11)
    walk([_call(rng) for _ in range(4000)])
