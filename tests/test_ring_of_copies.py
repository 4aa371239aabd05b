"""The numbers that go through a ring of places by copies, on the CPU: the kernels' own rules (which number is asked for next,
which phase it lands in, what is waited for before the end) on barriers and copies that keep to what mbarriers demand and land
in any order, one of them perhaps never.  No phase gets a second arrival, no number is taken for one that is not there, none is
asked for where readers are at work, and none is in flight at the end."""
import pytest

from .device_text import compiled, text_of

MODEL = r"""
#include <algorithm>
#include <climits>
#include <random>
#include <vector>
using std::max;
using std::min;
struct Place { int phase = 0, pending = 1, bytes = 0, holds = -1; };
struct Copy { int number, place; };
static std::vector<Place> places;
static std::vector<Copy> flying;
static std::mt19937 dice;
static int lost, broken;  // the number that never lands; the rules broken, as bits
enum { kTwice = 1, kEarly = 2, kRead = 4, kInFlight = 8 };

static void end_of(Place& p) {
    if (p.pending == 0 && p.bytes == 0) ++p.phase, p.pending = 1;
}
static void barrier_expect(uint32_t bar, uint32_t) {
    Place& p = places[bar / 8];
    if (p.pending == 0) broken |= kTwice;
    else --p.pending;
    ++p.bytes;
}
static bool land(int place = -1) {
    std::vector<int> can;
    for (int i = 0; i < static_cast<int>(flying.size()); ++i)
        if (flying[i].number != lost && (place < 0 || flying[i].place == place)) can.push_back(i);
    if (can.empty()) return false;
    const int i = can[dice() % can.size()];
    Place& p = places[flying[i].place];
    p.holds = flying[i].number, --p.bytes;
    flying.erase(flying.begin() + i);
    end_of(p);
    return true;
}
static bool passed(uint32_t bar, uint32_t parity) { return ((places[bar / 8].phase + 1) & 1) == static_cast<int>(parity); }
static bool barrier_wait(uint32_t bar, uint32_t parity) {
    while (dice() % 2 == 0 && land()) {}
    // a second goes by, in which what this barrier waits for lands, or never does, and the others perhaps no sooner than
    // somebody waits for them
    if (!passed(bar, parity)) land(bar / 8);
    return passed(bar, parity);
}
static bool barrier_wait_warp(uint32_t bar, uint32_t parity) { return barrier_wait(bar, parity); }
"""

BODY = r"""
// `count` numbers through a ring of kStages.  Returns the rules that were broken.
}
template <int kStages, int kBehind>
static int work(int count, int never, int seed) {
    places.assign(kStages, Place()), flying.clear(), dice.seed(seed), lost = never, broken = 0;
    Numbers<kStages, kBehind> numbers{0};
    int done = -1;
    const auto bring = [&](int i) {
        if (i - kStages > done) broken |= kRead;  // readers are still at what lies there
        barrier_expect(numbers.bar(i), 1);
        flying.push_back({i, numbers.place(i)});
    };
    for (int i = 0; i < std::min(kStages, count); ++i) bring(i);
    for (int i = 0; i < count; ++i) {
        if (numbers.wait(i) && places[numbers.place(i)].holds != i) broken |= kEarly;
        done = i - kBehind;
        if (numbers.asks(i) && numbers.next(i) < count) bring(numbers.next(i));
    }
    numbers.drain(count);
    for (const Copy& c : flying)
        if (c.number != lost) broken |= kInFlight;
    return broken;
}
extern "C" {
int work_through(int stages, int count, int never, int seed) {
    return stages == 1 ? work<1, 0>(count, never, seed) : stages == 2 ? work<2, 1>(count, never, seed) : work<3, 1>(count, never, seed);
}
"""

TWICE, EARLY, READ, IN_FLIGHT = 1, 2, 4, 8
RINGS = [1, 2, 3]  # places: the block's norm forward (its readers are done at once) and backward, the recurrence's tiles


def _build(folder, *changes):
    text = text_of("blackwell.cuh", "Numbers")
    for a, b in changes:
        assert text.count(a) == 1, a
        text = text.replace(a, b)
    return compiled(folder, [MODEL, text], BODY)


def _broken(lib, stages, never=-1, counts=range(0, 31)):
    got = 0
    for count in counts:
        for seed in range(40):
            got |= lib.work_through(stages, count, never, seed)
    return got


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return _build(tmp_path_factory.mktemp("ring"))


@pytest.mark.parametrize("stages", RINGS)
def test_every_number_in_its_turn(lib, stages):
    assert _broken(lib, stages) == 0


@pytest.mark.parametrize("stages", RINGS)
@pytest.mark.parametrize("never", range(8))
def test_a_copy_that_never_lands(lib, stages, never):
    assert _broken(lib, stages, never) == 0


@pytest.mark.parametrize("change,stages,never,rule", [
    (("return i / kStages & 1", "return i / 2 & 1"), 1, -1, EARLY),  # another ring's parity
    (("barrier_wait(bar(i), parity(i))", "barrier_wait(bar(i), parity(i + kStages))"), 3, 4, IN_FLIGHT),
    (("barrier_wait(bar(i), parity(i));", "if (!barrier_wait(bar(i), parity(i))) break;"), 3, 4, IN_FLIGHT),
    (("max(lost - kBehind, 0) + kStages)", "max(lost - kBehind, 0))"), 3, 4, IN_FLIGHT),
    (("return i - kBehind + kStages", "return i + kStages"), 2, -1, READ),
    (("i >= kBehind && lost == INT_MAX", "i >= kBehind"), 3, 4, TWICE),
], ids=["parity", "parity at the end", "no wait behind one in vain", "another ring's last ones", "a place that is read",
        "a second arrival"])
def test_the_model_sees(tmp_path, change, stages, never, rule):
    assert _broken(_build(tmp_path, change), stages, never, range(8, 31)) & rule
