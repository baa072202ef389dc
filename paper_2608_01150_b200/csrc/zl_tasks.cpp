// Host scheduler of libzellige: lowers a placement (whole sequences + shard descriptors, each
// over a range of heads) into task tables and longest-first work lists.  Pure host code.
//
// Paper Section IV-D: the engine "lowers the placement into a rank-local schedule" and packs
// all whole sequences of a rank into one block-diagonal call beside the rank's shards; its
// second coalescing mode batches Ulysses sequences, which hold all tokens of a sequence for a
// subset of the heads.  The paper orders segments by decreasing split degree so that
// collectives line up across ranks; on one GPU there are no collectives, and the order that
// matters is the one that keeps a long sequence from finishing last, so items are sorted
// longest-first.
#include <algorithm>
#include <functional>
#include <map>
#include <tuple>
#include <utility>

#include "zl_internal.h"

namespace zl {

namespace {

struct Range {
    int64_t off, len;
    bool operator<(const Range& o) const { return std::tie(off, len) < std::tie(o.off, o.len); }
    bool operator==(const Range& o) const { return off == o.off && len == o.len; }
};

using HeadRange = std::pair<int32_t, int32_t>;  // [first, second)

// Ranges must be pairwise identical or disjoint.
bool identical_or_disjoint(std::vector<Range> r) {
    std::sort(r.begin(), r.end());
    r.erase(std::unique(r.begin(), r.end()), r.end());
    for (size_t i = 1; i < r.size(); ++i)
        if (r[i - 1].off + r[i - 1].len > r[i].off) return false;
    return true;
}

// Head by head, the ranges of the tasks that cover the head must be pairwise identical or disjoint,
// and tasks with an identical range must cover the same heads (they form one accumulation group:
// a range claimed by two different head sets would be written by two groups).  Empty ranges are
// ignored.  The heads are walked as the elementary intervals between the tasks' range ends.
bool ranges_consistent(const std::vector<Range>& rng, const std::vector<HeadRange>& heads) {
    std::vector<int32_t> cuts;
    for (size_t i = 0; i < rng.size(); ++i)
        if (rng[i].len > 0) { cuts.push_back(heads[i].first); cuts.push_back(heads[i].second); }
    std::sort(cuts.begin(), cuts.end());
    cuts.erase(std::unique(cuts.begin(), cuts.end()), cuts.end());
    for (size_t c = 0; c + 1 < cuts.size(); ++c) {
        const int32_t a = cuts[c], b = cuts[c + 1];
        std::vector<Range> sel;
        std::map<Range, HeadRange> owner;
        for (size_t i = 0; i < rng.size(); ++i) {
            if (rng[i].len == 0 || heads[i].first > a || heads[i].second < b) continue;
            sel.push_back(rng[i]);
            auto it = owner.emplace(rng[i], heads[i]);
            if (!it.second && it.first->second != heads[i]) return false;
        }
        if (!identical_or_disjoint(std::move(sel))) return false;
    }
    return true;
}

constexpr int32_t kSms = 148;  // of a B200

// Keys of a shared prefix per chunk, a whole number of key tiles.  `blocks` (head, row block) items per chunk run on the SMs
// of a B200 in rounds; an item costs its key tiles and about two more to begin and to end (Q, the first S, the join, the
// partial output).  Of the numbers of chunks with the least total, the smallest; a chunk has 512 keys at least, because a
// partial row costs as much traffic as two key rows.
int64_t prefix_chunk(int64_t blocks, int64_t prefix_len) {
    constexpr int64_t kItemTiles = 2, kMinKeys = 512, kMaxChunks = 256;
    const int64_t most = std::min<int64_t>(kMaxChunks, std::max<int64_t>(1, prefix_len / kMinKeys));
    int64_t best = 0, best_cost = INT64_MAX;
    for (int64_t n = 1; n <= most; ++n) {
        const int64_t chunk = (int64_t)align_up((size_t)((prefix_len + n - 1) / n), kTileKV);
        const int64_t cost = ((blocks * n + kSms - 1) / kSms) * (chunk / kTileKV + kItemTiles);
        if (cost < best_cost) { best_cost = cost; best = chunk; }
    }
    return std::max<int64_t>(best, kTileKV);
}

// Positions leave room for the padded rows of a last tile in 32-bit arithmetic.
constexpr int64_t kMaxPos = INT32_MAX - 4 * 128;

using GroupKey = std::tuple<int64_t, int64_t, int32_t, int32_t>;  // range offset, length, head range

// Query tiles of a forward item cost about this many key-tile steps to begin and to end (descriptors, Q, the first S, the output).
constexpr int64_t kItemSteps = 2;

// Blocks of `block` query rows of every (task, head), in the order of the tasks.
std::vector<WorkItem> forward_blocks(const Schedule& s, int32_t block) {
    std::vector<WorkItem> items;
    for (size_t ti = 0; ti < s.tasks.size(); ++ti) {
        const Task& t = s.tasks[ti];
        for (int32_t h = s.task_head_begin[ti]; h < s.task_head_begin[ti] + s.task_head_count[ti]; ++h)
            for (int32_t r = 0; r < t.q_len; r += block)
                items.push_back({(int32_t)ti, h, r, std::min(block, t.q_len - r)});
    }
    return items;
}

// Steps an item takes: blocks of two query tiles take a key tile per step, the few-rows kernel takes two key tiles for
// its one query tile.  `masked`: only the visible keys.
int64_t item_steps(const Schedule& s, const WorkItem& w, bool few, bool masked) {
    const Task& t = s.tasks[w.unit];
    const int32_t parts = w.rows >> kPartsShift, rows = w.rows & ((1 << kPartsShift) - 1), row0 = parts > 1 ? 0 : w.row0;
    const int32_t keys = masked ? visible_keys(s.task_pos[w.unit], t.kv_len, row0 + rows - 1) : t.kv_len;
    int64_t tiles = (keys + kTileKV - 1) / kTileKV;
    if (parts > 1) tiles = (tiles + parts - 1) / parts + 2;  // the join costs about a step
    return (few ? (tiles + 1) / 2 : tiles) + kItemSteps;
}

// Of up to `parts` pieces along the keys, as many as the task's slot has room for.
int32_t pieces(const Task& t, int32_t parts) { return parts < 2 || t.partial_slot < 0 ? 1 : std::min(parts, kTileQ / t.q_len); }

// `items` (of one row block each) in up to `parts` pieces along the keys.
std::vector<WorkItem> in_pieces(const Schedule& s, const std::vector<WorkItem>& items, int32_t parts) {
    std::vector<WorkItem> out;
    for (const WorkItem& w : items) {
        const int32_t n = pieces(s.tasks[w.unit], parts);
        if (n < 2) { out.push_back(w); continue; }
        for (int32_t i = 0; i < n; ++i) out.push_back({w.unit, w.head, i, w.rows | (n << kPartsShift)});
    }
    return out;
}

// Whether blocks of one query tile (`few` steps) beat blocks of two: a step of theirs loads twice the keys, so a tenth
// fewer steps is where they start to pay.  Measured, d 128, blocks of two -> blocks of one, us.  Chosen: causal order over 1560
// tokens, 12 heads, 25.6 -> 19.1; over 2500 + 300 + 900, 8 heads, 39.4 -> 26.0; capped scores over 4096 tokens, 4 heads, 73 -> 43.
// Not chosen: causal order over 4 x 1560, 12 heads, 41 -> 53; 1560 + 1560 + 3600 under cap and mask 78 -> 99; 16 x 512 30 -> 48; 9450
// tokens 247 -> 309.  Of 64 cases (16 batches, mask or slopes, cap or none) two got the slower blocks, both by 4 %.
bool few_rows_pay(int64_t few, int64_t two) { return few * 10 < two * 9; }

// Beyond this many items per SM the rounds are even enough, whatever their blocks.
constexpr size_t kEvenItems = 16 * kSms;

// Numbers of pieces worth trying: a piece has two key tiles at least.  One token against 9450 keys, one piece -> the chosen
// pieces: 2 heads 95 -> 19 us, 12 heads x 4 chunks 99 -> 49, 40 heads x 8 chunks 296 -> 280.
constexpr int32_t kPieces[] = {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
bool worth_trying(const Schedule& s, int32_t parts, size_t n_items) {
    int32_t longest = 0;
    for (const Task& t : s.tasks) longest = std::max(longest, t.kv_len);
    return parts * s.max_item_rows <= kTileQ && parts * 2 * kTileKV <= longest + 2 * kTileKV && parts * n_items <= kEvenItems;
}

// Deals items out to CTAs: their work differs (ragged lengths, under a mask from a tile to the whole row), and walking items
// i, i + grid, ... would give the first CTA the longest item of every round.  So the items, longest first, go to the CTA
// with the least work so far; one CTA per SM, or per item where there are fewer.  Returns the most steps of a CTA.
// Walking in turn -> dealt: causal order over 9450 tokens 286 -> 247 us; without a mask, 16 texts of up to 512 tokens, 12
// heads, 31.9 -> 30.5 us, gradients of 8 continuations of a shared prefix 167 -> 159 us.
// Every handle pays for this, so it takes constant time per item: items are sorted by counting, and as the least load never
// falls, the CTAs wait in queues by their load, of which the first that is not empty only moves up.
int64_t deal(const std::vector<WorkItem>& items, const std::vector<int64_t>& steps, int32_t n_sms, DealtList* out) {
    const size_t n = items.size();
    const int32_t ctas = (int32_t)std::min<size_t>(n_sms, n);
    out->begin.assign(ctas + 1, 0);
    out->items.resize(n);
    if (n == 0) return 0;
    int64_t total = 0, longest = 0;
    for (int64_t st : steps) { total += st; longest = std::max(longest, st); }
    // steps in units of 2^shift: very long items need no finer queues
    constexpr int64_t kMaxUnits = 1 << 14;
    int shift = 0;
    while ((total / ctas + longest) >> shift > kMaxUnits) ++shift;
    auto units = [&](size_t i) { return (int32_t)((steps[i] + ((int64_t)1 << shift) - 1) >> shift); };
    int32_t most_units = 0;
    int64_t total_units = 0;
    for (size_t i = 0; i < n; ++i) { most_units = std::max(most_units, units(i)); total_units += units(i); }
    std::vector<int32_t> place(most_units + 2, 0), order(n), owner(n);
    for (size_t i = 0; i < n; ++i) ++place[most_units - units(i) + 1];
    for (int32_t u = 0; u <= most_units; ++u) place[u + 1] += place[u];
    for (size_t i = 0; i < n; ++i) order[place[most_units - units(i)]++] = (int32_t)i;
    // queues of CTAs by load; no load exceeds the mean and one item more
    std::vector<int32_t> first((size_t)(total_units / ctas) + most_units + 2, -1), last(first.size(), -1), next(ctas);
    std::vector<int64_t> load(ctas, 0);
    for (int32_t c = 0; c < ctas; ++c) next[c] = c + 1 < ctas ? c + 1 : -1;
    first[0] = 0;
    last[0] = ctas - 1;
    size_t least = 0;
    for (int32_t i : order) {
        while (first[least] < 0) ++least;
        const int32_t c = first[least];
        first[least] = next[c];
        const size_t to = least + units(i);
        next[c] = -1;
        if (first[to] < 0) first[to] = c; else next[last[to]] = c;
        last[to] = c;
        load[c] += steps[i];
        owner[i] = c;
        ++out->begin[c + 1];
    }
    for (int32_t c = 0; c < ctas; ++c) out->begin[c + 1] += out->begin[c];
    std::vector<int32_t> at(out->begin.begin(), out->begin.end() - 1);
    for (int32_t i : order) out->items[at[owner[i]]++] = items[i];
    return *std::max_element(load.begin(), load.end());
}

// No deal of items with these steps takes fewer: the mean, or the longest item.
struct LeastSteps {
    int64_t total = 0, longest = 0, items = 0;
    void add(int64_t steps, int64_t times) { total += steps * times; longest = std::max(longest, steps); items += times; }
    int64_t of(int32_t n_sms) const {
        const int64_t ctas = std::max<int64_t>(1, std::min<int64_t>(n_sms, items));
        return std::max((total + ctas - 1) / ctas, longest);
    }
};

// The same for deal_forward(): its items without a list of them.
int64_t least_forward(const Schedule& s, bool few, int32_t parts, bool masked, int32_t n_sms) {
    LeastSteps least;
    const int32_t block = few ? kTileQ : kFwdBlockQ;
    for (size_t ti = 0; ti < s.tasks.size(); ++ti) {
        const Task& t = s.tasks[ti];
        for (int32_t r = 0; r < t.q_len; r += block) {
            const int32_t rows = std::min(block, t.q_len - r), n = pieces(t, parts);
            for (int32_t i = 0; i < n; ++i)
                least.add(item_steps(s, n < 2 ? WorkItem{(int32_t)ti, 0, r, rows} : WorkItem{(int32_t)ti, 0, i, rows | (n << kPartsShift)}, few, masked),
                          s.task_head_count[ti]);
        }
    }
    return least.of(n_sms);
}

// Forward list in `parts` pieces, or in blocks of one query tile (`few`) or two.
int64_t deal_forward(const Schedule& s, bool few, int32_t parts, bool masked, int32_t n_sms, DealtList* out) {
    std::vector<WorkItem> made;
    if (parts > 1) made = in_pieces(s, s.fwd_items, parts);
    else if (few && s.max_item_rows > kTileQ) made = forward_blocks(s, kTileQ);
    const std::vector<WorkItem>& items = made.empty() ? s.fwd_items : made;
    std::vector<int64_t> steps;
    steps.reserve(items.size());
    for (const WorkItem& w : items) steps.push_back(item_steps(s, w, few, masked));
    out->few = few;
    out->parts = parts;
    return deal(items, steps, n_sms, out);
}

// The forward list that finishes soonest.  Blocks and pieces that `out` has chosen before stay: later positions may suit
// others better, but launches captured before have to find lists of their kind and length.
void choose_forward(const Schedule& s, bool masked, int32_t n_sms, DealtList* out) {
    if (out->parts > 0) {
        deal_forward(s, out->few, out->parts, masked, n_sms, out);
        return;
    }
    const bool all_few = s.max_item_rows <= kTileQ;
    int64_t best = deal_forward(s, all_few, 1, masked, n_sms, out);
    if (all_few && !s.shared_prefix) {
        // numbers of pieces by the least they could take, and of equal ones the smaller first
        std::vector<std::pair<int64_t, int32_t>> tries;
        for (int32_t parts : kPieces) {
            if (!worth_trying(s, parts, s.fwd_items.size())) break;
            tries.push_back({least_forward(s, true, parts, masked, n_sms), parts});
        }
        std::sort(tries.begin(), tries.end());
        for (const auto& [least, parts] : tries) {
            if (least > best || (least == best && parts > out->parts)) continue;
            DealtList other;
            const int64_t most = deal_forward(s, true, parts, masked, n_sms, &other);
            if (most < best || (most == best && parts < out->parts)) { best = most; *out = std::move(other); }
        }
    } else if (!all_few && s.fwd_items.size() <= kEvenItems && few_rows_pay(least_forward(s, true, 1, masked, n_sms), best)) {
        DealtList other;
        if (few_rows_pay(deal_forward(s, true, 1, masked, n_sms, &other), best)) *out = std::move(other);
    }
}

// Backward list: an item's work is the query tiles that see its keys.  Without a mask it is left empty where items c,
// c + grid, ... of the longest-first list are within 3 % of it: neighbours then read the same queries at the same time.
// With one, where no item has more than one query tile (a token against a long past): there is nothing to even out, and
// the keys of such a handle are many (23,680 items of 40 heads x 75,600 keys took 1.5 ms to deal).
void deal_backward(const Schedule& s, bool masked, int32_t n_sms, DealtList* out) {
    if (masked && std::all_of(s.kv_groups.begin(), s.kv_groups.end(), [](const KvGroup& g) { return g.n_q_tiles <= 1; })) return;
    std::vector<int64_t> steps;
    steps.reserve(s.bwd_items.size());
    for (const WorkItem& w : s.bwd_items) {
        const KvGroup& g = s.kv_groups[w.unit];
        int64_t tiles = kItemSteps + g.n_q_tiles;
        for (int32_t j = 0; masked && j < g.n_tasks; ++j) {
            const int32_t ti = s.kv_group_tasks[g.task_begin + j];
            tiles -= std::min((s.tasks[ti].q_len + kTileQ - 1) / kTileQ, first_query(s.task_pos[ti], w.row0) / kTileQ);
        }
        steps.push_back(tiles);
    }
    if (masked) { deal(s.bwd_items, steps, n_sms, out); return; }
    if (steps.empty()) return;
    std::vector<int64_t> load(std::min<size_t>(n_sms, steps.size()), 0);
    LeastSteps least;
    for (size_t i = 0; i < steps.size(); ++i) { load[i % load.size()] += steps[i]; least.add(steps[i], 1); }
    const int64_t in_turn = *std::max_element(load.begin(), load.end());
    if (least.of(n_sms) * 100 > in_turn * 97) return;
    if (deal(s.bwd_items, steps, n_sms, out) * 100 > in_turn * 97) *out = DealtList();
}

// Work lists, launch phases and workspace layout from the tasks, query groups and kv groups.
void finish_schedule(Schedule* s) {
    for (KvGroup& g : s->kv_groups) {
        g.tile_begin = s->n_kv_tiles;
        s->n_kv_tiles += (g.kv_len + kTileKV - 1) / kTileKV;
    }

    // forward work list: (task, head of the task's range, query block), longest-first
    auto longest_first = [&](const WorkItem& a, const WorkItem& b) {
        const int32_t ka = s->tasks[a.unit].kv_len, kb = s->tasks[b.unit].kv_len;
        if (ka != kb) return ka > kb;
        if (a.rows != b.rows) return a.rows > b.rows;
        return std::tie(a.unit, a.head, a.row0) < std::tie(b.unit, b.head, b.row0);
    };
    s->fwd_items = forward_blocks(*s, kFwdBlockQ);
    std::stable_sort(s->fwd_items.begin(), s->fwd_items.end(), longest_first);
    for (int32_t c : s->task_head_count) s->all_heads = s->all_heads && c == s->n_heads;
    for (const WorkItem& w : s->fwd_items) s->max_item_rows = std::max(s->max_item_rows, w.rows);
    // backward work list: (kv group, head of the group's range, key tile); cost = total query rows served
    std::vector<int64_t> group_cost(s->kv_groups.size(), 0);
    for (size_t g = 0; g < s->kv_groups.size(); ++g)
        for (int32_t j = 0; j < s->kv_groups[g].n_tasks; ++j)
            group_cost[g] += s->tasks[s->kv_group_tasks[s->kv_groups[g].task_begin + j]].q_len;
    for (size_t g = 0; g < s->kv_groups.size(); ++g) {
        const int32_t t0 = s->kv_group_tasks[s->kv_groups[g].task_begin];
        for (int32_t h = s->task_head_begin[t0]; h < s->task_head_begin[t0] + s->task_head_count[t0]; ++h)
            for (int32_t r = 0; r < s->kv_groups[g].kv_len; r += kTileKV)
                s->bwd_items.push_back({(int32_t)g, h, r, std::min(kTileKV, s->kv_groups[g].kv_len - r)});
    }
    auto bwd_order = [&](const WorkItem& a, const WorkItem& b) {
        if (group_cost[a.unit] != group_cost[b.unit]) return group_cost[a.unit] > group_cost[b.unit];
        if (a.rows != b.rows) return a.rows > b.rows;
        return std::tie(a.unit, a.head, a.row0) < std::tie(b.unit, b.head, b.row0);
    };
    std::stable_sort(s->bwd_items.begin(), s->bwd_items.end(), bwd_order);
    // the same list in units of two key tiles, for the CTA-pair form of the main kernel
    for (size_t g = 0; g < s->kv_groups.size(); ++g) {
        const int32_t t0 = s->kv_group_tasks[s->kv_groups[g].task_begin];
        for (int32_t h = s->task_head_begin[t0]; h < s->task_head_begin[t0] + s->task_head_count[t0]; ++h)
            for (int32_t r = 0; r < s->kv_groups[g].kv_len; r += 2 * kTileKV)
                s->bwd_pair_items.push_back({(int32_t)g, h, r, std::min(2 * kTileKV, s->kv_groups[g].kv_len - r)});
    }
    std::stable_sort(s->bwd_pair_items.begin(), s->bwd_pair_items.end(), bwd_order);

    if (s->fwd_items.size() <= kEvenItems) choose_forward(*s, false, kSms, &s->fwd_all);
    if (s->bwd_items.size() <= kEvenItems) deal_backward(*s, false, kSms, &s->bwd_all);

    // one launch phase until the caller says otherwise
    s->fwd_task_phase.assign(s->tasks.size(), 0);
    s->bwd_group_phase.assign(s->kv_groups.size(), 0);
    s->fwd_phase_begin = {0, (int32_t)s->fwd_items.size()};
    s->bwd_phase_begin = {0, (int32_t)s->bwd_items.size()};
    s->bwd_pair_phase_begin = {0, (int32_t)s->bwd_pair_items.size()};

    // backward workspace over the padded query slots: fp32 dQ accumulator [dq_acc_rows, H, d], then one
    // 4 KB "augmentation" tile per (head, 128-row query tile) holding -LSE/scale and -D split
    // into bf16 pieces (see the backward preprocess kernel)
    s->ws_dq_acc_off = 0;
    s->ws_aug_off = align_up((size_t)s->dq_acc_rows * s->n_heads * s->head_dim * sizeof(float), 256);
    s->bwd_workspace_bytes = s->ws_aug_off + align_up((size_t)(s->q_pad_total / kTileQ) * s->n_heads * 4096, 256);
}

}  // namespace

zl_status build_schedule(const std::vector<InputTask>& in, int32_t n_shards, int32_t total_q, int32_t total_kv,
                         int32_t n_heads, int32_t head_dim, uint32_t flags, Schedule* s) {
    if (!s || n_shards < 0 || total_q < 0 || total_kv < 0 || n_heads <= 0) return ZL_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return ZL_ERR_UNSUPPORTED;

    *s = Schedule();
    s->n_heads = n_heads; s->head_dim = head_dim; s->total_q = total_q; s->total_kv = total_kv;

    // ---- per-descriptor checks; the whole region ends where the last whole sequence ends
    int64_t whole_end = 0;
    for (const InputTask& t : in) {
        if (t.q_len < 0 || t.kv_len < 0 || t.q_off < 0 || t.kv_off < 0) return ZL_ERR_INVALID_ARG;
        if ((int64_t)t.q_off + t.q_len > total_q || (int64_t)t.kv_off + t.kv_len > total_kv) return ZL_ERR_INVALID_ARG;
        if (t.head_begin < 0 || t.head_count < 1 || (int64_t)t.head_begin + t.head_count > n_heads)
            return ZL_ERR_INVALID_ARG;
        if (t.shard_idx >= n_shards) return ZL_ERR_INVALID_ARG;
        if (t.shard_idx < 0 && t.q_len > 0) whole_end = std::max<int64_t>(whole_end, (int64_t)t.q_off + t.q_len);
    }
    const size_t n_in = in.size();
    std::vector<bool> live(n_in, false);  // contributes a task (or part of a fused one)
    for (size_t i = 0; i < n_in; ++i) {
        const InputTask& t = in[i];
        if (t.q_len == 0) continue;
        if (t.shard_idx >= 0 && (t.q_off < whole_end || (t.kv_len > 0 && t.kv_off < whole_end))) return ZL_ERR_OVERLAP;
        live[i] = true;
    }

    std::vector<Range> q_rng(n_in), kv_rng(n_in);
    std::vector<HeadRange> heads(n_in);
    for (size_t i = 0; i < n_in; ++i) {
        q_rng[i] = live[i] ? Range{in[i].q_off, in[i].q_len} : Range{0, 0};
        kv_rng[i] = live[i] ? Range{in[i].kv_off, in[i].kv_len} : Range{0, 0};
        heads[i] = {in[i].head_begin, in[i].head_begin + in[i].head_count};
    }
    if (!ranges_consistent(q_rng, heads) || !ranges_consistent(kv_rng, heads)) return ZL_ERR_OVERLAP;
    // the same (query range, key range) twice on a common head
    {
        std::map<std::tuple<int64_t, int64_t, int64_t, int64_t>, std::vector<HeadRange>> seen;
        for (size_t i = 0; i < n_in; ++i) {
            if (!live[i] || in[i].kv_len == 0) continue;
            auto& v = seen[std::make_tuple(q_rng[i].off, q_rng[i].len, kv_rng[i].off, kv_rng[i].len)];
            for (const HeadRange& h : v)
                if (h.first < heads[i].second && heads[i].first < h.second) return ZL_ERR_OVERLAP;
            v.push_back(heads[i]);
        }
    }

    // ---- optional fusion of local chunks: a (query range, head range) whose non-empty key chunks, sorted
    // by offset, tile one contiguous interval needs no partials and no merge -- it is exact attention
    // over the interval, i.e. one task that is final after the forward launch.  Done for all such
    // ranges or for none: the fused intervals must still be consistent with every other key range.
    std::vector<int32_t> fuse_leader(n_in, -1);  // per input: first input of its fused range, or -1
    std::vector<Range> fuse_union(n_in, Range{0, 0});
    if (flags & ZL_BUILD_FUSE_LOCAL_CHUNKS) {
        std::map<GroupKey, std::vector<int32_t>> by_q;
        for (size_t i = 0; i < n_in; ++i)
            if (live[i] && in[i].shard_idx >= 0)
                by_q[GroupKey(q_rng[i].off, q_rng[i].len, heads[i].first, heads[i].second)].push_back((int32_t)i);
        std::vector<Range> eff_kv = kv_rng;
        for (auto& kvp : by_q) {
            std::vector<Range> chunks;
            for (int32_t i : kvp.second)
                if (in[i].kv_len > 0) chunks.push_back(kv_rng[i]);
            std::sort(chunks.begin(), chunks.end());
            bool contiguous = chunks.size() >= 2;
            for (size_t c = 1; c < chunks.size() && contiguous; ++c)
                contiguous = chunks[c - 1].off + chunks[c - 1].len == chunks[c].off;
            if (!contiguous) continue;
            const Range u{chunks.front().off, chunks.back().off + chunks.back().len - chunks.front().off};
            for (int32_t i : kvp.second) {
                fuse_leader[i] = kvp.second.front();
                fuse_union[i] = u;
                eff_kv[i] = (i == kvp.second.front()) ? u : Range{0, 0};
            }
        }
        if (!ranges_consistent(eff_kv, heads)) std::fill(fuse_leader.begin(), fuse_leader.end(), -1);
    }

    // ---- tasks: whole sequences in placement order, then shards in the caller's order
    s->whole_to_task.clear();
    s->shard_to_task.assign(n_shards, -1);
    s->shard_slot_off.assign(n_shards, 0);
    s->shard_slot_rows.assign(n_shards, 0);
    s->shard_kv_off.assign(n_shards, 0);
    s->shard_kv_len.assign(n_shards, 0);
    for (const InputTask& t : in)
        if (t.shard_idx >= 0) { s->shard_kv_off[t.shard_idx] = t.kv_off; s->shard_kv_len[t.shard_idx] = t.kv_len; }
    std::map<GroupKey, int32_t> merge_index;          // (query range, head range) -> merge group
    std::vector<std::vector<int32_t>> merge_members;  // task indices per group
    std::vector<int32_t> merge_seq;
    auto push_task = [&](const Task& t, const InputTask& src) {
        s->tasks.push_back(t);
        s->task_head_begin.push_back(src.head_begin);
        s->task_head_count.push_back(src.head_count);
    };
    for (size_t i = 0; i < n_in; ++i) {
        if (in[i].shard_idx < 0) s->whole_to_task.push_back(live[i] ? (int32_t)s->tasks.size() : -1);
        if (!live[i]) continue;
        const InputTask& d = in[i];
        Task t{};
        t.q_off = d.q_off; t.q_len = d.q_len; t.kv_off = d.kv_off; t.kv_len = d.kv_len;
        t.partial_slot = -1; t.q_slot = 0; t.kv_group = -1; t.dq_slot = 0;
        if (d.shard_idx < 0) {  // whole sequence: final after the forward launch
            push_task(t, d);
            continue;
        }
        if (fuse_leader[i] >= 0) {
            // fused query range: its first shard carries the task over the whole interval, final
            // after the forward launch; the other shards of the range add nothing
            if (fuse_leader[i] != (int32_t)i) {
                if (in[fuse_leader[i]].seq_id != d.seq_id) return ZL_ERR_INVALID_ARG;
                s->shard_to_task[d.shard_idx] = s->shard_to_task[in[fuse_leader[i]].shard_idx];
                continue;
            }
            t.kv_off = (int32_t)fuse_union[i].off; t.kv_len = (int32_t)fuse_union[i].len;
            s->shard_to_task[d.shard_idx] = (int32_t)s->tasks.size();
            push_task(t, d);
            ++s->n_fused_ranges;
            continue;
        }
        const GroupKey mk(d.q_off, d.q_len, d.head_begin, d.head_begin + d.head_count);
        auto it = merge_index.find(mk);
        if (it == merge_index.end()) {
            it = merge_index.emplace(mk, (int32_t)merge_members.size()).first;
            merge_members.emplace_back();
            merge_seq.push_back(d.seq_id);
        } else if (merge_seq[it->second] != d.seq_id) {
            return ZL_ERR_INVALID_ARG;
        }
        // slot padded to whole query tiles so a full-tile store of a ragged last tile can
        // never reach another task's slot
        const int32_t padded = (int32_t)align_up((size_t)d.q_len, kTileQ);
        t.partial_slot = (int32_t)s->partial_rows;
        s->shard_slot_off[d.shard_idx] = t.partial_slot;
        s->shard_slot_rows[d.shard_idx] = padded;
        s->partial_rows += padded;
        if (s->partial_rows > INT32_MAX) return ZL_ERR_INVALID_ARG;
        s->shard_to_task[d.shard_idx] = (int32_t)s->tasks.size();
        merge_members[it->second].push_back((int32_t)s->tasks.size());
        push_task(t, d);
    }

    // merge groups, in order of first appearance; parts in ascending shard order
    s->merge_row_prefix.push_back(0);
    for (size_t g = 0; g < merge_members.size(); ++g) {
        const int32_t t0i = merge_members[g][0];
        const Task& t0 = s->tasks[t0i];
        MergeGroup mg{};
        mg.q_off = t0.q_off; mg.q_len = t0.q_len;
        mg.part_begin = (int32_t)s->merge_parts.size(); mg.n_parts = (int32_t)merge_members[g].size();
        mg.head_begin = s->task_head_begin[t0i]; mg.head_count = s->task_head_count[t0i];
        for (int32_t ti : merge_members[g]) s->merge_parts.push_back(s->tasks[ti].partial_slot);
        s->merge_groups.push_back(mg);
        s->merge_row_prefix.push_back(s->merge_row_prefix.back() + t0.q_len);
    }

    // query groups (distinct query range x head range) and kv groups (distinct key range x head range)
    {
        std::map<GroupKey, int32_t> qg, kg;
        std::vector<std::vector<int32_t>> kmembers;
        for (size_t ti = 0; ti < s->tasks.size(); ++ti) {
            Task& t = s->tasks[ti];
            const int32_t hb = s->task_head_begin[ti], he = hb + s->task_head_count[ti];
            const GroupKey qk(t.q_off, t.q_len, hb, he);
            auto qi = qg.find(qk);
            if (qi == qg.end()) {
                qi = qg.emplace(qk, (int32_t)s->q_groups.size()).first;
                const int32_t pad = (int32_t)align_up((size_t)t.q_len, kTileQ);
                QGroup g{};
                g.q_off = t.q_off; g.q_len = t.q_len; g.slot = (int32_t)s->q_pad_total; g.pad = pad;
                g.head_begin = hb; g.head_count = he - hb;
                s->q_groups.push_back(g);
                s->q_pad_total += pad;
                if (s->q_pad_total > INT32_MAX) return ZL_ERR_INVALID_ARG;
            }
            t.q_slot = t.dq_slot = s->q_groups[qi->second].slot;
            if (t.kv_len == 0) continue;
            const GroupKey kk(t.kv_off, t.kv_len, hb, he);
            auto ki = kg.find(kk);
            if (ki == kg.end()) {
                ki = kg.emplace(kk, (int32_t)kmembers.size()).first;
                kmembers.emplace_back();
            }
            t.kv_group = ki->second;
            kmembers[ki->second].push_back((int32_t)ti);
        }
        for (size_t g = 0; g < kmembers.size(); ++g) {
            const Task& t0 = s->tasks[kmembers[g][0]];
            KvGroup kgp{t0.kv_off, t0.kv_len, (int32_t)s->kv_group_tasks.size(), (int32_t)kmembers[g].size(), 0, 0, t0.q_len, 0};
            for (int32_t ti : kmembers[g]) {
                s->kv_group_tasks.push_back(ti);
                kgp.n_q_tiles += (s->tasks[ti].q_len + kTileQ - 1) / kTileQ;
            }
            s->kv_groups.push_back(kgp);
        }
    }

    s->dq_rows = s->dq_acc_rows = s->q_pad_total;
    finish_schedule(s);
    return ZL_OK;
}

zl_status build_prefix_schedule(const int32_t* cu_q, const int32_t* cu_kv, int32_t n_seqs, int32_t prefix_len,
                                int32_t total_q, int32_t total_kv, int32_t n_heads, int32_t head_dim, Schedule* s) {
    if (!s || n_seqs < 0 || prefix_len < 0 || total_q < 0 || total_kv < 0 || n_heads <= 0) return ZL_ERR_INVALID_ARG;
    if (n_seqs > 0 && (!cu_q || !cu_kv)) return ZL_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return ZL_ERR_UNSUPPORTED;
    if (n_seqs > 0 && (cu_q[0] != 0 || cu_kv[0] != 0)) return ZL_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_seqs; ++i)
        if (cu_q[i + 1] < cu_q[i] || cu_kv[i + 1] < cu_kv[i]) return ZL_ERR_INVALID_ARG;
    const int32_t batch = n_seqs > 0 ? cu_q[n_seqs] : 0;
    if (batch > total_q || (int64_t)prefix_len + (n_seqs > 0 ? cu_kv[n_seqs] : 0) > total_kv) return ZL_ERR_INVALID_ARG;

    *s = Schedule();
    s->n_heads = n_heads; s->head_dim = head_dim; s->total_q = total_q; s->total_kv = total_kv;
    s->shared_prefix = true;
    s->shard_to_task.assign(n_seqs, -1);
    s->shard_slot_off.assign(n_seqs, 0);
    s->shard_slot_rows.assign(n_seqs, 0);
    s->shard_kv_off.assign(n_seqs, 0);
    s->shard_kv_len.assign(n_seqs, 0);
    for (int32_t i = 0; i < n_seqs; ++i) {
        s->shard_kv_off[i] = prefix_len + cu_kv[i];
        s->shard_kv_len[i] = cu_kv[i + 1] - cu_kv[i];
    }
    s->merge_row_prefix.push_back(0);
    if (batch == 0) { finish_schedule(s); return ZL_OK; }

    auto push_task = [&](int32_t q_off, int32_t q_len, int32_t kv_off, int32_t kv_len) -> zl_status {
        Task t{};
        t.q_off = q_off; t.q_len = q_len; t.kv_off = kv_off; t.kv_len = kv_len;
        t.kv_group = -1;
        t.dq_slot = q_off;  // the accumulator holds the batch's rows once, whichever task adds to them
        t.partial_slot = (int32_t)s->partial_rows;
        s->partial_rows += align_up((size_t)q_len, kTileQ);
        if (s->partial_rows > INT32_MAX) return ZL_ERR_INVALID_ARG;
        if (kv_len > 0) {
            t.kv_group = (int32_t)s->kv_groups.size();
            s->kv_groups.push_back(KvGroup{kv_off, kv_len, (int32_t)s->kv_group_tasks.size(), 1, (q_len + kTileQ - 1) / kTileQ, 0, q_len, 0});
            s->kv_group_tasks.push_back((int32_t)s->tasks.size());
        }
        s->tasks.push_back(t);
        s->task_head_begin.push_back(0);
        s->task_head_count.push_back(n_heads);
        return ZL_OK;
    };
    auto push_q_group = [&](int32_t q_off, int32_t q_len) -> zl_status {
        QGroup g{};
        g.q_off = q_off; g.q_len = q_len; g.slot = (int32_t)s->q_pad_total; g.pad = (int32_t)align_up((size_t)q_len, kTileQ);
        g.head_begin = 0; g.head_count = n_heads;
        s->q_groups.push_back(g);
        s->q_pad_total += g.pad;
        return s->q_pad_total > INT32_MAX ? ZL_ERR_INVALID_ARG : ZL_OK;
    };
    // The whole batch is one query range over the prefix, cut into chunks along the keys so that its (head, row
    // block, chunk) items fill the SMs.
    zl_status st = push_q_group(0, batch);
    if (st != ZL_OK) return st;
    const int64_t chunk = prefix_chunk((int64_t)n_heads * ((batch + kFwdBlockQ - 1) / kFwdBlockQ), prefix_len);
    int32_t n_chunks = 0;
    for (int64_t k = 0; k < prefix_len; k += chunk, ++n_chunks) {
        st = push_task(0, batch, (int32_t)k, (int32_t)std::min<int64_t>(chunk, prefix_len - k));
        if (st != ZL_OK) return st;
    }
    for (int32_t i = 0; i < n_seqs; ++i) {
        const int32_t ql = cu_q[i + 1] - cu_q[i], kl = cu_kv[i + 1] - cu_kv[i];
        if (ql == 0) continue;
        MergeGroup mg{};
        mg.q_off = cu_q[i]; mg.q_len = ql;
        mg.part_begin = (int32_t)s->merge_parts.size();
        mg.head_begin = 0; mg.head_count = n_heads;
        for (int32_t c = 0; c < n_chunks; ++c) s->merge_parts.push_back(s->tasks[c].partial_slot + cu_q[i]);
        if (kl > 0 || n_chunks == 0) {  // a row without any key still gets its empty partial
            const int32_t ti = (int32_t)s->tasks.size();
            st = push_task(cu_q[i], ql, prefix_len + cu_kv[i], kl);
            if (st != ZL_OK) return st;
            s->shard_to_task[i] = ti;
            s->shard_slot_off[i] = s->tasks[ti].partial_slot;
            s->shard_slot_rows[i] = (int32_t)align_up((size_t)ql, kTileQ);
            s->merge_parts.push_back(s->tasks[ti].partial_slot);
            s->tasks[ti].q_slot = (int32_t)s->q_pad_total;
            st = push_q_group(cu_q[i], ql);
            if (st != ZL_OK) return st;
        }
        mg.n_parts = (int32_t)s->merge_parts.size() - mg.part_begin;
        s->merge_row_group.insert(s->merge_row_group.end(), ql, (int32_t)s->merge_groups.size());
        s->merge_groups.push_back(mg);
        s->merge_row_prefix.push_back(s->merge_row_prefix.back() + ql);
    }
    // Only the batch's own rows (the first query group) are accumulated and converted.  A ragged tile of a nested range
    // adds zeros to the rows that follow it, up to one tile past the batch.
    s->dq_rows = s->q_groups[0].pad;
    s->dq_acc_rows = s->dq_rows + kTileQ;
    finish_schedule(s);
    return ZL_OK;
}

zl_status set_positions(Schedule* s, const int32_t* whole_prefix, const zl_shard_pos* shard_pos, int32_t n_sms) {
    const size_t n_shards = s->shard_to_task.size();
    if (n_shards > 0 && !shard_pos) return ZL_ERR_INVALID_ARG;
    // chunks of a shared prefix come before every sequence's own keys: seen by all
    std::vector<TaskPos> pos(s->tasks.size(), TaskPos{0, 0, s->shared_prefix ? INT32_MAX : 0, 0});
    for (size_t i = 0; i < s->whole_to_task.size(); ++i) {
        const int32_t prefix = whole_prefix ? whole_prefix[i] : 0;
        if (prefix < 0) return ZL_ERR_INVALID_ARG;
        if (s->whole_to_task[i] >= 0) pos[s->whole_to_task[i]].prefix = prefix;
    }
    std::vector<char> placed(s->tasks.size(), 0);
    for (size_t i = 0; i < n_shards; ++i) {
        const zl_shard_pos& sp = shard_pos[i];
        if (sp.q_pos < 0 || sp.kv_pos < 0 || sp.prefix < 0) return ZL_ERR_INVALID_ARG;
        const int32_t ti = s->shard_to_task[i];
        if (ti < 0 || s->shard_kv_len[i] == 0) continue;
        const Task& t = s->tasks[ti];
        const int64_t kv_pos = (int64_t)sp.kv_pos - (s->shard_kv_off[i] - t.kv_off);  // a fused task starts where its first chunk does
        if (kv_pos < 0 || (int64_t)sp.q_pos + t.q_len > kMaxPos || kv_pos + t.kv_len > kMaxPos) return ZL_ERR_INVALID_ARG;
        const TaskPos tp{sp.q_pos, (int32_t)kv_pos, sp.prefix, 0};
        if (placed[ti] && (pos[ti].q_pos != tp.q_pos || pos[ti].kv_pos != tp.kv_pos || pos[ti].prefix != tp.prefix))
            return ZL_ERR_INVALID_ARG;  // the chunks of a fused task are one stretch of one sequence
        pos[ti] = tp;
        placed[ti] = 1;
    }
    s->task_pos = std::move(pos);

    choose_forward(*s, true, n_sms, &s->fwd_masked);
    deal_backward(*s, true, n_sms, &s->bwd_masked);
    return ZL_OK;
}

}  // namespace zl
