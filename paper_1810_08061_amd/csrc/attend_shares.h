// attend_shares.h -- a row's shares of the time axis in linear attention: which states the launches
// over them read and write.
#pragma once

namespace ldyn {

// Where a share's pass takes its state from: nowhere (behind the row's length), from the state that the call was given, or
// from its slot of the workspace.
enum class Start { NOTHING, GIVEN, SLOT };

// The shares of a row of L steps, `span` steps each; an empty row has its first.
constexpr int shares_used(int L, int span) { return L > span ? (L + span - 1) / span : 1; }

// The share whose pass leaves the row's state: the one that is gone through last.
constexpr bool ends_row(int share, int used, bool back) { return share == (back ? 0 : used - 1); }

// Whether another share takes up what this one adds to the state.
constexpr bool adds(int share, int used, bool back) { return share < used && !ends_row(share, used, back); }

// Where a row has several shares, the one that is gone through first has the given state from its slot too: the result may
// lie in the given state, and workgroups of one launch run in no order, so that state is read by the launch before, which
// joins the shares, and by no share whose row another one ends.
constexpr Start start_of(int share, int used) {
    return share >= used ? Start::NOTHING : used == 1 ? Start::GIVEN : Start::SLOT;
}

}  // namespace ldyn
