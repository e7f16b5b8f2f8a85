// The plan that rgd_paged_share leaves in the caller's memory (internal).
#pragma once
#include "paged.hpp"

namespace rgd {

// What the plan was made for.
struct PlanHead {
  int magic, S, n, Hq, Hkv, ps, D, width;
  RGD_DEV static PlanHead of(const PagedView& c, int n, int Hq) {
    return PlanHead{0x53684172, c.S, n, Hq, c.Hkv, c.ps, c.D, c.width};
  }
  RGD_DEV bool operator==(const PlanHead& o) const {
    return magic == o.magic && S == o.S && n == o.n && Hq == o.Hq && Hkv == o.Hkv && ps == o.ps && D == o.D &&
           width == o.width;
  }
};

// A group, at its first member; others have no tokens.
struct PlanGroup {
  int shared;  // positions, whole pages; 0: nothing
  int tokens;  // of all members
  int row;     // of its first token in the list
  int unused;
};

struct GroupAt {
  long long unit;
  int item, unused;
};

struct Plan {
  PlanHead* head;
  PlanGroup* group;  // [S]
  int* tokens;       // [S] new tokens
  int* shared;       // [S] positions that the sequence's group reads
  int* row;          // [S] the sequence's first token in the list
  int* leader;       // [S] the group's first member, or -1
  int* run;          // [S] leading pages in common with it
  int* rows;         // [S n] token rows, group by group
  __host__ __device__ Plan(int* p, int S)
      : head((PlanHead*)p), group((PlanGroup*)(p + 16)), tokens(p + 16 + 4 * S), shared(tokens + S), row(shared + S),
        leader(row + S), run(leader + S), rows(run + S) {}
  static size_t ints(int S, int n) { return 16 + 9 * (size_t)S + (size_t)S * n; }
};

}  // namespace rgd
