// How the paged attention kernels cut a call's chunks into runs, and find their way through the entries: plain arithmetic,
// the same on host and device.
//
// The loading warps read the entries' lengths where they need them, those of more than 32 entries several times.  A caller
// must not change them meanwhile; if one does, what was read does not add up, and the bounds here keep the kernels within
// their arrays and end them.
#pragma once

#ifdef __CUDACC__
#define MKV_BOTH __host__ __device__ __forceinline__
#else
#define MKV_BOTH inline
#endif

namespace mkv {

// `total` chunks in `runs` runs, the first total % runs of them one longer.
struct Runs {
  int runs, len, longer;
  MKV_BOTH Runs(int total, int grid) {
    runs = total < grid ? total : grid;
    len = runs > 0 ? total / runs : 0;
    longer = total - len * runs;
  }
  MKV_BOTH int start(int i) const { return i * len + (i < longer ? i : longer); }
  MKV_BOTH int of(int chunk) const {                      // the run that holds a chunk
    const int split = longer * (len + 1);
    return chunk < split ? chunk / (len + 1) : longer + (chunk - split) / len;
  }
};

// A unit that several runs share: the first one's run, the place of its piece (runs have two, for their first piece and for
// their last), and how many pieces there are: all of runs that exist.
struct Shares {
  int first, place0, count;
  MKV_BOTH Shares(const Runs& rs, int unit0, int chunks) {
    first = rs.of(unit0);
    place0 = 2 * first + (rs.start(first) < unit0 ? 1 : 0);
    const int last = rs.of(unit0 + chunks - 1);
    count = (last < rs.runs ? last : rs.runs - 1) - first + 1;
  }
};

// From entry b, whose `held` chunks (of all key heads) begin at `base`, on to the entry that holds chunk `cur` >= base:
// held = chunks_of(b) looks up the next one.  False if none of the B entries does.
template <typename Chunks>
MKV_BOTH bool walk_to(int cur, int B, int& b, int& base, int& held, Chunks chunks_of) {
  while (cur >= base + held) {
    base += held;
    if (++b >= B) return false;
    held = chunks_of(b);
  }
  return true;
}

}  // namespace mkv
