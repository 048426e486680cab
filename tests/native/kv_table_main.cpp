// Which entries of a page table the cache's kernels read ahead of their use: prints, for lengths on the command
// line, the last entry, and whether it is read from the table or from the place of a sequence without a slot.
// Usage: kv_table <page shift> <table width> <length>...
#include <cstdio>
#include <cstdlib>

#include "svf_kv_device.h"

int main(int argc, char** argv) {
    static int32_t table[3 * 100], nothing;
    svfk::KvView kv = {};
    kv.table = table;
    kv.table_stride = 100;
    kv.shift = std::atoi(argv[1]);
    kv.width = std::atoi(argv[2]);
    for (int i = 3; i < argc; i++) {
        const svfk::Table t = svfk::table_of(kv, 2, std::atoi(argv[i]), &nothing);
        std::printf("%d %d\n", t.last, t.base == (uint64_t)(table + 200) ? 1 : t.base == (uint64_t)&nothing ? 0 : -1);
    }
    return 0;
}
