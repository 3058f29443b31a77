// What the tests call in a translated library, beside the operators themselves.
namespace emu {
Grid* grid;
Fiber* self;
int resident = 3, lost = 0, lost_message = 0;
uint64_t state = 1;
char report[200];
std::vector<std::pair<const char*, size_t>> regions;
std::function<void()> body;
}  // namespace emu
extern "C" {
// before a call: clusters at most, the seed of the schedule, the bulk copy and the message that never land (0: none)
void emu_begin(int resident, uint64_t seed, int lost, int lost_message)
{
    emu::lost_message = lost_message;
    emu::resident = resident;
    emu::state = seed * 0x9E3779B97F4A7C15ull + 1;
    emu::lost = lost;
    emu::report[0] = 0;
    emu::regions.clear();
}
void emu_region(const void* p, size_t bytes) { emu::regions.push_back({(const char*)p, bytes}); }
const char* emu_report() { return emu::report; }
}
